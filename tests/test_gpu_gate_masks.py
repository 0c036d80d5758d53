"""moe_route_topk_backward on rows whose mask leaves nothing, little, or the lowest finite values, against float64.

Tolerance: an exponential, a quotient, a sum over at most 1024 places (16 in a lane, then a tree) and a mean of k terms, 64 * 2^-24 of the magnitudes that
enter; the logits that are left lie within 8 of each other, which adds 8 * 2^-24 to an exponential."""
import numpy as np
import pytest
import torch

from oracle import training as ot

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


@pytest.mark.parametrize("E,k", [(5, 2), (64, 1), (64, 3), (100, 3), (256, 8), (257, 2), (1024, 4)])
@pytest.mark.parametrize("renorm", [False, True])
def test_rows_whose_mask_leaves_nothing(E, k, renorm):
    import paper_2605_11537_amd as moe
    print(f"E={E} k={k} renorm={renorm}", flush=True)
    g = torch.Generator().manual_seed(E + k)
    T, low = 9, torch.finfo(torch.float32).min
    x = torch.rand(T, E, generator=g) * 4
    x[1] = -np.inf                                                   # nothing left
    x[2, 1:] = -np.inf                                               # one left
    x[3] = low                                                       # as good as equal
    x[4, ::2] = low
    x[5] = -1e9
    x[6, k:] = -np.inf                                               # the chosen ones left
    x[7, :k] = -np.inf                                               # the chosen ones masked
    idx = torch.arange(k)[:, None].expand(k, T).contiguous()         # a router's ids stand in falling order; the gradient takes any
    idx[:, 8] = -1                                                   # no choice made
    dw = torch.randn(k, T, generator=g)
    got = moe.moe_route_topk_backward(x.cuda(), idx.int().cuda(), dw.cuda(), renorm).double().cpu().numpy()
    assert (got[1] == 0).all() and (got[8] == 0).all()
    if renorm:
        assert (got[7] == 0).all()
    for s in (0, 2, 3, 4, 5, 6) if renorm else (0, 2, 3, 4, 5, 6, 7):
        row, i, d = x[s:s + 1].double().numpy(), idx[:, s:s + 1].numpy(), dw[:, s:s + 1].double().numpy()
        want = ot.route_backward(row, i, d, renorm)[0]
        p = np.exp(row[0] - row[0].max())
        p /= p.sum()
        w = ot.route_weights(row, i, renorm)[:, 0]
        mean = (w * np.abs(d[:, 0])).sum()
        size = np.zeros(E) if renorm else p * mean
        size[i[:, 0]] += w * (np.abs(d[:, 0]) + mean)
        assert (np.abs(got[s] - want) <= 72 * EPS * size + 1e-37).all(), s
    assert np.isfinite(got).all()


def test_a_nan_stays_in_its_row():
    import paper_2605_11537_amd as moe
    x = torch.zeros(3, 64)
    x[1] = -np.inf
    x[1, 7] = np.nan
    got = moe.moe_route_topk_backward(x.cuda(), torch.zeros(1, 3, dtype=torch.int32).cuda(), torch.ones(1, 3).cuda()).cpu()
    assert torch.isnan(got[1]).all() and torch.isfinite(got[[0, 2]]).all()


@pytest.mark.parametrize("E", [6, 64, 100, 300])
@pytest.mark.parametrize("renorm", [False, True])
def test_a_token_without_a_choice_has_no_gradient(E, renorm):
    """Whatever its logits hold: a padded token's are nobody's."""
    import paper_2605_11537_amd as moe
    g = torch.Generator().manual_seed(E)
    x = torch.randn(6, E, generator=g)
    x[1], x[2, 3], x[4, 0] = np.nan, np.inf, np.nan
    idx = torch.stack([torch.arange(6) % E, (torch.arange(6) + 1) % E]).int()
    idx[:, [1, 2]] = torch.tensor([-1, E], dtype=torch.int32)[:, None]
    dw = torch.randn(2, 6, generator=g)
    dw[:, 1] = np.nan
    got = moe.moe_route_topk_backward(x.cuda(), idx.cuda(), dw.cuda(), renorm).cpu()
    assert (got[[1, 2]] == 0).all() and torch.isfinite(got[[0, 3, 5]]).all()
    if not renorm:
        assert torch.isnan(got[4]).all()
