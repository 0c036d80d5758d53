"""moe_token_logprobs and its gradient on rows whose log-sum-exp is large: masks of the type's lowest value or of -1e9 throughout, rows far from
zero.  A binary32 lse does not hold log sum e^(x - max) beside a large maximum; the gradient's probabilities must add up to one all the same.

Tolerance, with e = 2^-24, relative to p: 16 e for exponentials and quotients, |x - lse| e for the exponent, the rounding of lse where it is taken as it
is (64 e; in bfloat16 2048 e), and a sum's additions (at most 64 in a lane for rows of up to 4096 logits, an eighth more than V / 256 beyond); the entropy
enters the gradient with its own error, 200 e (1 + log V) as in its own test.  A bfloat16 result rounds by 2^-8 of itself."""
import numpy as np
import pytest
import torch

from oracle import training as ot
from test_gpu_token_logprobs import DT, E, HALF, _f64

pytestmark = pytest.mark.gpu


def _rows(dtype, V, seed):
    g = torch.Generator().manual_seed(seed)
    low, high = torch.finfo(DT[dtype]).min, torch.finfo(DT[dtype]).max
    x = torch.randn(14, V, generator=g) * 2
    x[1] = low                                                       # nothing left, under a mask of the lowest value
    x[2] = -1e9                                                      # or of -1e9
    x[3] += 3000.0
    x[4] -= 3000.0
    x[5] += 70.0
    x[6] = high
    x[7] = -1e5 + 4096.0 * torch.randint(0, 2, (V,), generator=g)
    x[8] = low
    x[8, ::2] = -np.inf
    x[9] = 1e9
    x[9, 1:] = -1e9
    x[10] = -np.inf                                                  # nothing left at all
    x[11] = -np.inf
    x[11, 0] = low                                                   # one left
    x[12] -= 2e6
    x = x.to(DT[dtype])
    t = torch.randint(0, V, (14,), generator=g, dtype=torch.int32)
    t[4], t[9], t[11] = -1, 0, 0
    return x, t, torch.randn(14, generator=g), torch.randn(14, generator=g)


def _check(x, t, dl, de, dtype, d, H):
    xs, N, V = _f64(x), *x.shape
    tn, g, q = t.cpu().numpy(), _f64(dl), _f64(de)
    ref = ot.token_logprobs_backward(xs, tn, g, q)
    got = _f64(d)
    for n in range(N):
        top = xs[n].max()
        if top == -np.inf:
            assert (got[n] == 0).all()
            continue
        lp = xs[n] - top - np.log(np.exp(xs[n] - top).sum())
        p = np.exp(lp)
        on = p > 0
        gl = abs(g[n]) if 0 <= tn[n] < V else 0.0
        terms = (2048 if dtype == "bf16" else 64) + 16 + max(64, 9 * V // 2048)
        size = np.zeros(V)
        size[on] = p[on] * ((gl + abs(q[n]) * (np.abs(lp[on]) + H[n])) * (terms + np.abs(lp[on])) + abs(q[n]) * (200 * (1 + np.log(V)) + terms))
        if gl:
            size[tn[n]] += 2 * gl
        tol = HALF[dtype] * 1.001 * np.abs(ref[n]) + E * size + 1e-36
        over = np.abs(got[n] - ref[n]) / tol
        assert over.max() <= 1.0, (n, int(over.argmax()), over.max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 7, 60, 128, 250, 1000, 1500, 3001, 5000, 9001, 40000, 131073])
def test_rows_far_from_zero(dtype, V):
    import paper_2605_11537_amd as moe
    print(f"{dtype} V={V}", flush=True)
    x, t, dl, de = (v.cuda() for v in _rows(dtype, V, V))
    s = moe.moe_token_logprobs(x, t)
    want = ot.token_logprobs(_f64(x), t.cpu().numpy(), 0)
    with np.errstate(invalid="ignore"):
        bad = np.abs(_f64(s["entropy"]) - want["entropy"]) > 200 * E * (1 + np.log(V) + want["entropy"])
    assert not bad.any(), np.flatnonzero(bad)
    d = moe.moe_token_logprobs_backward(x, t, s["lse"], s["entropy"], dl, de)
    _check(x, t, dl, de, dtype, d, want["entropy"])
    # into rows that begin anywhere, and in place
    wide = torch.full((14, V + 9), 7.0, dtype=x.dtype, device="cuda")
    moe.moe_token_logprobs_backward(x, t, s["lse"], s["entropy"], dl, de, out=wide[:, 3:V + 3])
    _check(x, t, dl, de, dtype, wide[:, 3:V + 3], want["entropy"])
    assert (wide[:, :3] == 7).all() and (wide[:, V + 3:] == 7).all()
    at = x.clone()
    assert moe.moe_token_logprobs_backward(at, t, s["lse"], s["entropy"], dl, de, out=at) is at
    assert torch.equal(at, d)


def test_many_rows_among_others():
    """Far rows between ordinary ones: every row's gradient is what it is alone."""
    import paper_2605_11537_amd as moe
    for dtype, V in (("f32", 128), ("bf16", 3001), ("f32", 20000)):
        g = torch.Generator().manual_seed(V)
        x = torch.randn(500, V, generator=g)
        x[::3] -= 5000.0
        x[1::7] = torch.finfo(DT[dtype]).min
        x, t = x.to(DT[dtype]).cuda(), torch.randint(0, V, (500,), generator=g, dtype=torch.int32).cuda()
        dl, de = torch.randn(500, generator=g).cuda(), torch.randn(500, generator=g).cuda()
        s = moe.moe_token_logprobs(x, t)
        d = moe.moe_token_logprobs_backward(x, t, s["lse"], s["entropy"], dl, de)
        _check(x, t, dl, de, dtype, d, ot.token_logprobs(_f64(x), t.cpu().numpy(), 0)["entropy"])
        some = [0, 1, 2, 8, 9, 15, 498, 499]
        alone = moe.moe_token_logprobs_backward(x[some], t[some], s["lse"][some], s["entropy"][some], dl[some], de[some])
        assert torch.equal(alone, d[some])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 1000, 5000, 40000])
def test_a_padded_position_has_no_gradient(dtype, V):
    """Whatever its logits hold, where the entropy has no gradient either; with one, the row is one like the others."""
    import paper_2605_11537_amd as moe
    g = torch.Generator().manual_seed(V)
    x = torch.randn(6, V, generator=g).to(DT[dtype])
    x[1], x[2, V // 2], x[3] = np.nan, np.inf, -1e9
    t = torch.tensor([3, -1, V, -1, 5, -7], dtype=torch.int32)
    x, t, dl = x.cuda(), t.cuda(), torch.randn(6, generator=g).cuda()
    dl[1] = np.nan
    s = moe.moe_token_logprobs(x, t)
    assert (s["logprob"][[1, 2, 3, 5]] == 0).all()
    want = moe.moe_token_logprobs_backward(x, t, s["lse"], s["entropy"], dl)
    assert (want[[1, 2, 3, 5]] == 0).all() and torch.isfinite(want).all() and (want[0] != 0).any()
    de = torch.tensor([0.5, 0.0, 0.0, 0.0, 0.5, 0.5], device="cuda")
    d = moe.moe_token_logprobs_backward(x, t, s["lse"], s["entropy"], dl, de)
    assert (d[[1, 2, 3]] == 0).all() and torch.isfinite(d).all() and (d[5] != 0).any()
    de[1] = 0.5
    assert torch.isnan(moe.moe_token_logprobs_backward(x, t, s["lse"], s["entropy"], dl, de)[1]).all()
