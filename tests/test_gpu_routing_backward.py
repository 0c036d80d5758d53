"""moe_combine_topk_backward, moe_dispatch_topk_backward and moe_route_topk_backward against oracle/training.py in float64.

Tolerances.  A product or a sum of up to nine terms rounded to dtype: half a unit of the result (2^-24, 2^-8 in bfloat16), and for the
sums 8 * 2^-24 of the terms' magnitudes before that rounding.  A dot product of d terms: no order of binary32 additions is off by more
than d * 2^-24 of the sum of magnitudes.  The gate: an exponential, a quotient and a mean of k terms, 32 * 2^-24 of the magnitudes that
enter (a sum of up to 1024 exponentials adds 16 more, 16 in a lane and then a tree), and what a difference of logits far apart was rounded by."""
import numpy as np
import pytest
import torch

from oracle import training as ot

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
EPS = 2.0 ** -24


def _f64(t):
    return t.double().cpu().numpy()


def _tables(T, k, drop, seed):
    """inv [k,T]: `drop` of the assignments without a row, the others on a permutation of the first rows."""
    g = np.random.default_rng(seed)
    a = np.flatnonzero(g.random(k * T) >= drop)
    inv = np.full(k * T, -1)
    inv[a] = g.permutation(len(a))
    return inv.reshape(k, T), len(a)


CASES = [
    (1, 1, 8, 0.0), (1, 1, 8, 1.0), (2, 8, 8, 0.3), (37, 1, 768, 0.1), (64, 3, 104, 0.3), (1000, 1, 128, 0.2), (257, 2, 256, 0.0), (130, 8, 512, 0.6),
    (5, 4, 4096, 0.2), (3, 2, 16392, 0.2), (2500, 3, 64, 0.5), (5000, 2, 48, 0.1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,k,d,drop", CASES)
def test_combine(dtype, T, k, d, drop):
    import paper_2605_11537_amd as moe
    g = torch.Generator().manual_seed(T + k + d)
    inv, K = _tables(T, k, drop, T + d)
    dt = DT[dtype]
    dout, y = torch.randn(T, d, generator=g).to(dt), torch.randn(k * T, d, generator=g).to(dt)
    w = torch.rand(k, T, generator=g)
    y[K:] = float("nan")                                             # rows that no token has are not read
    dev = [t.cuda() for t in (dout, y, torch.from_numpy(inv).int(), w)]
    for residual in (0, 1):
        want = ot.combine_backward(_f64(dout), _f64(y), inv, _f64(w), residual)
        out = dict(dy_perm=torch.full((k * T, d), 7.0, dtype=dt, device="cuda"), dweight=torch.full((k, T), 7.0, device="cuda"),
                   dx=torch.full((T, d), 7.0, dtype=dt, device="cuda"))
        got = moe.moe_combine_topk_backward(*dev, residual, out=out)
        assert (got["dy_perm"][K:] == 7).all()
        assert np.array_equal(_f64(got["dx"]), want["dx"])
        dy = _f64(got["dy_perm"])[:K]
        assert (np.abs(dy - want["dy_perm"][:K]) <= HALF[dtype] * 1.001 * np.abs(want["dy_perm"][:K])).all()
        size = ot.combine_backward(np.abs(_f64(dout)), np.abs(np.nan_to_num(_f64(y))), inv, _f64(w), residual)["dweight"]
        assert (np.abs(_f64(got["dweight"]) - want["dweight"]) <= d * EPS * size).all()
        alone = moe.moe_combine_topk_backward(dev[0], None, *dev[2:], residual, out=dict(dy_perm=torch.full_like(out["dy_perm"], 7.0), dweight=None, dx=None))
        assert torch.equal(alone["dy_perm"], got["dy_perm"])
        fresh = moe.moe_combine_topk_backward(*dev, residual)
        assert (fresh["dy_perm"][K:] == 0).all() and torch.equal(fresh["dy_perm"][:K], got["dy_perm"][:K])
        assert torch.equal(fresh["dweight"], got["dweight"]) and torch.equal(fresh["dx"], got["dx"])
    if k == 1:
        flat = moe.moe_combine_topk_backward(dev[0], dev[1], dev[2][0], dev[3][0], 1)
        assert flat["dweight"].shape == (T,) and torch.equal(flat["dweight"], got["dweight"][0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,k,d,drop", CASES)
def test_dispatch(dtype, T, k, d, drop):
    import paper_2605_11537_amd as moe
    g = torch.Generator().manual_seed(T + k + d)
    inv, K = _tables(T, k, drop, T + d)
    dt = DT[dtype]
    dxp, add = torch.randn(k * T, d, generator=g).to(dt), torch.randn(T, d, generator=g).to(dt)
    dxp[K:] = float("nan")
    for base in (None, add):
        want = ot.dispatch_backward(_f64(dxp), inv, None if base is None else _f64(base))
        size = ot.dispatch_backward(np.abs(np.nan_to_num(_f64(dxp))), inv, None if base is None else np.abs(_f64(base)))
        dev = base.cuda() if base is not None else None
        got = moe.moe_dispatch_topk_backward(dxp.cuda(), torch.from_numpy(inv).int().cuda(), dev)
        assert (np.abs(_f64(got) - want) <= HALF[dtype] * 1.001 * np.abs(want) + 8 * EPS * 1.01 * size).all()
        if base is not None:                                         # added in place
            same = moe.moe_dispatch_topk_backward(dxp.cuda(), torch.from_numpy(inv).int().cuda(), dev, out=dev)
            assert same is dev and torch.equal(same, got)


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (3, 2, 2), (64, 8, 1), (37, 60, 3), (257, 64, 8), (300, 65, 2), (1000, 128, 3), (130, 256, 1), (50, 300, 4), (33, 1024, 8)])
@pytest.mark.parametrize("renorm", [False, True])
def test_gate(T, E, k, renorm):
    import paper_2605_11537_amd as moe
    g = torch.Generator().manual_seed(T + E)
    logits = torch.randn(T, E, generator=g) * 3
    if E > 2 and k < E:
        logits[:, E // 2] = float("-inf")                            # an expert that is masked out
    if T > 2:
        logits[2] *= 30                                              # a gate that is as good as certain
        logits[1] += 1000.0
    dw = torch.randn(k, T, generator=g)
    idx = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k].t().contiguous()
    got = moe.moe_route_topk_backward(logits.cuda(), idx.int().cuda(), dw.cuda(), renorm)
    x, i, d = _f64(logits), idx.numpy(), _f64(dw)
    want = ot.route_backward(x, i, d, renorm)
    w = ot.route_weights(x, i, renorm)
    size = np.zeros((T, E))
    p = np.exp(x - x.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    # a difference from the largest logit is rounded once: relative to its exponential, EPS of the difference
    far = np.where(np.isfinite(x), x.max(1, keepdims=True) - x, 0.0)
    far_j = np.stack([far[np.arange(T), e] for e in i])
    mean, far_mean = (w * np.abs(d)).sum(0), (w * np.abs(d) * far_j).sum(0)
    if not renorm:
        size += p * (mean[:, None] * (48 + far) + far_mean[:, None])
    for j in range(k):
        size[np.arange(T), i[j]] += w[j] * ((np.abs(d[j]) + mean) * (48 + far_j[j]) + far_mean)
    assert (np.abs(_f64(got) - want) <= EPS * size + 1e-37).all()
    if k == 1:
        flat = moe.moe_route_topk_backward(logits.cuda(), idx[0].int().cuda(), dw[0].cuda(), renorm)
        assert torch.equal(flat, got)


def test_ids_outside_the_experts_are_choices_not_made():
    import paper_2605_11537_amd as moe
    g = torch.Generator().manual_seed(1)
    logits = torch.randn(4, 16, generator=g).cuda()
    idx = torch.tensor([[3, 3, 3, 3], [-1, 16, 5, 1 << 30]], dtype=torch.int32).cuda()
    dw = torch.randn(2, 4, generator=g).cuda()
    for renorm in (False, True):
        got = moe.moe_route_topk_backward(logits, idx, dw, renorm)
        one = moe.moe_route_topk_backward(logits, idx[:1].contiguous(), dw[:1].contiguous(), renorm)
        assert torch.equal(got[[0, 1, 3]], one[[0, 1, 3]]) and not torch.equal(got[2], one[2])


def test_shapes_that_do_not_fit_are_refused():
    import paper_2605_11537_amd as moe
    f = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")
    inv = f(2, 6, dt=torch.int32)
    with pytest.raises(ValueError, match="y_perm"):
        moe.moe_combine_topk_backward(f(6, 8), f(6, 8), inv, f(2, 6))
    with pytest.raises(ValueError, match="inv"):
        moe.moe_combine_topk_backward(f(6, 8), f(12, 8), inv.long(), f(2, 6))
    with pytest.raises(ValueError, match="expert_weight"):
        moe.moe_combine_topk_backward(f(6, 8), f(12, 8), inv, f(2, 6, dt=torch.bfloat16))
    with pytest.raises(ValueError, match="dx_perm"):
        moe.moe_dispatch_topk_backward(f(11, 8), inv)
    with pytest.raises(ValueError, match="dweight"):
        moe.moe_route_topk_backward(f(6, 16), inv, f(6, 2))
    with pytest.raises(ValueError, match="contiguous"):
        moe.moe_dispatch_topk_backward(f(8, 12).t(), inv)
    with pytest.raises(ValueError, match="device"):
        moe.moe_dispatch_topk_backward(f(12, 8), inv.cpu())
    with pytest.raises(moe.MoeError, match="multiple of 16"):
        moe.moe_dispatch_topk_backward(f(12, 7), inv)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_outside_the_permuted_ones_are_named_by_no_one(dtype):
    """An entry of inv behind the last row is a choice without a row."""
    import paper_2605_11537_amd as moe
    T, k, d = 50, 2, 64
    g = torch.Generator().manual_seed(4)
    inv, _ = _tables(T, k, 0.2, 4)
    wild = inv.copy()
    out_of = np.flatnonzero(inv.reshape(-1) < 0)
    wild.reshape(-1)[out_of] = np.array([k * T, k * T + 1, 2 ** 31 - 1, -2 ** 31])[np.arange(len(out_of)) % 4]
    dt = DT[dtype]
    dout, y = (torch.randn(n, d, generator=g).to(dt).cuda() for n in (T, k * T))
    w = torch.rand(k, T, generator=g).cuda()
    a, b = (torch.from_numpy(i).int().cuda() for i in (inv, wild))
    x, z = (moe.moe_combine_topk_backward(dout, y, i, w) for i in (a, b))
    assert all(torch.equal(x[key], z[key]) for key in x)
    assert torch.equal(moe.moe_dispatch_topk_backward(y, a, dout), moe.moe_dispatch_topk_backward(y, b, dout))
