"""moe_token_logprobs and moe_token_logprobs_backward against oracle/training.py in float64.

Tolerances, with e = 2^-24.  d = x - max is rounded once (e |d|, as far as logits lie apart), the exponential and its argument are off by 4
more; the sums are trees over at most 2^18 terms behind runs of at most 2^10 (1100 e at most, an eighth of that for the row lengths
here): logprob and lse 200 e of 1 + the magnitudes added, the entropy that of its terms' magnitudes, log s + sum p |d|.  In the gradient p has the
relative error of its exponent, e (|x| + |lse|), and 8 e; a bfloat16 result rounds by 2^-8 of itself."""
import numpy as np
import pytest
import torch

from oracle import training as ot

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
E = 2.0 ** -24


def _f64(t):
    return t.double().cpu().numpy()


def _check(x, target, k, what, dl=None, de=None, dtype="f32"):
    """x: a device matrix, contiguous or not."""
    import paper_2605_11537_amd as moe
    xs, N, V = _f64(x), *x.shape
    t = target.cpu().numpy()
    want = ot.token_logprobs(xs, t, k)
    got = moe.moe_token_logprobs(x, target, k)
    assert np.array_equal(got["top_idx"].cpu().numpy(), want["top_idx"]), what
    top = np.max(xs, 1)
    for n in range(N):
        for key in ("logprob", "lse", "entropy"):
            g, w = float(got[key][n]), want[key][n]
            if not np.isfinite(w):
                assert g == w, (what, key, n)
                continue
            spread = 1.0 + abs(w) + np.log(V) + (abs(top[n]) if key == "lse" else 0.0)
            if key == "logprob" and 0 <= t[n] < V:
                spread += abs(xs[n, t[n]] - top[n])
            if key == "entropy":
                p = np.exp(xs[n] - want["lse"][n])
                on = p > 0
                spread += (p[on] * np.abs(xs[n][on] - top[n])).sum()
            assert abs(g - w) <= 200 * E * spread, (what, key, n, g, w)
    a, b = _f64(got["top_logprob"]), want["top_logprob"]
    fin = np.isfinite(b)
    assert np.array_equal(a[~fin], b[~fin])
    assert (np.abs(a - b)[fin] <= 200 * E * (1 + np.log(V) + 2 * np.abs(b[fin]))).all(), what
    if dl is None:
        return got
    d = moe.moe_token_logprobs_backward(x, target, got["lse"], got["entropy"], dl, de)
    dd = np.zeros(N) if de is None else _f64(de)
    ref = ot.token_logprobs_backward(xs, t, _f64(dl), dd)
    with np.errstate(invalid="ignore"):
        for n in range(N):
            if want["lse"][n] == -np.inf:
                assert (d[n] == 0).all(), what
                continue
            lp = xs[n] - want["lse"][n]
            p = np.exp(lp)
            on = p > 0
            gl = abs(_f64(dl)[n]) if 0 <= t[n] < V else 0.0
            size = np.zeros(V)
            step = 8 + np.abs(xs[n][on]) + abs(want["lse"][n]) + 200 * abs(want["entropy"][n])
            size[on] = p[on] * (gl + abs(dd[n]) * (np.abs(lp[on]) + want["entropy"][n] + 1)) * (1 + step)
            if gl:
                size[t[n]] += gl * (8 + abs(want["lse"][n]))
            tol = HALF[dtype] * 1.001 * np.abs(ref[n]) + 4 * E * size + 1e-36
            diff = np.abs(_f64(d[n]) - ref[n])
            assert (diff <= tol).all(), (what, n, int((diff / tol).argmax()), (diff / tol).max())
    return got


def _inputs(dtype, N, V, seed, std=2.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(N, V, generator=g) * std).to(DT[dtype]).cuda()
    t = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    t[N // 2] = -1
    if N > 3:
        t[1], t[3] = V, 1 << 30
    return x, t.cuda(), torch.randn(N, generator=g).cuda(), torch.randn(N, generator=g).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(1, 1), (5, 2), (3, 7), (70, 8), (2, 63), (9, 64), (6, 65), (300, 128), (5, 255), (7, 1000), (4, 1024), (3, 1025),
                                 (2, 2049), (6, 4099), (1, 8192), (3, 20001), (2, 50257), (1, 131072), (1, 200003), (600, 3000)])
def test_sizes(dtype, N, V):
    print(f"{dtype} N={N} V={V}", flush=True)
    x, t, dl, de = _inputs(dtype, N, V, N + V)
    _check(x, t, min(8, V), f"{dtype} {N}x{V}", dl, de, dtype)
    for k in (0, 1, 3):
        if k <= V and N <= 9:
            _check(x, t, k, f"{dtype} {N}x{V} k={k}", dl, None, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 130, 3001, 40000])
def test_masks(dtype, V):
    """Rows with nothing left, with one logit left, with less than k left; masks of -inf and of the type's lowest value, the target among
    them."""
    x, t, dl, de = _inputs(dtype, 8, V, V)
    low = torch.finfo(DT[dtype]).min
    t[:] = torch.tensor([0, V - 1, 1, 2, 3, 0, -1, 4], dtype=torch.int32)
    x[0] = -np.inf                                                   # nothing left
    x[1, :-1] = -np.inf                                              # one left, the target
    x[2] = -np.inf
    x[2, 0], x[2, 3] = 1.0, 0.5                                      # two left, the target masked
    x[3] = low                                                       # all at the lowest value: as good as equal
    x[4, ::2] = low
    x[5, 1:] = low
    x[6] = -np.inf                                                   # nothing left, padded
    x[7, : V // 2] = -np.inf
    _check(x, t, min(5, V), f"{dtype} masks {V}", dl, de, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 5000, 60000])
def test_ties_and_orders(dtype, V):
    """Equal logits (lowest id first), rows that rise or fall throughout (every next logit is a new best, or none is), one peak."""
    x, t, dl, de = _inputs(dtype, 7, V, V)
    x[0] = 0.25
    x[1] = torch.arange(V) % 3
    x[2] = torch.linspace(-20, 20, V)
    x[3] = torch.linspace(20, -20, V)
    x[4] = -50.0
    x[4, V // 2] = 50.0
    x[5] = torch.randint(0, 5, (V,))
    x[6] += 3000.0 if dtype == "f32" else 8.0
    _check(x, t, 8, f"{dtype} ties {V}", dl, de, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_apart_and_on_any_address(dtype):
    """Slices of a padded vocabulary, from every element offset in a 16-byte piece; the gradient into such a slice, and in place."""
    import paper_2605_11537_amd as moe
    for V, stride in ((1000, 1024), (37, 41), (5003, 5011), (20000, 20007)):
        for at in (0, 1, 3, 7):
            whole, t, dl, de = _inputs(dtype, 5, stride + 8, V + at)
            t = torch.where(t < V, t, -1).int()
            whole[:, at + V:] = float("nan")
            whole[:, :at] = float("nan")
            x = whole[:, at:at + V]
            got = _check(x, t, 4, f"{dtype} {V} of {stride} from {at}", dl, de, dtype)
            same = moe.moe_token_logprobs(x.contiguous(), t, 4)
            assert all(torch.equal(got[key], same[key]) for key in ("top_idx",))
            want = moe.moe_token_logprobs_backward(x, t, got["lse"], got["entropy"], dl, de)
            room = torch.full_like(whole, 7.0)
            moe.moe_token_logprobs_backward(x, t, got["lse"], got["entropy"], dl, de, out=room[:, at:at + V])
            assert torch.equal(room[:, at:at + V], want) and (room[:, :at] == 7).all() and (room[:, at + V:] == 7).all()
            moe.moe_token_logprobs_backward(x, t, got["lse"], got["entropy"], dl, de, out=x)
            assert torch.equal(x, want) and torch.isnan(whole[:, :at]).all() and torch.isnan(whole[:, at + V:]).all()


def test_infinity_and_nan():
    import paper_2605_11537_amd as moe
    for V in (50, 3000, 40000):
        x, t, dl, de = _inputs("f32", 4, V, V)
        t[:] = 0
        clean = x.clone()
        x[0, V // 2] = float("nan")
        x[1, V - 1] = float("inf")
        x[3] = float("-inf")
        x[3, 1] = float("nan")
        got = moe.moe_token_logprobs(x, t, 4)
        assert all(torch.isnan(got[key][[0, 1, 3]]).all() for key in ("logprob", "entropy", "lse"))
        ids = got["top_idx"].cpu().numpy()
        assert ((ids >= 0) & (ids < V)).all() and V // 2 not in ids[0] and ids[1, 0] == V - 1 and len(set(ids[3])) == 4
        d = moe.moe_token_logprobs_backward(x, t, got["lse"], got["entropy"], dl, de)
        assert torch.isnan(d[[0, 1, 3]]).all()
        ref = moe.moe_token_logprobs(clean, t, 4)                    # the other row does not notice
        assert all(torch.equal(got[key][2], ref[key][2]) for key in got)


def test_rows_do_not_depend_on_their_neighbours():
    """A row's numbers in one batch and in another of the same kind, and two equal calls, bit for bit."""
    import paper_2605_11537_amd as moe
    for V in (128, 5000):
        x, t, dl, de = _inputs("bf16", 1100, V, V)
        a, b = moe.moe_token_logprobs(x, t, 3), moe.moe_token_logprobs(x, t, 3)
        c = moe.moe_token_logprobs(x[:1050].contiguous(), t[:1050].contiguous(), 3)
        for key in a:
            assert torch.equal(a[key], b[key]) and torch.equal(a[key][:1050], c[key]), key


def test_no_rows_and_shapes_that_do_not_fit():
    import paper_2605_11537_amd as moe
    f = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")
    got = moe.moe_token_logprobs(f(0, 9), f(0, dt=torch.int32), 2)
    assert got["top_idx"].shape == (0, 2)
    assert moe.moe_token_logprobs_backward(f(0, 9), f(0, dt=torch.int32), f(0), f(0), f(0)).shape == (0, 9)
    with pytest.raises(ValueError, match="target"):
        moe.moe_token_logprobs(f(3, 9), f(3, dt=torch.int64))
    with pytest.raises(ValueError, match="rows of logits"):
        moe.moe_token_logprobs(f(9, 3).t(), f(3, dt=torch.int32))
    with pytest.raises(ValueError, match="rows of logits"):
        moe.moe_token_logprobs(f(1, 9).expand(3, 9), f(3, dt=torch.int32))
    with pytest.raises(moe.MoeError, match="k=9"):
        moe.moe_token_logprobs(f(3, 20), f(3, dt=torch.int32), 9)
    with pytest.raises(TypeError):
        moe.moe_token_logprobs(f(3, 20, dt=torch.float16), f(3, dt=torch.int32))
    with pytest.raises(ValueError, match="dlogprob"):
        moe.moe_token_logprobs_backward(f(3, 9), f(3, dt=torch.int32), f(3), f(3), f(4))
