"""The training and scoring calls on tensors whose offsets pass 32 bits, in elements and in bytes, held against the references of the small tests on
the rows and channels that lie furthest apart (their tolerances)."""
import numpy as np
import pytest
import torch

from oracle import training as ot
from test_gpu_sru_scan import _near
from test_gpu_token_logprobs import _check as _check_logprobs
from test_gpu_token_logprobs import _inputs as _logits

pytestmark = pytest.mark.gpu


def _f64(t):
    return t.double().cpu().numpy()


def _rows(g, *shape, dt=torch.bfloat16):
    return torch.empty(shape, dtype=dt, device="cuda").normal_(generator=g)


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def _pick(t, blocks, sel):
    """The chosen channels of every column block."""
    B, L, W = t.shape
    return _f64(t.view(B, L, blocks, W // blocks)[..., sel].reshape(B, L, -1))


@pytest.mark.parametrize("L,H,k,dtype,B", [(1 << 20, 1400, 3, "bf16", 1), (17, 1 << 22, 4, "f32", 1), (260, 1 << 20, 4, "f32", 5)])
def test_scan(L, H, k, dtype, B):
    """A long sequence, the most channels, and sequences that begin past 2^32 elements."""
    import paper_2605_11537_amd as moe
    print(f"{dtype} B={B} L={L} H={H} k={k}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(L)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    u, x, dh = _rows(g, B, L, k * H, dt=dt), _rows(g, B, L, H, dt=dt) if k == 3 else None, _rows(g, B, L, H, dt=dt)
    b_f, b_r, c0, dc = [_rows(g, *s, dt=torch.float32) for s in ((H,), (H,), (B, H), (B, H))]
    h, c_last, states = moe.sru_scan(u, x, b_f, b_r, c0, want_states=True)
    grads = moe.sru_scan_backward(dh, u, states, x, b_f, b_r, dc)
    states = states.view(B, (L + 7) // 8, H)
    assert torch.equal(states[:, 0], c0)
    sel = torch.tensor([0, 1, 63, 64, H // 2, H - 65, H - 2, H - 1], device="cuda")
    # windows: the reference begins 512 steps ahead, from a saved state, whose own error is forgotten before the first row that is compared
    for t0 in ((0, L // 2, L - 300) if L > 1000 else (0,)):
        t1, pre = min(t0 + 300, L), max(0, t0 - 512) // 8 * 8
        part, on = slice(pre, t1), slice(t0 - pre, None)
        args = [_pick(u[:, part], k, sel), None if x is None else _pick(x[:, part], 1, sel), _f64(b_f[sel]), _f64(b_r[sel]),
                _f64(states[:, pre // 8, sel]), np.full(B, t1 - pre), 64 if dtype == "bf16" else 32, dtype == "bf16"]
        want = ot.sru_scan(*args)
        _near(h[:, t0:t1][..., sel], want["h"][:, on], want["h_err"][:, on], dtype, f"h from {t0}")
        for t in range((t0 + 7) // 8 * 8, t1, 8):
            _near(states[:, t // 8, sel], want["c"][:, t - pre], want["c_err"][:, t - pre], "f32", f"state {t}")
        if t1 < L:
            continue
        _near(c_last[:, sel], want["c_last"], want["c_err"][:, -1], "f32", "c_last")
        want, bound = ot.sru_scan_backward(_pick(dh[:, part], 1, sel), _f64(dc[:, sel]), *args)
        du = grads["du"][:, t0:].view(B, L - t0, k, H)[..., sel].reshape(B, L - t0, -1)
        _near(du, want["du"][:, on], bound["du"][:, on], dtype, "du")
        if k == 3:
            _near(grads["dx"][:, t0:][..., sel], want["dx"][:, on], bound["dx"][:, on], dtype, "dx")
        if t0 == 0:
            for key in ("db_f", "db_r"):
                _near(grads[key][sel], want[key], bound[key], "f32", key)
            _near(grads["dc0"][:, sel], want["dc0"], bound["dc0"], "f32", "dc0")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [60, 1000, 50257, 131073])
def test_logits_rows_far_apart(dtype, V):
    import paper_2605_11537_amd as moe
    print(f"{dtype} V={V}", flush=True)
    x, t, dl, de = _logits(dtype, 3, V, V)
    far = torch.empty(2 * ((1 << 31) + 8) + V, dtype=x.dtype, device="cuda").as_strided((3, V), ((1 << 31) + 8, 1))
    far.copy_(x)
    got = _check_logprobs(far, t, 4, f"{dtype} {V}", dl, de, dtype)
    want = moe.moe_token_logprobs_backward(x, t, got["lse"], got["entropy"], dl, de)
    assert moe.moe_token_logprobs_backward(far, t, got["lse"], got["entropy"], dl, de, out=far) is far
    assert torch.equal(far, want)


def test_rows_to_experts_and_back():
    import paper_2605_11537_amd as moe
    T, d = (1 << 21) + 3, 2056
    print(f"T={T} d={d}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    dout, y = _rows(g, T, d), _rows(g, T, d)
    inv = torch.arange(T - 1, -1, -1, dtype=torch.int32, device="cuda")
    w = _rows(g, T, dt=torch.float32)
    got = moe.moe_combine_topk_backward(dout, y, inv, w, 1)
    for s in (0, 1, T // 2, T - 3, T - 2, T - 1):
        assert torch.equal(got["dy_perm"][T - 1 - s], (w[s] * dout[s].float()).bfloat16()) and torch.equal(got["dx"][s], dout[s]), s
        a, b = _f64(dout[s]), _f64(y[T - 1 - s])
        assert abs(float(got["dweight"][s]) - a @ b) <= d * 2.0 ** -24 * (np.abs(a) @ np.abs(b)), s
    half = T // 2
    two = inv[: 2 * half].view(2, half)
    dx = moe.moe_dispatch_topk_backward(y[: 2 * half], two - (T - 2 * half))
    for s in (0, 1, half - 2, half - 1):
        assert torch.equal(dx[s], (y[2 * half - 1 - s].float() + y[half - 1 - s].float()).bfloat16()), s


def test_gate():
    import paper_2605_11537_amd as moe
    T, E = (1 << 24) + 5, 260
    print(f"T={T} E={E}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(4)
    logits = _rows(g, T, E, dt=torch.float32)
    idx = (torch.arange(T, device="cuda") % E).int()
    dw = _rows(g, T, dt=torch.float32)
    got = moe.moe_route_topk_backward(logits, idx, dw)
    for part in (slice(0, 40), slice(T // 2, T // 2 + 40), slice(T - 40, T)):
        small = moe.moe_route_topk_backward(logits[part].clone(), idx[part].clone(), dw[part].clone())
        assert torch.equal(got[part], small) and (small != 0).any(1).all()
