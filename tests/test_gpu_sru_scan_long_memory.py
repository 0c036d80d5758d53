"""sru_scan and its gradient in channels that forget slowly: forget biases of 7 to 10, whose memories are a thousand to twenty thousand tokens.

Tolerance, with e = 2^-24 and rho = 1 - f.  A share rho has its own relative accuracy, K e (an exponential whose argument of up to 11 was rounded, a
reciprocal, a product: K = 32; 64 in bfloat16, where the argument is rounded three times), and f = 1 - rho the same absolute error: per step
K e rho (|z| + |c|), forgotten with f.  The state is carried from one run of at least 64 steps to the next by c + (C - R c) with R = 1 - product of f
known to a relative accuracy: 2 e |c| a run.  Inside a run every one of 16 steps, and 40 joins of runs, wavefronts and tiles, may round by e of what they
hold, which the next run does not inherit: 128 e (|c| + the largest |z|) beside it.
The gradient is the same recurrence from the other end, over e_t = dh r (1 - tanh^2 c), which is off by K e of itself and by the state's error.

Where each call takes one token, the state is rounded at every step.  With noise in z of 10^3 units in the last place and more these roundings are
as good as independent and uniform: six of their standard deviations, e / sqrt(3) sqrt(1 / (2 rho)) |c|."""
import numpy as np
import pytest
import torch

from test_gpu_sru_scan import DT, _f64

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def _inputs(dtype, B, L, H, seed, hi=10.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    u = n(B, L, 3, H)
    u[:, :, 1] *= 0.1
    third = H // 3
    u[:, :, 0, :third] = 1.0                                         # a constant, a mean with noise, noise alone
    u[:, :, 0, third:2 * third] = 1.0 + 0.1 * u[:, :, 0, third:2 * third]
    dh = n(B, L, H) * 0.1 + 1.0
    dh[:, :, ::2] -= 1.0
    b_f = 7.0 + (hi - 7.0) * torch.rand(H, generator=g, device="cuda")
    return dict(u=u.view(B, L, 3 * H).to(DT[dtype]), x=n(B, L, H).to(DT[dtype]), b_f=b_f, b_r=n(H), c0=0.1 * n(B, H), dh=dh.to(DT[dtype]),
                dc_last=0.1 * n(B, H))


def _lines(c, pick):
    """The chosen (sequence, channel) lines: u0, forget and reset pre-activations, highway [L, n]; dh; per line: c0, dc_last."""
    b, ch = (torch.tensor(v, device="cuda") for v in zip(*pick))
    B, L, H = c["x"].shape
    u = c["u"].view(B, L, 3, H)
    take = lambda t: _f64(t[b, :, ch]).T.copy()
    return dict(z=take(u[:, :, 0]), a=take(u[:, :, 1]) + _f64(c["b_f"][ch]), r=take(u[:, :, 2]) + _f64(c["b_r"][ch]), w=take(c["x"]), d=take(c["dh"]),
                c0=_f64(c["c0"][b, ch]), dc=_f64(c["dc_last"][b, ch]), b=b, ch=ch)


def _forward(s, K):
    """States [L+1, n] and the bound of their error."""
    L, n = s["z"].shape
    f, rho = 1.0 / (1.0 + np.exp(-s["a"])), 1.0 / (1.0 + np.exp(s["a"]))
    c, err = np.empty((L + 1, n)), np.zeros((L + 1, n))
    c[0] = s["c0"]
    for t in range(L):
        c[t + 1] = f[t] * c[t] + rho[t] * s["z"][t]
        err[t + 1] = f[t] * err[t] + K * E * rho[t] * (np.abs(s["z"][t]) + np.abs(c[t])) + 2 / 64 * E * np.abs(c[t])
    return f, rho, c, err + 128 * E * (np.abs(c) + np.abs(s["z"]).max(0))


def _holds(got, want, tol, dtype, what):
    got = _f64(got)
    tol = tol + (2.0 ** -8 if dtype == "bf16" else E) * 1.001 * np.abs(want) + 1e-30
    over = np.abs(got - want) / tol
    assert np.isfinite(got).all() and over.max() <= 1.0, f"{what}: {over.max():.2f} of the bound at {np.unravel_index(over.argmax(), over.shape)}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,H", [(1, 20001, 96), (128, 12003, 128), (1, 70001, 66), (3, 1000, 64), (300, 60, 60)])
def test_slow_channels(dtype, B, L, H):
    """In tiles, walked, over several stretches of tiles, and short."""
    import paper_2605_11537_amd as moe
    print(f"{dtype} B={B} L={L} H={H}", flush=True)
    K = 64 if dtype == "bf16" else 32
    c = _inputs(dtype, B, L, H, L)
    pick = [(i % B if i % 2 else B - 1 - i % B, i * (H // 48) + i % max(1, H // 48)) for i in range(48)]
    s = _lines(c, pick)
    f, rho, want, tol = _forward(s, K)
    h, c_last, states = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"], want_states=True)
    g = moe.sru_scan_backward(c["dh"], c["u"], states, c["x"], c["b_f"], c["b_r"], c["dc_last"])
    b, ch = s["b"], s["ch"]
    _holds(c_last[b, ch], want[-1], tol[-1], "f32", "c_last")
    saved = states.view(B, -1, H)[b, :, ch].T
    _holds(saved, want[:-1:8], tol[:-1:8], "f32", "states")
    r, off = 1.0 / (1.0 + np.exp(-s["r"])), 1.0 / (1.0 + np.exp(s["r"]))
    tanh = np.tanh(want[1:])
    tanh_off = 2.5e-5 if dtype == "bf16" else 0.0
    size = np.abs(r * tanh) + np.abs(off * s["w"])
    _holds(h[b, :, ch].T, r * tanh + off * s["w"], r * tol[1:] + K * E * size + tanh_off * np.abs(r * tanh), dtype, "h")

    slope = 1.0 - tanh * tanh
    e, e_err = s["d"] * r * slope, np.abs(s["d"]) * r * (0.77 * tol[1:] + K * E * slope)
    dc, dc_err = s["dc"].copy(), np.zeros_like(s["dc"])
    du0, du0_tol, du1, du1_tol = (np.empty_like(e) for _ in range(4))
    for t in reversed(range(L)):
        full = dc + e[t]
        near = dc_err + e_err[t] + 128 * E * np.abs(full)            # with the joins' own
        gap = want[t] - s["z"][t]
        du0[t], du0_tol[t] = full * rho[t], rho[t] * (near + K * E * np.abs(full))
        q = f[t] * rho[t]
        du1[t] = full * gap * q
        du1_tol[t] = q * (near * (np.abs(gap) + tol[t]) + np.abs(full) * (tol[t] + 4 * E * (np.abs(want[t]) + np.abs(s["z"][t])) + K * E * np.abs(gap)))
        dc_err = f[t] * (dc_err + e_err[t]) + K * E * rho[t] * np.abs(full) + 2 / 64 * E * np.abs(full)
        dc = full * f[t]
    _holds(g["dc0"][b, ch], dc, dc_err + 128 * E * np.abs(dc), "f32", "dc0")
    du = g["du"].view(B, L, 3, H)[b, :, :, ch]
    _holds(du[:, :, 0].T, du0, du0_tol, dtype, "du0")
    _holds(du[:, :, 1].T, du1, du1_tol, dtype, "du1")
    if B == 1:                                                       # the sums over the tokens of one sequence
        _holds(g["db_f"][ch], du1.sum(0), du1_tol.sum(0) + E * (L + 64) * np.abs(du1).sum(0), "f32", "db_f")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_slow_channels_token_by_token(dtype):
    import paper_2605_11537_amd as moe
    B, L, H = 2, 5000, 96
    K = 64 if dtype == "bf16" else 32
    c = _inputs(dtype, B, L, H, 7, hi=8.0)
    third = H // 3
    s = _lines(c, [(i % 2, third + i) for i in range(2 * third)])    # noise with a mean and alone
    f, rho, want, _ = _forward(s, K)
    err = np.zeros(2 * third)
    for t in range(L):
        err = f[t] * err + K * E * rho[t] * (np.abs(s["z"][t]) + np.abs(want[t]))
    size = np.abs(want).max(0)
    tol = err + 4 * E * size + 6 * E / np.sqrt(3) * np.sqrt(1 / (2 * rho.min(0))) * size
    state = c["c0"].clone()
    u, x, h = c["u"].transpose(0, 1).contiguous(), c["x"].transpose(0, 1).contiguous(), torch.empty(B, 1, H, dtype=DT[dtype], device="cuda")
    for t in range(L):
        moe.sru_scan(u[t].view(B, 1, 3 * H), x[t].view(B, 1, H), c["b_f"], c["b_r"], state, out=(h, state, None))
    _holds(state[s["b"], s["ch"]], want[-1], tol, "f32", "c_last")
