"""sru_scan at infinities, at values near the types' largest, and where a nearly shut gate meets a large value, in both types: f c + (1 - f) z and
r tanh c + (1 - r) w with each gate's own accuracy.

Tolerances: an infinity is one, of its sign.  Finite values: the bound of oracle/training.py without its terms for blends (32 half-units of
binary32 of |f c| + |(1 - f) z|; 64 for bfloat16, whose exponents are rounded once), and a bfloat16 result's own rounding."""
import numpy as np
import pytest
import torch

from oracle import training as ot
from test_gpu_sru_scan import DT, _f64, _inputs, _near

pytestmark = pytest.mark.gpu

INF = float("inf")


def _formula(c):
    """Token by token in float64, infinities as IEEE products and sums have them."""
    u, x = _f64(c["u"]), _f64(c["x"])
    B, L, W = u.shape
    H = c["c0"].shape[1]
    blocks = u.reshape(B, L, -1, H)
    s = lambda v: 1.0 / (1.0 + np.exp(-v))
    f, fr = s(blocks[:, :, 1] + _f64(c["b_f"])), s(-blocks[:, :, 1] - _f64(c["b_f"]))
    r, rr = s(blocks[:, :, 2] + _f64(c["b_r"])), s(-blocks[:, :, 2] - _f64(c["b_r"]))
    w = blocks[:, :, 3] if x is None else x
    state, h = _f64(c["c0"]), []
    with np.errstate(invalid="ignore"):
        for t in range(L):
            state = f[:, t] * state + fr[:, t] * blocks[:, t, 0]
            h.append(r[:, t] * np.tanh(state) + rr[:, t] * w[:, t])
    return np.stack(h, 1), state


def _same(got, want, dtype, what):
    got = _f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN at {np.argwhere(np.isnan(got) != np.isnan(want))[:4].tolist()}"
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), what
    on = np.isfinite(want)
    # values of order 1 after at most some ten steps that matter: 64 half-units each, and the type's rounding
    assert (np.abs(got - want)[on] <= (2.0 ** -8 * 1.01 + 2.5e-5 if dtype == "bf16" else 0) * np.abs(want[on]) + 4096 * 2.0 ** -24).all(), what


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L,k", [(1, 3), (40, 4), (700, 3), (5000, 4)])
def test_an_infinity_stays_where_it_is(dtype, L, k):
    """In u0, in the highway, in the state before: what follows in that channel has it, and nothing else does, however small the product of the gates
    behind it."""
    import paper_2605_11537_amd as moe
    print(f"{dtype} L={L} k={k}", flush=True)
    c = _inputs(dtype, 2, L, 16, k, 50 + L)
    blocks, at = c["u"].view(2, L, k, 16), L // 3
    w = c["x"] if k == 3 else blocks[:, :, 3]
    blocks[0, at, 0, 1] = INF
    blocks[0, at, 0, 2] = -INF
    w[0, at, 4] = INF
    w[1, at, 5] = -INF
    c["c0"][1, 6] = INF
    c["c0"][1, 7] = -INF
    blocks[1, L - 1, 0, 7] = INF                                     # inf - inf
    want_h, want_c = _formula(c)
    h, c_last, _ = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"])
    _same(c_last, want_c, "f32", "c_last")
    _same(h, want_h, dtype, "h")
    assert np.isinf(want_c[0, 1]) and np.isnan(want_c[1, 7]) and np.isinf(want_h[0, at, 4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_an_infinite_gradient_stays(dtype):
    """Behind the last token: every dc before it is infinite, and no other channel's."""
    import paper_2605_11537_amd as moe
    c = _inputs(dtype, 1, 900, 16, 3, 70)
    c["dc_last"][0, 3] = INF
    states = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"], want_states=True)[2]
    g = moe.sru_scan_backward(c["dh"], c["u"], states, c["x"], c["b_f"], c["b_r"], c["dc_last"])
    du0 = g["du"].view(1, 900, 3, 16)[:, :, 0]
    assert (g["dc0"][0, 3] == INF) and (du0[0, :, 3] == INF).all()
    others = [i for i in range(16) if i != 3]
    assert torch.isfinite(g["dc0"][:, others]).all() and torch.isfinite(g["du"].view(1, 900, 3, 16)[..., others]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_near_the_largest(dtype):
    """Differences of these overflow; the weighted sums do not."""
    import paper_2605_11537_amd as moe
    c = _inputs(dtype, 2, 30, 16, 3, 60)
    big = 3e38
    blocks = c["u"].view(2, 30, 3, 16)
    blocks[:, ::2, 0, :4] = big
    blocks[:, 1::2, 0, :4] = -big
    c["c0"][:, :8] = -big
    c["x"][:, :, 8:12] = -big
    args = [_f64(c[key]) for key in ("u", "x", "b_f", "b_r", "c0")]
    want = ot.sru_scan(*args, [30, 30], 64 if dtype == "bf16" else 32)
    h, c_last, _ = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"])
    _near(c_last, want["c_last"], want["c_err"][:, -1], "f32", "c_last")
    _near(h, want["h"], want["h_err"] + 2.5e-5 * np.minimum(np.abs(want["h"]), 1.0), dtype, "h")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [6.0, 10.0, 16.0, -6.0, -16.0])
def test_a_nearly_shut_gate_lets_its_share_through(dtype, gate):
    """The states are binary32 in both types: a share of e^-16 of a large value keeps its own accuracy."""
    import paper_2605_11537_amd as moe
    c = _inputs(dtype, 3, 4, 64, 3, 61)
    blocks = c["u"].view(3, 4, 3, 64)
    blocks[:, :, 1] = gate
    c["b_f"][:] = 0
    if gate > 0:
        blocks[:, :, 0] *= 4096
        c["c0"] *= 1e-3
    else:
        c["c0"] *= 4096
        blocks[:, :, 0] *= 1e-3
    args = [_f64(c[key]) for key in ("u", "x", "b_f", "b_r", "c0")]
    want = ot.sru_scan(*args, [4] * 3, 64 if dtype == "bf16" else 32)
    _, c_last, states = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"], want_states=True)
    _near(c_last, want["c_last"], want["c_err"][:, -1], "f32", "c_last")
    one = moe.sru_scan(c["u"][:, :1].contiguous(), c["x"][:, :1].contiguous(), c["b_f"], c["b_r"], c["c0"])[1]
    _near(one, want["c"][:, 1], want["c_err"][:, 1], "f32", "one token")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block", [0, 1, 2])
def test_a_nan_goes_from_tile_to_tile(dtype, block):
    """In the state's own blocks it reaches every later token of its channel and every earlier one's gradient; in the reset gate's its token alone."""
    import paper_2605_11537_amd as moe
    L, at = 9000, 4321
    c = _inputs(dtype, 1, L, 8, 3, 80)
    c["u"].view(1, L, 3, 8)[0, at, block, 3] = float("nan")
    h, c_last, states = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"], want_states=True)
    bad = torch.isnan(h[0])
    others = [0, 1, 2, 4, 5, 6, 7]
    assert not bad[:, others].any() and not bad[:at].any() and bad[at, 3]
    assert bool(bad[at + 1:, 3].all()) == (block < 2) and bool(bad[at + 1:, 3].any()) == (block < 2)
    assert bool(torch.isnan(c_last[0, 3])) == (block < 2) and torch.isfinite(c_last[0, others]).all()
    g = moe.sru_scan_backward(c["dh"], c["u"], states, c["x"], c["b_f"], c["b_r"], c["dc_last"])
    du = torch.isnan(g["du"].view(L, 3, 8))
    assert not du[..., others].any() and torch.isfinite(g["dc0"][0, others]).all()
    assert du[:at + 1, 0, 3].all() and torch.isnan(g["dc0"][0, 3])
    assert not torch.isnan(g["db_f"][others]).any() and torch.isnan(g["db_f"][3])
