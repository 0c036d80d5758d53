"""Gates of moe_gated_ffn over their whole range.  The products are with ones and zeros, so that g, u and dh are the inputs' own values and y, dx hold
act(g) u and its derivatives, rounded once or twice to the tensors' type (half a step each).  The activation by itself: exponentials with (|x| + 8) steps of 2^-23
for an argument x; a sigmoid or a tail below the smallest normal number may be zero."""
import math

import numpy as np
import pytest
import torch

from oracle.learning import STEP
from test_gpu_gated_ffn import ACT, DT, HALF, f64

pytestmark = pytest.mark.gpu

TINY = 2.0 ** -126
GATES = [0.0, 1e-30, -1e-30, 1e-3, -1e-3, 0.5, -0.5, 1.0, -1.0, 2.5, -2.5, 3.0, -3.0, -4.0, 5.0, -5.0, -6.0, -7.0, 8.0, -8.0, -9.0, -10.0, -11.0, -12.0, 13.0, -16.0,
         -20.0, 40.0, -40.0, -60.0, -79.0, -80.0, -81.0, 85.0, -86.0, -90.0, 100.0, -100.0, -200.0, 1e4, -1e4, 1e10, -1e10, 1e19, -1e19, -1e25, 1e30, -1e30, 1e36, -1e36, -1e38]


def reference(act, g):
    """act and slope in float64 with what they may be off by."""
    if act == "silu":
        e = np.exp(-abs(g))
        s, rest = np.where(g >= 0, 1.0, e) / (1.0 + e), np.where(g >= 0, e, 1.0) / (1.0 + e)
        a, slope = g * s, s * (1.0 + g * rest)
        rel = (abs(g) + 8) * STEP
        off_a, off_slope = rel * abs(a), 2 * rel * s * (1.0 + abs(g) * rest)
    elif act == "gelu":
        with np.errstate(over="ignore", under="ignore"):
            phi = 0.5 * np.array([math.erfc(-v * math.sqrt(0.5)) for v in g])
            bell = np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
        a, slope = g * phi, phi + g * bell
        # an argument g / sqrt 2 off by a step moves erfc by g^2 steps of itself; 1e-6: what a rational form of the tail leaves of it
        rel = (np.minimum(g * g, 1e4) + 16) * STEP + 1e-6
        off_a, off_slope = rel * abs(a), rel * (phi + abs(g) * bell)
    else:
        a, slope = np.maximum(g, 0.0), (g > 0) * 1.0
        off_a = off_slope = 0.0 * g
    return a, off_a, slope, off_slope


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("copies", [1, 30])                          # few rows and many: other tiles
def test_gates_near_and_far(copies, dtype, act):
    import paper_2605_11537_amd as moe
    t, half = DT[dtype], HALF[dtype]
    values = torch.tensor(GATES, device="cuda").to(t)
    R, F, d = len(GATES) * copies, 8, 16
    x, dy = torch.zeros(R, d, dtype=t, device="cuda"), torch.zeros(R, d, dtype=t, device="cuda")
    x[:, 0], x[:, 8], dy[:, 0] = values.repeat(copies), 1.5, 0.75
    w_gate, w_up, w_down = (torch.zeros(1, *s, dtype=t, device="cuda") for s in ((d, F), (d, F), (F, d)))
    w_gate[0, 0, 0] = w_up[0, 8, 0] = w_down[0, 0, 0] = 1.0
    y, states = moe.moe_gated_ffn(x, w_gate, w_up, w_down, activation=ACT[act], want_states=True)
    grads = moe.moe_gated_ffn_backward(dy, x, w_gate, w_up, w_down, states, activation=ACT[act])
    a, off_a, slope, off_slope = reference(act, f64(x[:, 0]))
    for what, got, want, off in (("y", y[:, 0], 1.5 * a, 1.5 * off_a), ("dg", grads["dx"][:, 0], 1.125 * slope, 1.125 * off_slope),
                                 ("du", grads["dx"][:, 8], 0.75 * a, 0.75 * off_a)):
        # the product beside it, one rounding to the type
        room = off + (half + 3 * STEP) * (abs(want) + off) + 2 * TINY * (1 + np.minimum(abs(f64(x[:, 0])), 200.0))
        ok = abs(f64(got) - want) <= room
        assert ok.all(), (what, [(f64(x[i, 0]).item(), f64(got[i]).item(), want[i]) for i in np.nonzero(~ok)[0][:6]])


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_closed_gate_beside_large_values(dtype, act):
    """dh u passes the range; behind a gate that is shut the gradient is 0 all the same."""
    import paper_2605_11537_amd as moe
    t = DT[dtype]
    x, dy = torch.zeros(3, 16, dtype=t, device="cuda"), torch.zeros(3, 16, dtype=t, device="cuda")
    x[:, 0], x[:, 8], dy[:, 0] = torch.tensor([-1e25, -1e3, 2.0], device="cuda").to(t), 1e30, 1e10
    w_gate, w_up, w_down = (torch.zeros(1, *s, dtype=t, device="cuda") for s in ((16, 8), (16, 8), (8, 16)))
    w_gate[0, 0, 0] = w_up[0, 8, 0] = w_down[0, 0, 0] = 1.0
    _, states = moe.moe_gated_ffn(x, w_gate, w_up, w_down, activation=ACT[act], want_states=True)
    dx = moe.moe_gated_ffn_backward(dy, x, w_gate, w_up, w_down, states, activation=ACT[act])["dx"]
    assert not dx[:2, 0].any() and not dx[:2, 8].any()
    assert torch.isinf(dx[2, 0])                                     # and infinite where the gate is open
