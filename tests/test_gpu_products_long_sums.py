"""Weights' gradients of bfloat16 over very many rows, all of one sign: an accumulator in binary32 holds them.  A matrix instruction adds the products of 32 rows, and each of
the R / 32 additions is off by half a step, 2^-24 of what the sum is by then, at most: R 2^-29 of the result where all err to one side, as for equal rows, and
its root over what differs from row to row (2^-12 here).  Rounding is monotonic: what is behind it lies between the bfloat16 values of the result made smaller and larger by
that.  (The errors of bfloat16's rounding have no mean of 0 over the columns here: a column's sum is 1.008 steps of bfloat16 from its neighbour's, R 1.0078 / 128 beside R 2^-7, so
that they wander slowly.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def rows(g, R, columns, equal):
    """Eight significant bits; a column's own range, so that the columns' sums differ."""
    if equal:
        return (1 + torch.arange(columns, device="cuda") % 128 / 128.0).to(BF).expand(R, columns).contiguous()
    spread = 1 + 2 * torch.arange(columns, device="cuda")
    out = torch.empty(R, columns, dtype=BF, device="cuda")
    for part in out.split(1 << 18):
        part.copy_(1 + (torch.rand(part.shape, generator=g, device="cuda") * spread).floor() / 128)
    return out


def check(got, want, R, equal):
    drift = R * 2.0 ** -29 if equal else 2.0 ** -12
    one, other = (want * (1 - drift)).to(BF).double(), (want * (1 + drift)).to(BF).double()
    ok = (got.double() >= torch.minimum(one, other)) & (got.double() <= torch.maximum(one, other))
    assert ok.all(), (int((~ok).sum()), float(((got.double() - want) / want).abs().max()))


@pytest.mark.parametrize("equal", [False, True])
@pytest.mark.parametrize("N,V", [(1 << 17, 600), (1 << 20, 600), ((1 << 22) + 5, 200)])
def test_head(N, V, equal):
    import paper_2605_11537_amd as moe
    d = 64
    g = torch.Generator(device="cuda").manual_seed(N)
    h = rows(g, N, d, equal)
    # dz: -0.50390625 in every row but the first
    dlogprob = torch.full((N,), 1.0078125, device="cuda")
    dlogprob[0] = 2.0
    got = moe.moe_head_logprobs_backward(h, torch.zeros(V, d, dtype=BF, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda"), torch.zeros(N, device="cuda"),
                                         dlogprob)
    want = -1.0078125 * sum(p.double().sum(0) for p in h.split(1 << 18)) - (2.0 - 1.0078125) * h[0].double()
    check(got["dw_head"][1:, 1:], want[1:].expand(V - 1, d - 1), N, equal)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("equal", [False, True])
@pytest.mark.parametrize("R,F", [(1 << 18, 2048), (1 << 20, 256)])
def test_gated(R, F, equal):
    import paper_2605_11537_amd as moe
    d = 64
    g = torch.Generator(device="cuda").manual_seed(R)
    x = torch.zeros(R, d, dtype=BF, device="cuda")
    x[:, :2] = 1.0
    w_gate, w_up, w_down = (torch.zeros(1, *s, dtype=BF, device="cuda") for s in ((d, F), (d, F), (F, d)))
    w_gate[0, 0], w_up[0, 1] = 1.0, (1 + torch.arange(F, device="cuda") % 128 / 128.0).to(BF)       # h = w_up's row
    dy = rows(g, R, d, equal)
    y, states = moe.moe_gated_ffn(x, w_gate, w_up, w_down, activation=moe.ACT_RELU, want_states=True)
    got = moe.moe_gated_ffn_backward(dy, x, w_gate, w_up, w_down, states, activation=moe.ACT_RELU)["dw_down"][0]
    want = w_up[0, 1].double()[:, None] * sum(p.double().sum(0) for p in dy.split(1 << 18))[None]
    check(got[:, 1:], want[:, 1:], R, equal)
    del x, dy, y, states
    torch.cuda.empty_cache()
