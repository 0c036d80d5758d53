"""moe_head_logprobs_backward where logits lie far from zero: their binary32 log sum holds a part of the sum's logarithm or none of it, and the
probabilities have to add up to one all the same.

Products and biases are multiples of 1/8 with few bits, and the biases of 1e6 and beyond have logits that binary32 holds or that all products vanish beside, so that the logits
in binary32 are known exactly and no bound of theirs enters.  An exponential: its argument is off by 2^-23 of itself, and the logarithm beside it
(at most log2 2^24) by 24 steps; 8 more for the exponential, the sum and the product.  A log sum below the limit from which rows are summed again (64; in
bfloat16 2048) is off by half a step, 2^-24 of itself."""
import numpy as np
import pytest
import torch

from oracle import learning as ol
from test_gpu_gated_ffn import DT, HALF, f64

pytestmark = pytest.mark.gpu

FAR = {"f32": 64.0, "bf16": 2048.0}
LOWEST = float(np.finfo(np.float32).min)


def make(dtype, N, d, V, base, seed, bias_on=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ints = lambda n, *s: torch.randint(-n, n + 1, s, generator=g, device="cuda").float()
    s = dict(h=ints(1, N, d), w=ints(4, V, d) / 8 * (torch.rand(V, d, generator=g, device="cuda") < 12.0 / d))
    if abs(base) > 1e7:
        s["w"].zero_()
        s["w"][:, 3] = ints(2, V)                                    # beside such a base products of +-2 vanish
        s["h"][:, 3] = ints(1, N)
    s["b"] = ints(16, V) / 8 * (abs(base) <= 1e7) + base if bias_on else None
    if not bias_on:                                                  # each row with a base of its own, from its first column
        s["w"][:, 0] = 1.0
        s["h"][:, 0] = torch.tensor([0.0, 96.0, -160.0, base, -base, 4096.0, -16384.0, 1.0], device="cuda").repeat(N // 8 + 1)[:N]
    s["h"], s["w"] = s["h"].to(DT[dtype]), s["w"].to(DT[dtype])
    s["target"] = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    s["target"][torch.rand(N, generator=g, device="cuda") < 0.1] = -1
    s["target"][0] = V - 1
    s["dlogprob"] = torch.randn(N, generator=g, device="cuda") / N
    return s


def gradients(s, dtype):
    """The gradients in float64 from the binary32 logits, with their bounds."""
    step, half = ol.STEP, HALF[dtype]
    h, w, t = f64(s["h"]), f64(s["w"]), f64(s["target"]).astype(np.int64)
    on = ((t >= 0) & (t < w.shape[0]))[:, None]
    h = np.where(on, h, 0.0)
    z = h @ w.T
    z = np.float32(z + (0.0 if s["b"] is None else f64(s["b"]))).astype(np.float64)
    m = z.max(1, keepdims=True)
    e = np.exp(z - m)
    total = e.sum(1, keepdims=True)
    p, lse = e / total, m + np.log(total)
    near = np.where(abs(lse) < FAR[dtype], abs(lse) * 2.0 ** -24, 0.0)
    p_off = p * ((m - z + 24 + 8) * step + 1.01 * near)
    hit = np.zeros_like(p)
    np.put_along_axis(hit, np.clip(t, 0, None)[:, None], 1.0, 1)
    g = np.where(on, f64(s["dlogprob"])[:, None], 0.0)
    top = abs(g).max()
    g = g / top
    dz = ol.Bounded(g, abs(g) * step) * ol.Bounded(hit - p, p_off + step * abs(hit - p))
    scale = ol.Bounded(np.full((1, 1), top))
    dzr = dz.rounded(half)
    db = ((ol.Bounded(np.ones((1, h.shape[0]))) @ dz) * scale).rounded(2.0 ** -24)
    return dict(dh=((dzr @ ol.Bounded(w)) * scale).rounded(half), dw_head=((dzr.T @ ol.Bounded(h)) * scale).rounded(half),
                db_head=ol.Bounded(db.value[0], db.off[0]))


def check(s, dtype, got):
    for k, want in gradients(s, dtype).items():
        if got[k] is None:
            continue
        v = f64(got[k])
        ok = abs(v - want.value) <= want.off + 1e-37
        assert ok.all(), (k, int((~ok).sum()), float(abs(v - want.value).max()), float(abs(want.value).max()))


def run(s):
    import paper_2605_11537_amd as moe
    out = moe.moe_head_logprobs(s["h"], s["w"], s["target"], s["b"])
    return out, moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], out["lse"], s["dlogprob"], s["b"])


# tiles whose wavefronts share the sum, of 16 rows, 32 (binary32), 64 and more
SIZES = [(1, 16, 64), (18, 64, 64), (130, 1032, 500), (16, 24, 9000), (20, 40, 9001), (100, 136, 1500), (350, 72, 400), (700, 264, 2049)]


@pytest.mark.parametrize("base", [200.0, -300.0, 3000.0, -1e6, -1e9, LOWEST])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d,V", SIZES)
def test_biases_far_from_zero(N, d, V, dtype, base):
    s = make(dtype, N, d, V, base, N + V)
    _, got = run(s)
    check(s, dtype, got)


@pytest.mark.parametrize("base", [3000.0, -1e9])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d,V", [(600, 16, 20001), (4096, 16, 300), (4097, 16, 300), (9001, 24, 77)])
def test_many_rows_and_many_ids(N, d, V, dtype, base):
    """More than 64 tiles to a row, and as many rows as the launch that makes them again looks at, or more."""
    s = make(dtype, N, d, V, base, N + V)
    check(s, dtype, run(s)[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d,V", [(18, 64, 64), (20, 40, 9001), (100, 136, 1500), (700, 264, 2049), (600, 16, 20001), (5000, 16, 300)])
def test_rows_far_and_near_side_by_side(N, d, V, dtype):
    """Rows near zero get the same bits whether others are far or not."""
    s = make(dtype, N, d, V, 2560.0, N + V, bias_on=False)
    s["h"][s["target"] < 0] = float("nan")
    s["dlogprob"][0] = 1.0                                           # a near row has the largest
    out, got = run(s)
    check(s, dtype, got)
    near = out["lse"].abs() < 40
    assert near[0] and not near.all()
    alone = run(dict(s, target=torch.where(near, s["target"], -1)))[1]["dh"]
    assert torch.equal(alone[near], got["dh"][near])


@pytest.mark.parametrize("N,V", [(1, 700), (1, 9001), (40, 9001), (300, 2049)])
def test_binary32_exponentials(N, V):
    """Far below the largest logit, whose sum is 1: an exponential keeps binary32's accuracy whatever its argument (exact here).  A step each for the exponential, what
    its exponent's product has lost, three products; the rows' sum is of N equal terms."""
    g = torch.Generator(device="cuda").manual_seed(V)
    b = 4096.0 - torch.randint(40 * 8, 84 * 8, (V,), generator=g, device="cuda").float() / 8
    b[5] = 4096.0
    s = dict(h=torch.zeros(N, 16, device="cuda"), w=torch.zeros(V, 16, device="cuda"), b=b, target=torch.full((N,), 5, dtype=torch.int32, device="cuda"),
             dlogprob=torch.ones(N, device="cuda"))
    db = run(s)[1]["db_head"].double()
    want = -N * torch.exp(b.double() - 4096.0)
    off = (db - want).abs() > (5 + N.bit_length()) * ol.STEP * want.abs()
    off[5] = False
    assert not off.any(), float(((db - want) / want).abs()[off].max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pieces_and_equal_bits(dtype):
    """Far rows in a vocabulary of which one piece's gradient is in memory at a time, and one gradient alone."""
    import paper_2605_11537_amd as moe
    N, d, V = 30000, 8, (20001 if dtype == "bf16" else 10001)
    s = make(dtype, N, d, V, -1e9, 5)
    out, got = run(s)
    p = 1.0 / V
    t, on = s["target"].long(), s["target"] >= 0
    g = torch.where(on, s["dlogprob"].double(), 0.0)
    want = -p * g.sum() * torch.ones(V, dtype=torch.float64, device="cuda")
    want.index_add_(0, t.clamp(min=0), g)
    # p off by some 40 steps; of a sum's parts some ten hold a target's share, and a dozen additions of half a step each
    room = 1e-5 * p * g.abs().sum() + 2.0 ** -16 * g.abs().max()
    assert ((got["db_head"].double() - want).abs() <= room).all()
    for k in ("dh", "dw_head", "db_head"):
        one = dict(dh=None, dw_head=None, db_head=None)
        one[k] = torch.empty_like(got[k])
        moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], out["lse"], s["dlogprob"], s["b"], out=one)
        assert torch.equal(one[k], got[k]), k


def test_in_a_graph():
    """Captured where all rows are near, replayed where they are far and near again."""
    import paper_2605_11537_amd as moe
    a, b = make("bf16", 100, 136, 1500, 0.0, 1), make("bf16", 100, 136, 1500, -1e6, 2)
    s = {k: v.clone() for k, v in a.items()}
    lse, out = torch.empty(100, device="cuda"), {}
    need = moe.lib().moe_head_logprobs_backward_workspace_bytes(100, 136, 1500, moe.MOE_BF16)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    want = [run(v)[1] for v in (a, b)]
    lses = [run(v)[0]["lse"] for v in (a, b)]
    out = {k: torch.empty_like(v) for k, v in want[0].items()}
    call = lambda: moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], lse, s["dlogprob"], s["b"], out=out, ws=ws)
    lse.copy_(lses[0])
    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in (0, 1, 1, 0, 1, 0):
        for k in s:
            s[k].copy_((a, b)[i][k])
        lse.copy_(lses[i])
        ws.random_(0, 256)
        for v in out.values():
            v.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[i][k]) for k in out), i
