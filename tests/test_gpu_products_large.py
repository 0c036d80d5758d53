"""The gated experts' and the head's calls where a workgroup has several tiles of a product, tiles of every size, sums in parts and two products in a launch;
and on tensors whose offsets pass 32 bits.  The bounds of oracle/learning.py, carried along on the card in float64."""
import numpy as np
import pytest
import torch

from oracle import learning as ol
from test_gpu_gated_ffn import ACT, DT, HALF, f64, inputs, near
from test_gpu_head_logprobs import inputs as head_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def near_here(got, want, what):
    over = (got.double() - want.value).abs() > want.off + 1e-37
    over |= got.isnan()
    assert not over.any(), (what, int(over.sum()), over.nonzero()[:4].tolist())


# dtype, act, rows of the experts, d, F: what is left of the last round in halves .. sixteenths, long sums in few tiles (parts of the rows), both pairs,
# experts without rows among many
GATED = [
    ("bf16", "silu", [1300, 0, 270, 5, 2049, 700, 1, 300], 768, 1376), ("bf16", "gelu", [5000], 512, 4096), ("bf16", "silu", [16000], 256, 264),
    ("bf16", "relu", [8192], 1024, 4096), ("bf16", "silu", [2100, 900, 1500, 40, 1024, 600, 0, 3000], 1024, 2816), ("bf16", "silu", [20] * 100 + [0] * 20, 256, 2048),
    ("f32", "silu", [91, 8, 16, 94, 0, 30, 10] * 4, 512, 1376), ("f32", "gelu", [3000], 264, 520), ("f32", "silu", [700, 0, 1300, 129], 512, 2048),
    ("f32", "relu", [2400], 136, 1976), ("f32", "silu", [500, 620, 100], 1544, 1032),
    # tiles of 64 x 64 for long sums, tiles whose wavefronts share the sum
    ("bf16", "silu", [1334], 512, 2048), ("bf16", "gelu", [300, 0, 1200, 257, 513], 264, 1376), ("bf16", "relu", [30], 1024, 4096), ("bf16", "silu", [200], 768, 2056),
    ("f32", "silu", [200], 768, 2056), ("f32", "gelu", [40, 0, 90], 264, 1376),
]


@pytest.mark.parametrize("dtype,act,counts,d,F", GATED, ids=range(len(GATED)))
def test_gated(dtype, act, counts, d, F):
    import paper_2605_11537_amd as moe
    print(dtype, act, counts[:8], d, F, flush=True)
    K, R = sum(counts), sum(counts) + 3
    s = inputs(dtype, counts, R, d, F, K)
    s["x"][K:], s["dy"][K:] = float("nan"), float("nan")
    y, states = moe.moe_gated_ffn(s["x"], *s["w"], s["offset"], ACT[act], want_states=True)
    grads = moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, s["offset"], ACT[act])
    for e, (lo, hi) in enumerate(zip(s["first"], s["first"][1:])):
        if lo == hi:
            assert not any(grads[k][e].any() for k in ("dw_gate", "dw_up", "dw_down"))
            continue
        want = ol.gated_ffn(s["x"][lo:hi].double(), *(w[e].double() for w in s["w"]), act, HALF[dtype], s["dy"][lo:hi].double())
        near_here(y[lo:hi], want["y"], (e, "y"))
        near_here(grads["dx"][lo:hi], want["dx"], (e, "dx"))
        for k in ("dw_gate", "dw_up", "dw_down"):
            near_here(grads[k][e], want[k], (e, k))
    again = moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, s["offset"], ACT[act])
    assert all(torch.equal(again[k], grads[k]) for k in grads)


def head_here(s, dtype):
    """The head's gradient on the card: values in float64, the bounds of its two products (each rounding of dz, the logits', the sums')."""
    half, step = HALF[dtype], ol.STEP
    h, w = s["h"].double(), s["w"].double()
    on = s["target"] >= 0
    z = ol.Bounded(h) @ ol.Bounded(w.t())
    value = z.value + (0.0 if s["b"] is None else s["b"].double())
    lse = torch.logsumexp(value, 1, keepdim=True)
    p = torch.exp(value - lse)
    off = z.off + step * value.abs()
    lse_off = (p * (1.01 * off + (lse - value + 8) * step)).sum(1, keepdim=True) + (64 + w.shape[0] / 4096) * step + 2 * step * lse.abs()
    p_off = 1.01 * p * (off + lse_off + ((value - lse).abs() + 8) * step) + step
    top = float(s["dlogprob"][on].abs().max())
    g = torch.where(on, s["dlogprob"].double(), 0.0)[:, None] / top
    dz = -g * p
    dz.scatter_add_(1, s["target"].long().clamp(min=0)[:, None], g)
    dz = ol.Bounded(dz, g.abs() * p_off + step * dz.abs())
    dzr, scale = dz.rounded(half), ol.Bounded(torch.full((1, 1), top, dtype=torch.float64, device="cuda"))
    lp = torch.where(on, value.gather(1, s["target"].long().clamp(min=0)[:, None])[:, 0] - lse[:, 0], 0.0)
    lp_off = off.gather(1, s["target"].long().clamp(min=0)[:, None])[:, 0] + lse_off[:, 0] + 4 * step * (lp.abs() + lse[:, 0].abs())
    out = dict(logprob=ol.Bounded(lp, lp_off), lse=ol.Bounded(lse[:, 0], lse_off[:, 0]), dh=((dzr @ ol.Bounded(w)) * scale).rounded(half),
               dw_head=((dzr.T @ ol.Bounded(torch.where(on[:, None], h, 0.0))) * scale).rounded(half))
    ones = ol.Bounded(torch.ones(1, h.shape[0], dtype=torch.float64, device="cuda"))
    db = ((ones @ dz) * scale).rounded(2.0 ** -24)
    out["db_head"] = ol.Bounded(db.value[0], db.off[0])
    return out


# many tiles of a row, one of each size, dh in many parts, dW in parts of the rows, both in one launch, an odd vocabulary
HEAD = [("bf16", 3000, 264, 20001, True), ("bf16", 4096, 256, 128, True), ("bf16", 15009, 520, 256, True), ("bf16", 9000, 768, 33001, False),
        ("bf16", 700, 1024, 9973, False), ("f32", 777, 320, 5003, True), ("f32", 5000, 264, 300, True), ("f32", 2500, 512, 12007, False), ("bf16", 100, 768, 70001, False),
        ("f32", 900, 136, 6001, True), ("f32", 1400, 72, 5003, False)]


@pytest.mark.parametrize("dtype,N,d,V,bias", HEAD, ids=range(len(HEAD)))
def test_head(dtype, N, d, V, bias):
    import paper_2605_11537_amd as moe
    print(dtype, N, d, V, flush=True)
    s = head_inputs(dtype, N, d, V, bias, 0.1, N + V)
    want = head_here(s, dtype)
    s["h"][s["target"] < 0] = float("nan")
    out = dict(moe.moe_head_logprobs(s["h"], s["w"], s["target"], s["b"]))
    on = s["target"] >= 0
    near_here(out["lse"][on], ol.Bounded(want["lse"].value[on], want["lse"].off[on]), "lse")
    near_here(out["logprob"], want["logprob"], "logprob")
    out.update(moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], out["lse"], s["dlogprob"], s["b"]))
    for k in ("dh", "dw_head") + (("db_head",) if bias else ()):
        near_here(out[k], want[k], k)
    again = moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], out["lse"], s["dlogprob"], s["b"])
    assert all(torch.equal(again[k], out[k]) for k in ("dh", "dw_head"))


def test_gated_far_offsets():
    """Rows, hidden rows and states past 4 GB, two experts' weights past 4 GB; rows and weights from both ends."""
    import paper_2605_11537_amd as moe
    g = torch.Generator(device="cuda").manual_seed(1)
    for R, E, d, F in ((300001, 1, 64, 8192), (60, 3, 8192, 65536 + 8)):
        print(R, E, d, F, flush=True)
        n = lambda *s, std: torch.empty(*s, dtype=torch.bfloat16, device="cuda").normal_(generator=g).mul_(std)
        x, dy = n(R, d, std=1.0), n(R, d, std=0.1)
        w = n(E, d, F, std=d ** -0.5), n(E, d, F, std=d ** -0.5), n(E, F, d, std=F ** -0.5)
        first = [0] + [R * (i + 1) // E for i in range(E)]
        table = torch.tensor(first, dtype=torch.int32, device="cuda")
        y, states = moe.moe_gated_ffn(x, *w, table, want_states=True)
        dx = torch.empty_like(x)
        grads = moe.moe_gated_ffn_backward(dy, x, *w, states, table, out=dict(dx=dx, dw_gate=torch.empty_like(w[0]), dw_up=torch.empty_like(w[1]),
                                                                            dw_down=torch.empty_like(w[2])))
        for e in (0, E - 1):
            lo, hi = first[e], first[e + 1]
            rows = list(range(lo, min(lo + 7, hi))) + list(range(max(lo, hi - 7), hi))
            want = ol.gated_ffn(x[rows].double(), *(v[e].double() for v in w), "silu", HALF["bf16"], dy[rows].double())
            near_here(y[rows], want["y"], (e, "y"))
            near_here(dx[rows], want["dx"], (e, "dx"))
            if hi - lo < 100:                                        # all rows of the expert are few: its weights' gradients at both ends
                full = ol.gated_ffn(x[lo:hi].double(), *(v[e].double() for v in w), "silu", HALF["bf16"], dy[lo:hi].double())
                for k in ("dw_gate", "dw_up", "dw_down"):
                    near_here(grads[k][e], full[k], (e, k))
                del full
            del want
        del x, dy, w, y, states, dx, grads
        torch.cuda.empty_cache()


def test_head_far_offsets():
    """A head of more than 4 GB, few rows; and rows past 4 GB under a small one, of which the last ones count."""
    import paper_2605_11537_amd as moe
    g = torch.Generator(device="cuda").manual_seed(2)
    N, d, V = 20, 1024, (1 << 21) + 77
    w = torch.empty(V, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g).mul_(d ** -0.5)
    h = torch.empty(N, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    target = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    target[0], target[1], target[2] = V - 1, 0, -1
    s = dict(h=h, w=w, b=None, target=target, dlogprob=torch.full((N,), -1.0 / N, device="cuda"))
    out = dict(moe.moe_head_logprobs(h, w, target))
    out.update(moe.moe_head_logprobs_backward(h, w, target, out["lse"], s["dlogprob"]))
    value = torch.cat([h.double() @ w[i:i + 262144].double().t() for i in range(0, V, 262144)], 1)
    lse = torch.logsumexp(value, 1)
    on = target >= 0
    lp = torch.where(on, value.gather(1, target.long().clamp(min=0)[:, None])[:, 0] - lse, 0.0)
    mag = h.double().abs().sum(1) * float(w.abs().max())
    e = (d + 4) * ol.STEP * mag + (64 + V / 4096) * ol.STEP + 8 * ol.STEP * lse.abs() + 30 * ol.STEP
    assert ((out["logprob"].double() - lp).abs() <= 2 * e).all() and ((out["lse"].double() - lse).abs() <= e).all()
    dz = torch.where(on, s["dlogprob"].double(), 0.0)[:, None] * -torch.exp(value - lse[:, None])
    dz.scatter_add_(1, target.long().clamp(min=0)[:, None], torch.where(on, s["dlogprob"].double(), 0.0)[:, None])
    ids = torch.cat([target[on].long(), torch.tensor([0, 1, V - 1, V - 2, V // 2], device="cuda")])
    want = dz[:, ids].t() @ h.double()
    room = dz[:, ids].abs().t() @ h.double().abs()
    assert ((out["dw_head"][ids].double() - want).abs() <= HALF["bf16"] * want.abs() + room * (1.01 * HALF["bf16"] + 4 * float(e.max()))).all()
    del w, value, out
    torch.cuda.empty_cache()
    N, d, V = (1 << 22) + 5, 520, 8
    h = torch.empty(N, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = torch.empty(V, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g).mul_(d ** -0.5)
    target = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    target[-300:] = 3
    dl = torch.full((N,), -1.0 / 300, device="cuda")
    out = dict(moe.moe_head_logprobs(h, w, target))
    out.update(moe.moe_head_logprobs_backward(h, w, target, out["lse"], dl))
    tail = dict(h=h[-300:].contiguous(), w=w, b=None, target=target[-300:].contiguous(), dlogprob=dl[-300:].contiguous())
    want = head_here(tail, "bf16")
    near_here(out["logprob"][-300:], want["logprob"], "logprob")
    near_here(out["dh"][-300:], want["dh"], "dh")
    near_here(out["dw_head"], want["dw_head"], "dw_head")
    assert not out["dh"][:-300].any()


def test_clip_far_offsets():
    import paper_2605_11537_amd as moe
    g = torch.Generator(device="cuda").manual_seed(3)
    t = torch.empty((1 << 32) + 1001, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    ends = torch.cat([t[:1000], t[-1000:]])
    total = sum(float(p.double().square().sum()) for p in t.split(1 << 28)) ** 0.5
    norm, out = moe.moe_clip_gradients([t], 0.5 * total, out=[t])
    assert abs(float(norm) - total) <= 2.0 ** -24 * 1.01 * total
    v = ends.double() * (np.float32(0.5 * total).item() / total)
    assert ((torch.cat([t[:1000], t[-1000:]]).double() - v).abs() <= v.abs() * (2.0 ** -8 + 2.0 ** -22)).all()
