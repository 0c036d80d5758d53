"""The gated experts' and the head's products on small whole numbers, whose sums binary32 holds: every element has to be the exact sum, rounded once to the
tensors' type, whatever its length, so that a lost or doubled term of some thousand is seen."""
import pytest
import torch

from test_gpu_gated_ffn import DT

pytestmark = pytest.mark.gpu


def sparse(g, share, *s):
    return torch.randint(0, 2, s, generator=g, device="cuda").mul_(2).sub_(1).float() * (torch.rand(*s, generator=g, device="cuda") < share)


def same(got, want, dtype, what):
    over = got.double() != want.to(DT[dtype]).double()
    assert not over.any(), (what, int(over.sum()), over.nonzero()[:4].tolist())


# rows of the experts, d, F: every kind of tile, pairs, parts of the rows, rows left over
GATED = [([1], 768, 2048), ([2, 0, 5, 1], 264, 3176), ([40, 0, 90], 512, 1376), ([200], 768, 2056), ([20] * 64, 256, 2048), ([1334], 512, 2048),
         ([1300, 0, 270, 5, 2049, 700, 1, 300], 768, 1376), ([16000], 256, 264), ([8192], 512, 2048), ([4100, 900, 40, 3000], 1024, 1032)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,d,F", GATED, ids=range(len(GATED)))
def test_gated(counts, d, F, dtype):
    import paper_2605_11537_amd as moe
    print(counts[:8], d, F, flush=True)
    g = torch.Generator(device="cuda").manual_seed(d + F)
    E, R, t = len(counts), sum(counts), DT[dtype]
    first = [0]
    for n in counts:
        first.append(first[-1] + n)
    x, dy = sparse(g, 0.25, R, d), sparse(g, 0.25, R, d)
    w = sparse(g, 8.0 / d, E, d, F), sparse(g, 8.0 / d, E, d, F), sparse(g, 8.0 / d, E, F, d)
    offset = torch.tensor(first, dtype=torch.int32, device="cuda")
    y, states = moe.moe_gated_ffn(x.to(t), *(v.to(t) for v in w), offset, moe.ACT_RELU, want_states=True)
    whole = [dy.to(t), x.to(t)] + [v.to(t) for v in w] + [states, offset, moe.ACT_RELU]
    grads = moe.moe_gated_ffn_backward(*whole)
    plain = moe.moe_gated_ffn(x.to(t), *(v.to(t) for v in w), offset, moe.ACT_RELU)[0]
    for e, (lo, hi) in enumerate(zip(first, first[1:])):
        xe, dye, wg, wu, wd = (v.double() for v in (x[lo:hi], dy[lo:hi], w[0][e], w[1][e], w[2][e]))
        gate, up, dh = xe @ wg, xe @ wu, dye @ wd.t()
        h, dg, du = gate.clamp(min=0) * up, dh * up * (gate > 0), dh * gate.clamp(min=0)
        if hi > lo:
            assert max(float(v.abs().max()) for v in (h, dg, du)) <= 256            # what bfloat16 holds of whole numbers
        same(y[lo:hi], h @ wd, dtype, (e, "y"))
        same(plain[lo:hi], h @ wd, dtype, (e, "plain y"))
        same(grads["dx"][lo:hi], dg @ wg.t() + du @ wu.t(), dtype, (e, "dx"))
        same(grads["dw_gate"][e], xe.t() @ dg, dtype, (e, "dw_gate"))
        same(grads["dw_up"][e], xe.t() @ du, dtype, (e, "dw_up"))
        same(grads["dw_down"][e], h.t() @ dye, dtype, (e, "dw_down"))


# tiles of every kind, dh and dW in parts, in one launch, one after the other
HEAD = [(1, 2056, 8192), (130, 1032, 500), (16, 264, 9000), (100, 136, 6001), (190, 72, 6001), (700, 1024, 9973), (3000, 264, 20001), (15009, 520, 256), (9000, 768, 33001), (4096, 256, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d,V", HEAD, ids=range(len(HEAD)))
def test_head(N, d, V, dtype):
    """Logits of zero under a log sum of zero have e^0 = 1 for a probability: dz is -1, and 0 at the target."""
    import paper_2605_11537_amd as moe
    print(N, d, V, flush=True)
    g = torch.Generator(device="cuda").manual_seed(N + V)
    t = DT[dtype]
    target = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    target[torch.rand(N, generator=g, device="cuda") < 0.1] = -1
    target[0] = V - 1
    on = target >= 0
    lse, one, none = torch.zeros(N, device="cuda"), torch.ones(N, device="cuda"), torch.zeros(V, device="cuda")
    rows, ids = sparse(g, 0.3, N, d), sparse(g, 0.3, V, d)
    kept = torch.where(on[:, None], rows, 0.0).double()
    dw = -kept.sum(0, keepdim=True).expand(V, d).clone()
    dw.index_add_(0, target[on].long(), kept[on])
    db = -on.double().sum().expand(V).clone()
    db.index_add_(0, target[on].long(), torch.ones_like(target[on], dtype=torch.float64))
    dh = torch.where(on[:, None], ids.double()[target.long().clamp(min=0)] - ids.double().sum(0, keepdim=True), 0.0)
    got = moe.moe_head_logprobs_backward(rows.to(t), torch.zeros(V, d, dtype=t, device="cuda"), target, lse, one, none)
    same(got["dw_head"], dw, dtype, "dw_head")
    assert torch.equal(got["db_head"].double(), db) and not got["dh"].any()
    got = moe.moe_head_logprobs_backward(torch.zeros(N, d, dtype=t, device="cuda"), ids.to(t), target, lse, one, none)
    same(got["dh"], dh, dtype, "dh")
    assert torch.equal(got["db_head"].double(), db) and not got["dw_head"].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d,V", HEAD, ids=range(len(HEAD)))
def test_head_scores(N, d, V, dtype):
    """Whole logits: their log sum is off by the exponentials and the sum's joins alone (oracle/learning.py), whatever d is."""
    import paper_2605_11537_amd as moe
    g = torch.Generator(device="cuda").manual_seed(N + V + 1)
    t, step = DT[dtype], 2.0 ** -23
    h, w = sparse(g, 0.3, N, d), sparse(g, min(1.0, 8.0 / d), V, d)
    target = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    got = moe.moe_head_logprobs(h.to(t), w.to(t), target)
    z = h.double() @ w.double().t()
    lse = torch.logsumexp(z, 1)
    far = (torch.softmax(z, 1) * (z.amax(1, keepdim=True) - z + 8)).sum(1)
    room = (far + 64 + V / 4096 + 2 * lse.abs()) * step
    at = z.gather(1, target.long()[:, None])[:, 0]
    assert ((got["lse"].double() - lse).abs() <= room).all()
    assert ((got["logprob"].double() - (at - lse)).abs() <= room + 4 * step * (at - lse).abs()).all()
