"""moe_head_logprobs_backward over a vocabulary in several pieces, whose logits' gradients take turns in the workspace: against float64 on the card, each gradient
alone, and targets on both sides of the pieces' borders."""
import pytest
import torch

from test_gpu_head_logprobs import inputs
from test_gpu_products_large import head_here, near_here

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def pieces_of(dtype, N, V):
    """First ids of the pieces: as many as 1 GiB of gradients asks for, of equal size up to 256."""
    fits = max(256, (1 << 30) // (N * (4 if dtype == "f32" else 2)) // 256 * 256)
    n = -(-V // min(fits, V))
    size = -(-(-(-V // n)) // 256) * 256
    return list(range(0, V, size))


# three and two pieces, an odd last one; dh and dW in launches of their own, in one launch; few rows; dh in parts
CASES = [("bf16", 60000, 64, 20001, True), ("f32", 20501, 72, 20001, False), ("bf16", 8200, 512, 70001, False), ("f32", 8200, 264, 33001, True), ("bf16", 100, 8, 5500001, True),
         ("f32", 150, 16, 1800003, False)]


@pytest.mark.parametrize("dtype,N,d,V,bias", CASES, ids=range(len(CASES)))
def test_gradients(dtype, N, d, V, bias):
    import paper_2605_11537_amd as moe
    print(dtype, N, d, V, flush=True)
    s = inputs(dtype, N, d, V, bias, 0.1, N + V)
    first = pieces_of(dtype, N, V)
    assert len(first) > 1
    edges = [v + i for v in first for i in (-1, 0)][1:] + [V - 1]
    s["target"][:len(edges)] = torch.tensor(edges, dtype=torch.int32, device="cuda")
    lse = moe.moe_head_logprobs(s["h"], s["w"], s["target"], s["b"])["lse"]
    want = head_here(s, dtype)
    kept = {k: want[k] for k in ("dh", "dw_head", "db_head")}
    near_here(lse, want["lse"], "lse")
    del want
    s["h"][s["target"] < 0] = float("nan")
    got = moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], lse, s["dlogprob"], s["b"])
    for k, v in kept.items():
        if k != "db_head" or bias:
            near_here(got[k], v, k)
    for k in ("dh", "dw_head", "db_head"):
        if got[k] is None:
            continue
        one = dict(dh=None, dw_head=None, db_head=None)
        one[k] = torch.full_like(got[k], 7.0)
        moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], lse, s["dlogprob"], s["b"], out=one)
        assert torch.equal(one[k], got[k]), k
