"""moe_token_logprobs and its gradient on very many short rows, held bit for bit against the same rows in a small batch (which the other tests hold
against float64)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_sixteen_million_rows():
    """Rows as short as a gate over eight experts are not refused for their number."""
    import paper_2605_11537_amd as moe
    N, V = (1 << 24) + 37, 8
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.empty(N, V, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    t = (torch.arange(N, device="cuda") % 9).int()
    dl = torch.empty(N, device="cuda").normal_(generator=g)
    s = moe.moe_token_logprobs(x, t, 2)
    d = moe.moe_token_logprobs_backward(x, t, s["lse"], s["entropy"], dl, dl)
    for part in (slice(0, 50), slice(N // 2, N // 2 + 50), slice(N - 50, N)):
        few = moe.moe_token_logprobs(x[part].clone(), t[part].clone(), 2)
        assert all(torch.equal(few[key], s[key][part]) for key in few)
        assert torch.equal(moe.moe_token_logprobs_backward(x[part].clone(), t[part].clone(), few["lse"], few["entropy"], dl[part].clone(), dl[part].clone()),
                           d[part])
