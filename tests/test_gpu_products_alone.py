"""Each gradient of moe_gated_ffn_backward and moe_head_logprobs_backward has the same bits whichever others are asked for: where products share a launch, where their
sums are in parts, and where neither is so."""
import itertools

import pytest
import torch

from test_gpu_gated_ffn import inputs
from test_gpu_head_logprobs import inputs as head_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,counts,d,F", [
    ("bf16", [8192], 1024, 4096), ("bf16", [2100, 900, 1500, 40, 1024, 600, 0, 3000], 1024, 2816), ("bf16", [16000], 256, 264), ("bf16", [400] * 64, 512, 1376),
    ("bf16", [300, 0, 1200, 257, 513], 264, 1376), ("bf16", [20] * 40, 256, 512), ("bf16", [5000, 4000], 2048, 512), ("f32", [700, 0, 1300, 129], 512, 2048),
    ("f32", [2400], 136, 1976), ("f32", [500, 620, 100], 1544, 1032), ("f32", [91, 8, 16, 94, 0, 30, 10] * 4, 512, 1376)])
def test_gated(dtype, counts, d, F):
    import paper_2605_11537_amd as moe
    s = inputs(dtype, counts, sum(counts), d, F, 3)
    y, states = moe.moe_gated_ffn(s["x"], *s["w"], s["offset"], want_states=True)
    whole = moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, s["offset"])
    groups = [("dx",), ("dw_gate", "dw_up"), ("dw_down",)]
    for n in (1, 2):
        for some in itertools.combinations(groups, n):
            names = sum(some, ())
            out = {k: torch.full_like(v, 7.0) if k in names else None for k, v in whole.items()}
            moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, s["offset"], out=out)
            assert all(torch.equal(out[k], whole[k]) for k in names), names


@pytest.mark.parametrize("dtype,N,d,V", [("bf16", 9000, 768, 33001), ("bf16", 15009, 520, 256), ("bf16", 100, 136, 1500), ("bf16", 16, 24, 9000), ("bf16", 18, 2048, 8),
                                         ("f32", 2500, 512, 12007), ("f32", 777, 320, 5003), ("f32", 5000, 264, 300)])
def test_head(dtype, N, d, V):
    import paper_2605_11537_amd as moe
    s = head_inputs(dtype, N, d, V, True, 0.1, 4)
    lse = moe.moe_head_logprobs(s["h"], s["w"], s["target"], s["b"])["lse"]
    whole = moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], lse, s["dlogprob"], s["b"])
    for n in (1, 2):
        for names in itertools.combinations(whole, n):
            out = {k: torch.full_like(v, 7.0) if k in names else None for k, v in whole.items()}
            moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], lse, s["dlogprob"], s["b"], out=out)
            assert all(torch.equal(out[k], whole[k]) for k in names), names
