"""moe_head_logprobs where every logit of a row lies far below zero, beside columns that are not there or are masked: a wavefront's columns, a tile's, several tiles'.
Against oracle/learning.py in float64, within the bounds that it carries along."""
import numpy as np
import pytest
import torch

from oracle import learning as ol
from test_gpu_gated_ffn import f64
from test_gpu_head_logprobs import inputs, want_of

pytestmark = pytest.mark.gpu

SIZES = [(1, 64, 77), (18, 2048, 8), (130, 1032, 500), (16, 24, 9000), (20, 40, 9001), (100, 136, 1500), (350, 72, 400), (700, 264, 2049), (3, 64, 20001)]


@pytest.mark.parametrize("masked", [None, (0, 64), (17, 1100), (128, 100000)])
@pytest.mark.parametrize("base", [-70.0, -100.0, -300.0, -20000.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d,V", SIZES)
def test_scores(N, d, V, dtype, base, masked):
    import paper_2605_11537_amd as moe
    s = inputs(dtype, N, d, V, True, 0.1, N + V)
    s["b"] += base
    if masked and masked[0] < V:
        s["b"][masked[0]:masked[1]] = -float("inf")
    if masked and masked[0] == 0:
        s["b"][V // 2] = base                                        # one id at least
    want = want_of(s, dtype)
    got = moe.moe_head_logprobs(s["h"], s["w"], s["target"], s["b"])
    for k in ("lse", "logprob"):
        v, w = f64(got[k]), want[k].value
        none = np.isneginf(w)
        assert (np.isneginf(v) == none).all()
        ok = abs(v[~none] - w[~none]) <= want[k].off[~none] + 1e-37
        assert ok.all(), (k, int((~ok).sum()), int(np.isnan(v).sum()))
