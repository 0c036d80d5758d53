"""moe_head_logprobs and its gradient against oracle/learning.py in float64, within the bounds that it carries along: binary32 products, exponentials and
sums, one rounding of dz, one of the result."""
import numpy as np
import pytest
import torch

from oracle import learning as ol
from test_gpu_gated_ffn import DT, HALF, f64, near

pytestmark = pytest.mark.gpu


def inputs(dtype, N, d, V, bias, padded, seed, std=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(h=torch.randn(N, d, generator=g, device="cuda").to(DT[dtype]), w=(torch.randn(V, d, generator=g, device="cuda") * std * d ** -0.5).to(DT[dtype]),
             b=torch.randn(V, generator=g, device="cuda") if bias else None,
             target=torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32),
             dlogprob=torch.randn(N, generator=g, device="cuda") / max(N, 1))
    s["target"][torch.rand(N, generator=g, device="cuda") < padded] = -1
    return s


def want_of(s, dtype):
    h = f64(s["h"])
    return ol.head_logprobs(np.where(np.isfinite(h), h, 0.0), f64(s["w"]), None if s["b"] is None else f64(s["b"]), s["target"].cpu().numpy().astype(np.int64),
                            HALF[dtype], f64(s["dlogprob"]))


def run(moe, s):
    out = dict(moe.moe_head_logprobs(s["h"], s["w"], s["target"], s["b"]))
    out.update(moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], out["lse"], s["dlogprob"], s["b"]))
    return out


def check(got, want, bias):
    for k, v in want.items():
        if k == "db_head" and not bias:
            assert got[k] is None
            continue
        inf = np.isneginf(v.value)
        assert (np.isneginf(f64(got[k])) == inf).all(), k
        if not inf.all():
            keep = ~inf
            a, b = f64(got[k])[keep], ol.Bounded(v.value[keep], v.off[keep])
            near(torch.from_numpy(a), b, k)


CASES = [
    (1, 8, 1, 0.0), (1, 8, 2, 0.0), (1, 768, 5003, 0.0), (3, 64, 20001, 0.0), (15, 72, 127, 0.2), (16, 128, 129, 0.0), (17, 136, 255, 0.3), (64, 64, 64, 1.0), (65, 200, 257, 0.1),
    (129, 256, 128, 0.05), (255, 264, 1003, 0.5), (257, 512, 513, 0.1), (700, 40, 2049, 0.1), (40, 1032, 300, 0.0), (2000, 16, 8, 0.1), (333, 8, 33, 0.0),
    # the wavefronts share a tile's sum: parts with one stage, many and none, as many tiles as compute units and one more row of them
    (18, 2048, 8, 0.1), (1, 2056, 8192, 0.0), (130, 1032, 500, 0.1), (4096, 72, 32, 0.1), (4097, 72, 32, 0.1), (2, 8, 8193, 0.0),
    # just beyond: tiles of 16, 64 and more rows
    (16, 24, 9000, 0.1), (100, 136, 1500, 0.1), (150, 40, 1003, 0.1), (350, 72, 400, 0.1), (20, 264, 6000, 0.1), (70, 136, 3001, 0.1), (130, 40, 2000, 0.1), (191, 24, 1500, 0.1),
]


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d,V,padded", CASES)
def test_scores_and_gradient(N, d, V, padded, dtype, bias):
    import paper_2605_11537_amd as moe
    s = inputs(dtype, N, d, V, bias, padded, N + d + V)
    got = run(moe, s)
    check(got, want_of(s, dtype), bias)
    off = s["target"] < 0
    assert not got["logprob"][off].any() and not got["dh"][off].any()
    # one gradient alone gives the same bits
    for k in ("dh", "dw_head", "db_head"):
        if got[k] is None:
            continue
        out = dict(dh=None, dw_head=None, db_head=None)
        out[k] = torch.full_like(got[k], 7.0)
        moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], got["lse"], s["dlogprob"], s["b"], out=out)
        assert torch.equal(out[k], got[k]), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(5, 400), (90, 400), (300, 400), (12, 9000), (90, 4000), (300, 1500)])
def test_masked_ids_and_padded_rows(N, V, dtype):
    """Biases of -infinity and of the lowest value; rows of NaN and infinity at padded positions, and targets past the vocabulary, leave no trace."""
    import paper_2605_11537_amd as moe
    s = inputs(dtype, N, 64, V, True, 0.2, N)
    s["b"][::3], s["b"][1::7] = -float("inf"), torch.finfo(torch.float32).min
    s["target"][0], s["target"][1], s["target"][2], s["target"][3] = V, 2 ** 31 - 1, -2 ** 31, 3      # the last one is masked
    clean = want_of(s, dtype)
    off = (s["target"] < 0) | (s["target"] >= V)
    s["h"][off] = float("nan")
    s["h"][1] = float("inf")
    got = run(moe, s)
    for k in ("logprob", "dh"):
        assert not got[k][off].any()
    keep = ~off.cpu().numpy()
    for k in ("logprob", "lse", "dh"):
        v = clean[k]
        fin = np.isfinite(v.value[keep])
        assert (np.isneginf(f64(got[k])[keep]) == ~fin).all()
        near(torch.from_numpy(f64(got[k])[keep][fin]), ol.Bounded(v.value[keep][fin], v.off[keep][fin]), k)
    near(got["dw_head"], clean["dw_head"], "dw_head")
    near(got["db_head"], clean["db_head"], "db_head")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(3, 77), (100, 77), (200, 77), (3, 9000), (100, 2000), (200, 1000)])
def test_everything_masked(N, V, dtype):
    import paper_2605_11537_amd as moe
    s = inputs(dtype, N, 32, V, True, 0.3, N)
    s["b"].fill_(-float("inf"))
    got = run(moe, s)
    on = s["target"] >= 0
    assert torch.isneginf(got["lse"]).all() and torch.isneginf(got["logprob"][on]).all() and not got["logprob"][~on].any()
    check({k: got[k] for k in ("dh", "dw_head", "db_head")}, {k: v for k, v in want_of(s, dtype).items() if k.startswith("d")}, True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_weights_and_no_gradient(dtype):
    """A mean's equal dlogprob, one far above the others, all zero, none that counts."""
    import paper_2605_11537_amd as moe
    s = inputs(dtype, 200, 64, 300, True, 0.1, 9)
    for fill in (-1.0 / 180, 0.0, 3e-38, 1e30):
        s["dlogprob"].fill_(fill)
        check(run(moe, s), want_of(s, dtype), True)
    s["dlogprob"].fill_(1e-6)
    s["dlogprob"][7] = 1.0
    check(run(moe, s), want_of(s, dtype), True)
    s["target"].fill_(-1)
    got = run(moe, s)
    assert not any(got[k].any() for k in ("logprob", "dh", "dw_head", "db_head"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 1300])
def test_nan_and_infinity_stay_in_their_row(V, dtype):
    import paper_2605_11537_amd as moe
    s = inputs(dtype, 150, 64, V, False, 0.0, 10)
    good = run(moe, s)
    s["h"][4, 3], s["h"][149, 0] = float("nan"), float("inf")
    got = run(moe, s)
    rows = [i for i in range(150) if i not in (4, 149)]
    for k in ("logprob", "lse", "dh"):
        assert torch.equal(got[k][rows], good[k][rows]) and torch.isnan(got[k][4]).all() and torch.isnan(got[k][149]).all()


def test_no_rows():
    import paper_2605_11537_amd as moe
    s = inputs("bf16", 0, 64, 300, True, 0.0, 11)
    got = run(moe, s)
    assert got["logprob"].numel() == 0 and not got["dw_head"].any() and not got["db_head"].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_calls_give_equal_bits(dtype):
    import paper_2605_11537_amd as moe
    s = inputs(dtype, 700, 136, 3001, True, 0.1, 12)
    first = run(moe, s)
    for _ in range(2):
        again = run(moe, s)
        assert all(torch.equal(again[k], first[k]) for k in first)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 2, 511, 512, 513])
def test_few_rows_of_many_ids(N, dtype):
    """Rows in few workgroups each, whose tiles are masked as a whole, all but one id, and throughout."""
    import paper_2605_11537_amd as moe
    V = 9001
    s = inputs(dtype, N, 16, V, True, 0.0, 40 + N)
    s["b"][1000:7000] = -float("inf")
    s["target"][0] = 500
    want = want_of(s, dtype)
    got = moe.moe_head_logprobs(s["h"], s["w"], s["target"], s["b"])
    check(got, {k: want[k] for k in ("logprob", "lse")}, True)
    s["b"][:-1] = -float("inf")
    s["target"].fill_(V - 1)
    want = want_of(s, dtype)
    got = moe.moe_head_logprobs(s["h"], s["w"], s["target"], s["b"])
    check(got, {k: want[k] for k in ("logprob", "lse")}, True)
    s["b"][-1] = -float("inf")
    got = moe.moe_head_logprobs(s["h"], s["w"], s["target"], s["b"])
    assert torch.isneginf(got["lse"]).all() and torch.isneginf(got["logprob"]).all()
