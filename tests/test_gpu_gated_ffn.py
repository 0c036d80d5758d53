"""moe_gated_ffn and its gradient against oracle/learning.py in float64, expert by expert, within the bounds that it carries along: binary32 products and
sums, one rounding of h, dg and du, one of the result."""
import numpy as np
import pytest
import torch

from oracle import learning as ol

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
ACT = {"silu": 0, "gelu": 1, "relu": 2}


def f64(t):
    return t.double().cpu().numpy()


def near(got, want, what):
    g = f64(got)
    assert g.shape == want.value.shape, what
    over = np.abs(g - want.value) > want.off + 1e-37
    assert not over.any(), (what, int(over.sum()), float(np.abs(g - want.value).max()), float(want.off.max()))


def inputs(dtype, counts, R, d, F, seed, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    E = len(counts)
    n = lambda *s, std: (torch.randn(*s, generator=g, device="cuda") * std).to(DT[dtype])
    s = dict(x=n(R, d, std=spread), w=(n(E, d, F, std=d ** -0.5), n(E, d, F, std=d ** -0.5), n(E, F, d, std=F ** -0.5)), dy=n(R, d, std=0.1))
    s["first"] = np.concatenate([[0], np.cumsum(counts)]).tolist()
    s["offset"] = torch.tensor(s["first"], dtype=torch.int32, device="cuda")
    return s


def check(s, dtype, act, y, grads, experts=None):
    for e in range(len(s["first"]) - 1) if experts is None else experts:
        lo, hi = s["first"][e], s["first"][e + 1]
        want = ol.gated_ffn(f64(s["x"][lo:hi]), *(f64(w[e]) for w in s["w"]), act, HALF[dtype], f64(s["dy"][lo:hi]))
        near(y[lo:hi], want["y"], (e, "y"))
        near(grads["dx"][lo:hi], want["dx"], (e, "dx"))
        for k in ("dw_gate", "dw_up", "dw_down"):
            near(grads[k][e], want[k], (e, k))


# rows of each expert, rows behind the last, d, F: one row, none, one more than a tile, experts without rows between others, tiles of every height
CASES = [
    ([1], 0, 8, 8), ([1], 0, 72, 136), ([0, 1, 0], 2, 16, 24), ([3, 0, 5, 1], 1, 64, 64), ([63, 64, 65], 0, 72, 40), ([255], 0, 136, 264), ([257, 200], 3, 128, 256),
    ([100, 0, 0, 513], 5, 264, 200), ([16, 17, 15, 9, 8, 7], 0, 256, 512), ([2] * 40, 7, 48, 72), ([0, 0], 4, 16, 16), ([300, 1, 129, 33], 0, 520, 72), ([5, 120], 0, 1032, 24),
    ([1, 0, 3] * 300, 2, 24, 40),
]


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,behind,d,F", CASES)
def test_layer_and_gradient(counts, behind, d, F, dtype, act):
    import paper_2605_11537_amd as moe
    K, R = sum(counts), sum(counts) + behind
    s = inputs(dtype, counts, R, d, F, K + d + F)
    s["x"][K:], s["dy"][K:] = float("nan"), float("nan")             # not read
    y, states = moe.moe_gated_ffn(s["x"], *s["w"], s["offset"], ACT[act], want_states=True)
    plain, none = moe.moe_gated_ffn(s["x"], *s["w"], s["offset"], ACT[act])
    assert none is None and torch.equal(plain, y)
    grads = moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, s["offset"], ACT[act])
    check(s, dtype, act, y, grads)
    assert not y[K:].any() and not grads["dx"][K:].any()
    # rows behind the last are left as they were, every weight's gradient is written, a part of them alone gives the same bits
    out = dict(dx=torch.full_like(s["x"], 7.0), dw_gate=None, dw_up=None, dw_down=torch.full_like(s["w"][2], 7.0))
    moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, s["offset"], ACT[act], out=out)
    assert torch.equal(out["dx"][:K], grads["dx"][:K]) and (out["dx"][K:] == 7).all() and torch.equal(out["dw_down"], grads["dw_down"])
    seven = torch.full_like(y, 7.0)
    moe.moe_gated_ffn(s["x"], *s["w"], s["offset"], ACT[act], out=seven)
    assert torch.equal(seven[:K], y[:K]) and (seven[K:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,d,F", [(1, 768, 2048), (2, 64, 8), (33, 200, 104), (130, 256, 512), (600, 136, 72)])
def test_one_block(R, d, F, dtype):
    """Without a table all rows are one expert's; E = 1 with a table gives the same bits."""
    import paper_2605_11537_amd as moe
    s = inputs(dtype, [R], R, d, F, R + d)
    y, states = moe.moe_gated_ffn(s["x"], *s["w"], want_states=True)
    grads = moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states)
    check(s, dtype, "silu", y, grads)
    assert torch.equal(y, moe.moe_gated_ffn(s["x"], *s["w"], s["offset"])[0])


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,d,F", [([1, 2, 0, 1, 3], 200, 3176), ([1, 2, 0, 1, 3], 3176, 72), ([16], 264, 8200), ([1, 0, 1], 4104, 136)])
def test_few_tiles_of_a_long_sum(counts, d, F, dtype, act):
    """Tiles whose sum the wavefronts share, several to a workgroup; parts of the sum with one stage, with many, with none."""
    import paper_2605_11537_amd as moe
    K = sum(counts)
    s = inputs(dtype, counts, K + 2, d, F, K + d + F)
    s["x"][K:], s["dy"][K:] = float("nan"), float("nan")
    y, states = moe.moe_gated_ffn(s["x"], *s["w"], s["offset"], ACT[act], want_states=True)
    grads = moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, s["offset"], ACT[act])
    check(s, dtype, act, y, grads)
    for _ in range(2):
        again = moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, s["offset"], ACT[act])
        assert torch.equal(moe.moe_gated_ffn(s["x"], *s["w"], s["offset"], ACT[act])[0], y) and all(torch.equal(again[k], grads[k]) for k in grads)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_and_special_values(dtype):
    """Gates far on either side, and a NaN and an infinity in one row, which stay in that row (and in the gradients of its expert's weights)."""
    import paper_2605_11537_amd as moe
    s = inputs(dtype, [40, 30], 70, 64, 96, 5, spread=12.0)
    for act in ACT:
        y, states = moe.moe_gated_ffn(s["x"], *s["w"], s["offset"], ACT[act], want_states=True)
        check(s, dtype, act, y, moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, s["offset"], ACT[act]))
        bad = s["x"].clone()
        bad[3, 5], bad[60, 1] = float("nan"), float("inf")
        z, st = moe.moe_gated_ffn(bad, *s["w"], s["offset"], ACT[act], want_states=True)
        rows = [i for i in range(70) if i not in (3, 60)]
        assert torch.equal(z[rows], y[rows]) and torch.isnan(z[3]).all() and not torch.isfinite(z[60]).any()
        dx = moe.moe_gated_ffn_backward(s["dy"], bad, *s["w"], st, s["offset"], ACT[act])["dx"]
        assert torch.isfinite(dx[rows]).all() and torch.isnan(dx[3]).all()


def test_a_table_out_of_order():
    """Entries past the rows, negative or going back are taken for the nearest that are not: nothing outside the tensors is touched."""
    import paper_2605_11537_amd as moe
    s = inputs("bf16", [20, 30, 14], 64, 64, 64, 6)
    good, _ = moe.moe_gated_ffn(s["x"], *s["w"], s["offset"])
    for table, rows in (([0, 20, 50, 1000], 64), ([-5, 20, 50, 64], 64), ([0, 20, 10, 10], 20)):
        y, _ = moe.moe_gated_ffn(s["x"], *s["w"], torch.tensor(table, dtype=torch.int32, device="cuda"))
        assert torch.equal(y[:20], good[:20])
        if rows == 64:
            assert torch.equal(y, good)


def test_a_table_that_names_rows_twice():
    """Groups that would share rows: the later ones have what is left, forward and backward (the states hold each row once)."""
    import paper_2605_11537_amd as moe
    s = inputs("bf16", [64] * 5, 64, 64, 64, 8)
    for table, same in (([0, 64, 0, 64, 0, 64], [0, 64, 64, 64, 64, 64]), ([0, 40, 7, 50, -3, 90], [0, 40, 40, 50, 50, 64]), ([70, 5, 3, 2, 1, 0], [64] * 6)):
        got = []
        for t in (table, same):
            t = torch.tensor(t, dtype=torch.int32, device="cuda")
            y, states = moe.moe_gated_ffn(s["x"], *s["w"], t, want_states=True)
            got.append([y] + list(moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, t).values()))
        assert all(torch.equal(a, b) for a, b in zip(*got))


def test_no_rows():
    import paper_2605_11537_amd as moe
    for counts in ([0], [0, 0, 0]):
        s = inputs("bf16", counts, 0, 64, 96, 9)
        y, states = moe.moe_gated_ffn(s["x"], *s["w"], s["offset"], want_states=True)
        grads = moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, s["offset"])
        assert y.shape == (0, 64) and grads["dx"].shape == (0, 64) and not any(grads[k].any() for k in ("dw_gate", "dw_up", "dw_down"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_calls_give_equal_bits(dtype):
    import paper_2605_11537_amd as moe
    s = inputs(dtype, [500, 3, 0, 140], 650, 136, 392, 7)
    runs = []
    for _ in range(3):
        y, states = moe.moe_gated_ffn(s["x"], *s["w"], s["offset"], want_states=True)
        runs.append([y] + list(moe.moe_gated_ffn_backward(s["dy"], s["x"], *s["w"], states, s["offset"]).values()))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))
