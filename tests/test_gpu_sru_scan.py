"""sru_scan and sru_scan_backward against the float64 recurrence of oracle/training.py.

Tolerances: the bound that the oracle carries along the recurrence (32 half-units of binary32 for every gate, product and sum; 64 in
bfloat16, whose exponentials are a rounding coarser and whose states and outputs are blends), and for a bfloat16 result the half-unit of its own rounding, 2^-8 of the value.  A gate
does not go below e^-80 = 2e-35: 1e-33 absolute, for factors up to 50."""
import numpy as np
import pytest
import torch

from oracle import training as ot

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _f64(t):
    return None if t is None else t.double().cpu().numpy()


def _inputs(dtype, B, L, H, k, seed, lengths=None, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    n = lambda *s: torch.randn(*s, generator=g)
    c = dict(u=(n(B, L, k * H) * scale).to(dt), x=n(B, L, H).to(dt) if k == 3 else None, b_f=n(H) + 1.0, b_r=n(H), c0=n(B, H),
             lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32), dh=n(B, L, H).to(dt), dc_last=n(B, H))
    return {key: None if v is None else v.cuda() for key, v in c.items()}


def _near(got, want, bound, dtype, what):
    got = _f64(got)
    assert got.shape == want.shape, what
    tol = bound * 1.0001 + (2.0 ** -8 * 1.0001 * np.abs(want) if dtype == "bf16" else 2.0 ** -24 * np.abs(want)) + 1e-33
    over = np.abs(got - want) / tol
    assert np.isfinite(got).all(), what
    assert got.size == 0 or over.max() <= 1.0, f"{what}: {over.max():.2f} of the bound at {np.unravel_index(over.argmax(), over.shape)}"


def _check(dtype, c, what):
    import paper_2605_11537_amd as moe
    B, L, H = c["dh"].shape
    lengths = np.full(B, L) if c["lengths"] is None else c["lengths"].cpu().numpy()
    steps = 64 if dtype == "bf16" else 32
    zero = np.zeros(H)
    args = [_f64(c["u"]), _f64(c["x"]), zero if c["b_f"] is None else _f64(c["b_f"]), zero if c["b_r"] is None else _f64(c["b_r"]),
            np.zeros((B, H)) if c["c0"] is None else _f64(c["c0"]), lengths, steps, dtype == "bf16"]
    want = ot.sru_scan(*args)
    h, c_last, states = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"], c["lengths"], want_states=True)
    _near(h, want["h"], want["h_err"], dtype, f"{what} h")
    _near(c_last, want["c_last"], want["c_err"][:, -1], "f32", f"{what} c_last")
    h2, c2, none = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"], c["lengths"])
    assert none is None and torch.equal(h, h2) and torch.equal(c_last, c2), f"{what}: states change the outputs"
    g = moe.sru_scan_backward(c["dh"], c["u"], states, c["x"], c["b_f"], c["b_r"], c["dc_last"], c["lengths"])
    dc = np.zeros((B, H)) if c["dc_last"] is None else _f64(c["dc_last"])
    want, bound = ot.sru_scan_backward(_f64(c["dh"]), dc, *args)
    for key in ("du", "dx", "db_f", "db_r", "dc0"):
        if want[key] is None:
            assert g[key] is None
        else:
            _near(g[key], want[key], bound[key], dtype if key in ("du", "dx") else "f32", f"{what} {key}")
    again = moe.sru_scan_backward(c["dh"], c["u"], states, c["x"], c["b_f"], c["b_r"], c["dc_last"], c["lengths"])
    assert all(g[key] is None or torch.equal(g[key], again[key]) for key in g), f"{what}: two calls differ"
    for b, n in enumerate(lengths):                                  # behind the end: zero, whatever lies there
        assert (h[b, n:] == 0).all() and (g["du"][b, n:] == 0).all() and (g["dx"] is None or (g["dx"][b, n:] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,H,k", [
    (1, 1, 1, 3), (2, 1, 64, 4), (300, 1, 40, 3), (1, 2, 3, 4), (3, 15, 7, 3), (2, 16, 66, 4), (2, 17, 127, 3), (1, 31, 130, 4),
    (2, 100, 129, 3), (1, 127, 64, 4), (3, 128, 320, 3), (2, 129, 65, 4), (1, 511, 70, 3), (1, 1025, 33, 3), (1, 2049, 128, 4), (1, 5000, 5, 3),
])
def test_sizes(dtype, B, L, H, k):
    c = _inputs(dtype, B, L, H, k, 1000 + L + H)
    print(f"{dtype} B={B} L={L} H={H} k={k}", flush=True)
    _check(dtype, c, f"{dtype} {B}x{L}x{H} k={k}")


@pytest.mark.parametrize("dtype,lengths", [("f32", None), ("bf16", [70001, 32768, 35000])])
def test_very_long(dtype, lengths):
    """Beyond 32768 steps, where a sequence's pairs go through states at every 256th tile."""
    B, L, H = (1, 70001, 2) if lengths is None else (3, 70001, 1)
    _check(dtype, _inputs(dtype, B, L, H, 3, 6, lengths), f"{dtype} {L}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,lengths,L,H", [
    (3, [9, 0, 1, 5], 9, 34), (4, [0], 3, 8), (3, [16, 17, 15, 32], 32, 65), (4, [260, 0, 1, 128, 129, 255], 300, 66), (3, [1, 2300, 1111], 2300, 30),
])
def test_padded_batches(dtype, k, lengths, L, H):
    """Lengths from 0 on, some whole parts of the sequence empty; NaN behind the ends must not come through."""
    c = _inputs(dtype, len(lengths), L, H, k, 77 + L, lengths)
    for b, n in enumerate(lengths):
        for key in ("u", "x", "dh"):
            if c[key] is not None:
                c[key][b, n:] = float("nan")
    print(f"{dtype} k={k} lengths={lengths}", flush=True)
    clean = {key: torch.nan_to_num(v) if key in ("u", "x", "dh") and v is not None else v for key, v in c.items()}
    import paper_2605_11537_amd as moe
    _check(dtype, clean, f"{dtype} {lengths}")
    a = [moe.sru_scan(q["u"], q["x"], q["b_f"], q["b_r"], q["c0"], q["lengths"], want_states=True) for q in (c, clean)]
    assert torch.equal(a[0][0], a[1][0]) and torch.equal(a[0][1], a[1][1])
    g = [moe.sru_scan_backward(q["dh"], q["u"], s[2], q["x"], q["b_f"], q["b_r"], q["dc_last"], q["lengths"]) for q, s in zip((c, clean), a)]
    for key in g[0]:
        assert g[0][key] is None or torch.equal(g[0][key], g[1][key]), key


def test_lengths_are_taken_to_the_rows_there_are():
    import paper_2605_11537_amd as moe
    c = _inputs("f32", 3, 40, 24, 3, 5, [-7, 40, 1 << 30])
    d = dict(c, lengths=torch.tensor([0, 40, 40], dtype=torch.int32).cuda())
    a, b = (moe.sru_scan(q["u"], q["x"], q["b_f"], q["b_r"], q["c0"], q["lengths"], want_states=True) for q in (c, d))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    g = [moe.sru_scan_backward(q["dh"], q["u"], s[2], q["x"], q["b_f"], q["b_r"], q["dc_last"], q["lengths"]) for q, s in ((c, a), (d, b))]
    assert all(torch.equal(g[0][k], g[1][k]) for k in g[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_may_be_left_out(dtype):
    """Biases, states before and after, and their gradients."""
    import paper_2605_11537_amd as moe
    c = _inputs(dtype, 2, 37, 48, 4, 9)
    for key in ("b_f", "b_r", "c0", "dc_last"):
        c[key] = None
    _check(dtype, c, f"{dtype} bare")
    states = moe.sru_scan(c["u"], want_states=True)[2]
    full = moe.sru_scan_backward(c["dh"], c["u"], states)
    only = dict(du=torch.empty_like(c["u"]), dx=None, db_f=None, db_r=None, dc0=None)
    moe.sru_scan_backward(c["dh"], c["u"], states, out=only)
    assert torch.equal(full["du"], only["du"])
    some = dict(only, db_r=torch.empty(48, device="cuda"))
    moe.sru_scan_backward(c["dh"], c["u"], states, out=some)
    assert torch.equal(full["db_r"], some["db_r"])
    h, none, _ = moe.sru_scan(c["u"], out=(torch.empty(2, 37, 48, dtype=DT[dtype], device="cuda"), None, None))
    assert torch.equal(h, moe.sru_scan(c["u"])[0])


@pytest.mark.parametrize("value", [0.0, 40.0, -40.0, 300.0, -300.0, 3e38, -3e38])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_open_and_shut(dtype, value):
    """Pre-activations far beyond the exponential's range: a gate is exactly 0 or 1 there, nothing becomes infinite or NaN."""
    c = _inputs(dtype, 2, 20, 16, 3, 11)
    u = c["u"].view(2, 20, 3, 16)
    u[:, :, 1, :8] = value
    u[:, :, 2, 4:12] = value
    _check(dtype, c, f"{dtype} gates at {value}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_and_large_states(dtype):
    """tanh near zero keeps its relative accuracy, and far out its slope does not turn to noise."""
    c = _inputs(dtype, 2, 24, 64, 3, 12)
    scale = torch.logspace(-12, 2, 64, device="cuda")
    u = c["u"].view(2, 24, 3, 64)
    u[:, :, 0] *= scale.to(u.dtype)
    c["c0"] *= scale
    c["x"][:] = 0
    _check(dtype, c, dtype)


def test_nan_comes_through_from_where_it_is_on():
    import paper_2605_11537_amd as moe
    for block in range(3):
        c = _inputs("f32", 1, 40, 8, 3, 13)
        c["u"].view(1, 40, 3, 8)[0, 21, block, 3] = float("nan")
        h, c_last, _ = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"])
        bad = torch.isnan(h[0])
        assert bad[21, 3] and not bad[:21].any() and not bad[:, [0, 1, 2, 4, 5, 6, 7]].any()
        assert bool(bad[22:, 3].all()) == (block < 2) and bool(torch.isnan(c_last[0, 3])) == (block < 2)


@pytest.mark.parametrize("L", [0, 1, 5000])
def test_state_in_place_and_no_tokens(L):
    import paper_2605_11537_amd as moe
    c = _inputs("f32", 2, L, 96, 3, 14)
    h, c_last, states = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"], want_states=True)
    state = c["c0"].clone()
    h2 = torch.empty_like(h)
    moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], state, out=(h2, state, None))
    assert torch.equal(state, c_last) and torch.equal(h, h2)
    g = moe.sru_scan_backward(c["dh"], c["u"], states, c["x"], c["b_f"], c["b_r"], c["dc_last"])
    d = c["dc_last"].clone()
    g2 = moe.sru_scan_backward(c["dh"], c["u"], states, c["x"], c["b_f"], c["b_r"], d, out=dict(g, du=torch.empty_like(g["du"]),
                               dx=torch.empty_like(g["dx"]), db_f=torch.empty(96, device="cuda"), db_r=torch.empty(96, device="cuda"), dc0=d))
    for key in ("du", "dx", "db_f", "db_r"):
        assert torch.equal(g[key], g2[key]), key
    if L == 0:
        assert torch.equal(c_last, c["c0"]) and torch.equal(d, c["dc_last"]) and (g["db_f"] == 0).all() and (g["db_r"] == 0).all()


def test_no_sequences():
    import paper_2605_11537_amd as moe
    c = _inputs("f32", 0, 5, 96, 3, 14)
    h, c_last, states = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"], want_states=True)
    g = moe.sru_scan_backward(c["dh"], c["u"], states, c["x"], c["b_f"], c["b_r"], c["dc_last"])
    assert h.shape == (0, 5, 96) and (g["db_f"] == 0).all() and (g["db_r"] == 0).all()


def test_token_by_token_is_the_whole():
    """A sequence decoded one token a call, its state carried, against the sequence at once: the same recurrence, each within its bound."""
    import paper_2605_11537_amd as moe
    c = _inputs("f32", 3, 50, 64, 3, 15)
    want = ot.sru_scan(_f64(c["u"]), _f64(c["x"]), _f64(c["b_f"]), _f64(c["b_r"]), _f64(c["c0"]), [50] * 3)
    state, rows = c["c0"].clone(), []
    for t in range(50):
        h, _, _ = moe.sru_scan(c["u"][:, t:t + 1].contiguous(), c["x"][:, t:t + 1].contiguous(), c["b_f"], c["b_r"], state,
                               out=(torch.empty(3, 1, 64, device="cuda"), state, None))
        rows.append(h)
    _near(torch.cat(rows, 1), want["h"], want["h_err"], "f32", "h")
    _near(state, want["c_last"], want["c_err"][:, -1], "f32", "c")


def test_guards_around_the_outputs_stay():
    """Nothing is written beside the outputs, at sizes where tiles end inside."""
    import paper_2605_11537_amd as moe
    for dtype in ("f32", "bf16"):
        for B, L, H, k in ((1, 1, 1, 3), (2, 33, 65, 4), (1, 700, 130, 3)):
            c = _inputs(dtype, B, L, H, k, 16)

            def guarded(n, dt):
                n = int(n)
                t = torch.full((n + 128,), 7.0, dtype=dt, device="cuda")
                return t, t[64:64 + n]

            t, f32 = DT[dtype], torch.float32
            n_states = moe.lib().sru_scan_states_bytes(B, L, H) // 4
            made = {key: guarded(n, dt) for key, n, dt in (("h", B * L * H, t), ("c", B * H, f32), ("s", n_states, f32), ("du", B * L * k * H, t),
                    ("dx", B * L * H, t), ("db_f", H, f32), ("db_r", H, f32), ("dc0", B * H, f32),
                    ("ws", max(moe.lib().sru_scan_workspace_bytes(B, L, H, moe.MOE_F32 if t == f32 else moe.MOE_BF16),
                               moe.lib().sru_scan_backward_workspace_bytes(B, L, H, moe.MOE_F32 if t == f32 else moe.MOE_BF16)) // 4, f32))}
            v = {key: q[1] for key, q in made.items()}
            ws = v["ws"].view(torch.uint8)
            _, _, states = moe.sru_scan(c["u"], c["x"], c["b_f"], c["b_r"], c["c0"], ws=ws, out=(v["h"].view(B, L, H), v["c"].view(B, H), v["s"]))
            moe.sru_scan_backward(c["dh"], c["u"], states, c["x"], c["b_f"], c["b_r"], c["dc_last"], ws=ws,
                                  out=dict(du=v["du"].view(B, L, k * H), dx=v["dx"].view(B, L, H) if k == 3 else None, db_f=v["db_f"],
                                           db_r=v["db_r"], dc0=v["dc0"].view(B, H)))
            for key, (whole, inner) in made.items():
                assert (whole[:64] == 7).all() and (whole[64 + inner.numel():] == 7).all(), (dtype, B, L, H, key)
