"""Arguments that the gated experts', the head's and the clipping calls refuse on the host, before anything is launched, empty calls that they take, and
the sizes that their queries give."""
import ctypes as C

import pytest

import paper_2605_11537_amd as moe

INV, UNS, WS = -1, -2, -3


@pytest.fixture(scope="module")
def buf():
    b = (C.c_char * 16384)()
    at = (C.addressof(b) + 15) & ~15
    return [C.c_void_p(at + 512 * i) for i in range(20)] + [b]


def off(p, n=8):
    return C.c_void_p(p.value + n)


def test_gated(buf):
    x, t, g, u, w, y, s, ws = buf[:8]
    L = moe.lib()

    def call(x=x, t=t, g=g, u=u, w=w, R=4, E=2, d=8, F=8, dtype=1, act=0, y=y, s=None, ws=ws, size=1 << 20):
        return L.moe_gated_ffn(x, t, g, u, w, R, E, d, F, dtype, act, y, s, ws, size, None)

    assert call(R=-1) == INV and call(E=0) == INV and call(d=0) == INV and call(F=-8) == INV
    assert call(d=12) == INV and call(F=4) == INV and call(dtype=2) == INV and call(act=3) == INV and call(act=-1) == INV
    assert call(E=1025) == UNS and call(d=1 << 21) == UNS and call(F=1 << 20) == UNS and call(R=2 ** 31 - 1, E=1024, d=1 << 20, F=1 << 19) == UNS
    for k in ("x", "t", "g", "u", "w", "y"):
        assert call(**{k: None}) == INV, k
    for k, v in dict(x=x, g=g, u=u, w=w, y=y, s=s).items():
        assert call(**{k: off(v)}) == INV, k
    assert call(y=x) == INV and call(y=g) == INV and call(s=y) == INV and call(s=x) == INV
    assert call(ws=None) == WS and call(size=8) == WS and call(ws=off(ws)) == WS
    assert call(R=0, x=None, t=None, y=None, ws=None, size=0) == 0                  # no rows


def test_gated_backward(buf):
    dy, x, t, g, u, w, s, dx, dg, du, dw, ws = buf[:12]
    L = moe.lib()

    def call(dy=dy, x=x, t=t, g=g, u=u, w=w, s=s, R=4, E=2, d=8, F=8, dtype=1, act=0, dx=dx, dg=dg, du=du, dw=dw, ws=ws, size=1 << 20):
        return L.moe_gated_ffn_backward(dy, x, t, g, u, w, s, R, E, d, F, dtype, act, dx, dg, du, dw, ws, size, None)

    assert call(R=-1) == INV and call(E=0) == INV and call(d=4) == INV and call(dtype=7) == INV and call(act=9) == INV and call(E=1025) == UNS
    for k in ("dy", "x", "t", "g", "u", "w", "s"):
        assert call(**{k: None}) == INV, k
    assert call(dg=None) == INV and call(du=None) == INV                            # the pair comes together
    for k, v in dict(dy=dy, x=x, g=g, u=u, w=w, s=s, dx=dx, dg=dg, du=du, dw=dw).items():
        assert call(**{k: off(v)}) == INV, k
    for a in (dy, x, g, u, w, s, dg, du, dw):
        assert call(dx=a) == INV
    assert call(dw=w) == INV and call(dg=du) == INV and call(du=x) == INV
    assert call(ws=None) == WS and call(size=16) == WS and call(ws=off(ws)) == WS


def test_head(buf):
    h, w, b, t, lp, lse, ws = buf[:7]
    L = moe.lib()

    def call(h=h, w=w, b=b, t=t, N=4, d=8, V=5, dtype=1, lp=lp, lse=lse, ws=ws, size=1 << 20):
        return L.moe_head_logprobs(h, w, b, t, N, d, V, dtype, lp, lse, ws, size, None)

    assert call(N=-1) == INV and call(d=0) == INV and call(V=0) == INV and call(d=12) == INV and call(dtype=3) == INV
    assert call(d=1 << 21) == UNS and call(V=(1 << 24) + 1) == UNS and call(N=(1 << 24) + 1) == UNS
    assert call(N=1 << 24, V=1 << 24) == UNS and call(d=1 << 20, V=1 << 24) == UNS and call(d=1 << 20, N=1 << 24) == UNS
    for k in ("h", "w", "t", "lp", "lse"):
        assert call(**{k: None}) == INV, k
    assert call(h=off(h)) == INV and call(w=off(w)) == INV and call(lse=lp) == INV
    assert call(ws=None) == WS and call(size=8) == WS and call(ws=off(ws)) == WS
    assert call(N=0, h=None, t=None, lp=None, lse=None, ws=None, size=0) == 0


def test_head_backward(buf):
    h, w, b, t, lse, g, dh, dw, db, ws = buf[:10]
    L = moe.lib()

    def call(h=h, w=w, b=b, t=t, lse=lse, g=g, N=4, d=8, V=5, dtype=1, dh=dh, dw=dw, db=db, ws=ws, size=1 << 30):
        return L.moe_head_logprobs_backward(h, w, b, t, lse, g, N, d, V, dtype, dh, dw, db, ws, size, None)

    assert call(N=-1) == INV and call(d=9) == INV and call(V=0) == INV and call(dtype=3) == INV and call(V=1 << 25) == UNS
    for k in ("h", "w", "t", "lse", "g"):
        assert call(**{k: None}) == INV, k
    for k, v in dict(h=h, w=w, dh=dh, dw=dw).items():
        assert call(**{k: off(v)}) == INV, k
    assert call(dh=h) == INV and call(dh=w) == INV and call(dw=h) == INV and call(dw=w) == INV and call(dh=dw) == INV and call(db=b) == INV and call(db=lse) == INV
    assert call(ws=None) == WS and call(size=256) == WS and call(ws=off(ws)) == WS
    assert call(N=0, h=None, t=None, lse=None, g=None, dh=None, dw=None, db=None, ws=None, size=0) == 0


def test_clip(buf):
    a, b, norm, ws = buf[:4]
    L = moe.lib()

    def call(tensors, outs, counts, dtypes=None, n=None, most=1.0, norm=norm, ws=ws, size=1 << 20):
        k = len(tensors)
        return L.moe_clip_gradients((C.c_void_p * max(k, 1))(*[t.value if t else None for t in tensors]),
                                    (C.c_void_p * max(k, 1))(*[t.value if t else None for t in outs]), (C.c_longlong * max(k, 1))(*counts),
                                    (C.c_int * max(k, 1))(*(dtypes or [0] * k)), k if n is None else n, most, norm, ws, size, None)

    assert call([a], [b], [4], n=-1) == INV and call([a], [b], [4], n=5000) == UNS and call([a], [b], [-1]) == INV and call([a], [b], [1 << 45]) == INV
    assert call([a], [b], [4], dtypes=[2]) == INV
    assert call([a], [b], [4], most=0.0) == INV and call([a], [b], [4], most=-1.0) == INV and call([a], [b], [4], most=float("nan")) == INV
    assert call([a], [b], [4], norm=None) == INV and call([None], [b], [4]) == INV and call([a], [None], [4]) == INV
    assert call([off(a, 2)], [b], [4]) == INV and call([off(a, 1)], [b], [4], dtypes=[1]) == INV
    assert call([a], [b], [4], ws=None) == WS and call([a], [b], [4], size=8) == WS
    # what is written lies apart: named twice, on another gradient, half on its own
    assert call([a, a], [a, a], [4, 4]) == INV and call([a, b], [b, a], [4, 4]) == INV and call([a], [off(a, 4)], [4]) == INV
    assert call([a, off(a, 16)], [a, off(a, 16)], [5, 4]) == INV
    assert b"named twice" in L.moe_last_error()


def test_sizes():
    L = moe.lib()
    for q, args in (("moe_gated_ffn_states_bytes", (4, 2, 8, 1)), ("moe_gated_ffn_workspace_bytes", (4, 2, 8, 8, 1)),
                    ("moe_gated_ffn_backward_workspace_bytes", (4, 2, 8, 8, 1)), ("moe_head_logprobs_workspace_bytes", (4, 8, 5, 1)),
                    ("moe_head_logprobs_backward_workspace_bytes", (4, 8, 5, 1))):
        f = getattr(L, q)
        assert f(*args) > 0
        for i in range(len(args) - 1):
            assert f(*[0 if j == i else v for j, v in enumerate(args)]) == 0 or q == "moe_head_logprobs_workspace_bytes", (q, i)
            assert f(*[-3 if j == i else v for j, v in enumerate(args)]) == 0 or q == "moe_head_logprobs_workspace_bytes", (q, i)
    # past 32 bits
    assert L.moe_gated_ffn_states_bytes(1 << 20, 8, 1 << 13, 1) >= (1 << 33) * 10
    assert L.moe_head_logprobs_backward_workspace_bytes(1 << 16, 1024, 1 << 17, 1) < 6 << 30        # the logits would be 17 GB
    assert L.moe_clip_gradients_workspace_bytes(0) > 0
