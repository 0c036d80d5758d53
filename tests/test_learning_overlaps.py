"""The gated experts', the head's and the clipping calls refuse, on the host and before anything is launched, tensors of which one that is written lies on another at
any offset: outputs, states and workspaces.  What is only read may lie on each other."""
import ctypes as C

import pytest

import paper_2605_11537_amd as moe

INV = -1


@pytest.fixture(scope="module")
def at():
    """at(i): 16 KB apart."""
    b = (C.c_char * (32 << 14))()
    first = (C.addressof(b) + 255) & ~255
    return lambda i, n=0, keep=b: C.c_void_p(first + (i + 2 << 14) + n)


def test_clip(at):
    L = moe.lib()

    def call(tensors, outs, counts, norm, ws):
        k = len(tensors)
        return L.moe_clip_gradients((C.c_void_p * k)(*[t.value for t in tensors]), (C.c_void_p * k)(*[t.value for t in outs]), (C.c_longlong * k)(*counts),
                                    (C.c_int * k)(*([0] * k)), k, 1.0, norm, ws, 1 << 14, None)

    assert L.moe_clip_gradients_workspace_bytes(2) == 1 << 14
    a, b, n, w = at(0), at(1), at(2), at(3)
    for norm in (a, at(0, 4), at(0, 396), b, at(1, 396), w, at(3, 64), at(4, -4)):
        assert call([a], [b], [100], norm, w) == INV, "norm"
        assert b"overlaps" in L.moe_last_error()
    assert call([a], [a], [100], at(0, 40), w) == INV and call([a, b], [a, b], [100, 100], at(1, 8), w) == INV
    for ws in (a, b, n, at(0, 384), at(1, -1024), at(0, -(1 << 14) + 16), at(2, -(1 << 14) + 16)):
        assert call([a], [b], [100], n, ws) == INV, "workspace"
    assert call([a], [b], [100], at(2, 2), w) == INV                                # off its element


def refused(call, arguments, written):
    """Every written tensor on every other one: at its first byte, inside it, from in front of it into it."""
    for w in written:
        for o in arguments:
            if o == w:
                continue
            for by in (0, 16, 48, -16, -48):
                moved = C.c_void_p(arguments[o].value + by)
                assert call(**{w: moved}) == INV, (w, o, by)
                assert b"alias" in moe.lib().moe_last_error(), (w, o, by)


def test_gated(at):
    L = moe.lib()
    a = dict(x=at(0), t=at(1), g=at(2), u=at(3), w=at(4), y=at(5), ws=at(6), s=at(8))

    def call(states=False, R=4, E=15, d=8, F=8, dtype=0, size=1 << 14, **over):
        v = dict(a, **over)
        return L.moe_gated_ffn(v["x"], v["t"], v["g"], v["u"], v["w"], R, E, d, F, dtype, 0, v["y"], v["s"] if states else None, None if states else v["ws"],
                               0 if states else size, None)

    read = {k: a[k] for k in ("x", "t", "g", "u", "w")}
    refused(call, dict(read, y=a["y"], ws=a["ws"]), ("y", "ws"))
    refused(lambda **k: call(states=True, **k), dict(read, y=a["y"], s=a["s"]), ("y", "s"))


def test_gated_backward(at):
    L = moe.lib()
    a = dict(dy=at(0), x=at(1), t=at(2), g=at(3), u=at(4), w=at(5), s=at(6), dx=at(8), dg=at(9), du=at(10), dw=at(11), ws=at(12))

    def call(**over):
        v = dict(a, **over)
        return L.moe_gated_ffn_backward(v["dy"], v["x"], v["t"], v["g"], v["u"], v["w"], v["s"], 4, 15, 8, 8, 0, 0, v["dx"], v["dg"], v["du"], v["dw"], v["ws"],
                                        1 << 14, None)

    refused(call, a, ("dx", "dg", "du", "dw", "ws"))


def test_head(at):
    L = moe.lib()
    a = dict(h=at(0), w=at(1), b=at(2), t=at(3), lp=at(4), lse=at(5), ws=at(6))

    def call(**over):
        v = dict(a, **over)
        return L.moe_head_logprobs(v["h"], v["w"], v["b"], v["t"], 16, 8, 16, 0, v["lp"], v["lse"], v["ws"], 1 << 14, None)

    refused(call, a, ("lp", "lse", "ws"))


def test_head_backward(at):
    L = moe.lib()
    a = dict(h=at(0), w=at(1), b=at(2), t=at(3), lse=at(4), g=at(5), dh=at(6), dw=at(7), db=at(8), ws=at(9))

    def call(N=16, **over):
        v = dict(a, **over)
        return L.moe_head_logprobs_backward(v["h"], v["w"], v["b"], v["t"], v["lse"], v["g"], N, 8, 16, 0, v["dh"], v["dw"], v["db"], v["ws"], 8 << 14, None)

    refused(call, a, ("dh", "dw", "db", "ws"))
    for k in ("dw", "db"):                                           # sums over nothing are written too
        assert call(N=0, **{k: C.c_void_p(a["w"].value + 16)}) == INV
