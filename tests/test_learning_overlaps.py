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
