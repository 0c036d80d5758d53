"""Arguments that the training and scoring calls refuse on the host, before anything is launched, and empty batches that they take."""
import ctypes as C

import pytest
import torch

import paper_2605_11537_amd as moe

INV, UNS, WS = -1, -2, -3


@pytest.fixture(scope="module")
def buf():
    b = (C.c_char * 8192)()
    at = (C.addressof(b) + 15) & ~15
    return [C.c_void_p(at + 512 * i) for i in range(15)] + [b]


def test_combine_backward(buf):
    p, q, i, w, o, dw, dx = buf[:7]
    f = moe.lib().moe_combine_topk_backward
    assert f(p, q, i, w, -1, 1, 8, 0, 0, o, dw, dx, None) == INV                    # T
    assert f(p, q, i, w, 4, 0, 8, 0, 0, o, dw, dx, None) == INV                     # k
    assert f(p, q, i, w, 4, 9, 8, 0, 0, o, dw, dx, None) == INV
    assert f(p, q, i, w, 4, 1, 6, 0, 0, o, dw, dx, None) == INV                     # row bytes
    assert f(p, q, i, w, 1 << 30, 3, 8, 0, 0, o, dw, dx, None) == INV               # more rows than an int counts
    assert f(p, q, i, w, 4, 1, 8, 2, 0, o, dw, dx, None) == INV                     # dtype
    assert f(p, q, i, w, 4, 1, 8, 0, 2, o, dw, dx, None) == INV                     # residual
    assert f(None, q, i, w, 4, 1, 8, 0, 0, o, dw, dx, None) == INV
    assert f(p, None, i, w, 4, 1, 8, 0, 0, o, dw, dx, None) == INV                  # dweight wants y_perm
    assert f(p, q, i, w, 4, 1, 8, 0, 0, p, dw, dx, None) == INV                     # aliases
    assert f(p, q, i, w, 4, 1, 8, 0, 0, o, dw, p, None) == INV
    assert f(p, q, i, w, 4, 1, 8, 0, 0, o, dw, o, None) == INV
    assert f(C.c_void_p(p.value + 4), q, i, w, 4, 1, 8, 0, 0, o, dw, dx, None) == INV
    assert b"misaligned" in moe.lib().moe_last_error()
    assert f(None, None, None, None, 0, 1, 8, 0, 0, None, None, None, None) == 0    # no tokens


def test_dispatch_backward(buf):
    p, i, a, o = buf[:4]
    f = moe.lib().moe_dispatch_topk_backward
    assert f(p, i, a, -1, 1, 8, 0, o, None) == INV
    assert f(p, i, a, 4, 9, 8, 0, o, None) == INV
    assert f(p, i, a, 4, 1, 4, 1, o, None) == INV                                   # row bytes
    assert f(p, None, a, 4, 1, 8, 0, o, None) == INV
    assert f(p, i, a, 4, 1, 8, 0, p, None) == INV                                   # alias
    assert f(p, i, C.c_void_p(a.value + 8), 4, 1, 8, 0, o, None) == INV
    assert f(None, None, None, 0, 1, 8, 0, None, None) == 0


def test_route_backward(buf):
    p, i, w, o = buf[:4]
    f = moe.lib().moe_route_topk_backward
    assert f(p, i, w, -1, 8, 1, 0, o, None) == INV
    assert f(p, i, w, 4, 8, 9, 0, o, None) == INV
    assert f(p, i, w, 4, 2, 3, 0, o, None) == INV                                   # k > E
    assert f(p, i, w, 4, 8, 1, 2, o, None) == INV
    assert f(p, i, w, 4, 1025, 1, 0, o, None) == UNS
    assert f(p, i, None, 4, 8, 1, 0, o, None) == INV
    assert f(p, i, w, 4, 8, 1, 0, p, None) == INV                                   # alias
    assert f(None, None, None, 0, 8, 1, 0, None, None) == 0


def test_scan(buf):
    u, x, b, h, c, s, ws = buf[:7]
    L = moe.lib()
    f = L.sru_scan

    def call(u=u, x=x, B=2, T=4, H=8, n=3, dtype=0, h=h, ws=ws, size=8192):
        return f(u, x, b, b, c, None, B, T, H, n, dtype, h, c, s, ws, size, None)

    assert call(B=-1) == INV and call(T=-1) == INV and call(H=0) == INV and call(dtype=5) == INV and call(n=2) == INV and call(n=5) == INV
    assert call(n=4) == INV                                                         # x beside a fourth block
    assert call(u=None) == INV and call(x=None) == INV and call(h=None) == INV
    assert call(h=u) == INV and call(h=x) == INV
    assert call(u=C.c_void_p(u.value + 8)) == INV
    assert call(B=1 << 30, H=1 << 20) == UNS and call(H=(1 << 22) + 1) == UNS
    assert call(B=0, u=None, x=x, h=None) == 0
    need = L.sru_scan_workspace_bytes(1, 16384, 128, 1)
    if need:
        assert call(B=1, T=16384, H=128, dtype=1, ws=None, size=0) == WS
        assert call(B=1, T=16384, H=128, dtype=1, size=need - 1) == WS
    assert L.sru_scan_states_bytes(2, 4, 8) >= 2 * 8 * 4 and L.sru_scan_states_bytes(0, 4, 8) == 0 and L.sru_scan_states_bytes(-1, 4, 8) == 0


def test_scan_backward(buf):
    dh, u, x, b, s, du, dx, db, dc, ws = buf[:10]
    L = moe.lib()
    need = L.sru_scan_backward_workspace_bytes(2, 4, 8, 0)

    def call(dh=dh, u=u, x=x, s=s, du=du, dx=dx, B=2, T=4, H=8, n=3, dtype=0, ws=ws, size=max(need, 512)):
        return L.sru_scan_backward(dh, None, u, x, b, b, s, None, B, T, H, n, dtype, du, dx, db, db, dc, ws, size, None)

    assert call(B=-1) == INV and call(T=-1) == INV and call(H=-3) == INV and call(dtype=-1) == INV and call(n=6) == INV
    assert call(n=4) == INV and call(n=4, x=None) == INV                            # x, then dx beside a fourth block
    assert call(dh=None) == INV and call(u=None) == INV and call(s=None) == INV and call(du=None) == INV and call(dx=None) == INV
    assert call(du=u) == INV and call(dx=x) == INV and call(du=dh) == INV and call(dx=du) == INV
    assert call(s=C.c_void_p(s.value + 8)) == INV
    assert call(ws=None, size=0) == WS and call(size=need - 1) == WS
    assert b"workspace" in L.moe_last_error()


def test_token_logprobs(buf):
    x, t, a, b, c, i, p, ws = buf[:8]
    L = moe.lib()

    def call(x=x, stride=8, N=2, V=8, dtype=0, k=2, a=a, i=i, ws=ws, size=0):
        return L.moe_token_logprobs(x, stride, t, N, V, dtype, k, a, b, c, i, p, ws, size, None)

    assert call(N=-1) == INV and call(V=0) == INV and call(stride=7) == INV and call(dtype=2) == INV
    assert call(k=-1) == INV and call(k=9) == INV and call(V=1, k=2) == INV
    assert call(x=None) == INV and call(a=None) == INV and call(i=None) == INV
    assert call(N=0, x=None, a=None, i=None) == 0
    assert call(V=(1 << 21) + 1, stride=1 << 22) == UNS and call(N=(1 << 31) - 1, V=2000, stride=2000) == UNS
    assert L.moe_token_logprobs_workspace_bytes(4, (1 << 21) + 1, 2, 1) == 0 and L.moe_token_logprobs_workspace_bytes(4, 1 << 21, 2, 7) == 0
    need = L.moe_token_logprobs_workspace_bytes(1, 1 << 18, 8, 1)
    if need:
        assert call(N=1, V=1 << 18, stride=1 << 18, dtype=1, k=8, size=need - 1) == WS
    f = L.moe_token_logprobs_backward
    assert f(x, 8, t, a, b, c, None, -1, 8, 0, p, 8, None) == INV
    assert f(x, 7, t, a, b, c, None, 2, 8, 0, p, 8, None) == INV
    assert f(x, 8, t, a, b, c, None, 2, 8, 0, p, 7, None) == INV
    assert f(x, 8, t, a, None, c, c, 2, 8, 0, p, 8, None) == INV                    # dentropy wants entropy
    assert f(x, 9, t, a, b, c, None, 2, 8, 0, x, 8, None) == INV                    # in place with another stride
    assert f(x, 8, t, a, b, c, None, 2, 8, 0, None, 8, None) == INV
    assert f(None, 8, None, None, None, None, None, 0, 8, 0, None, 8, None) == 0


def test_the_binding_takes_device_tensors_only():
    f, i = torch.zeros(4, 8), torch.zeros(1, 4, dtype=torch.int32)
    w = torch.zeros(1, 4)
    for call in (lambda: moe.moe_combine_topk_backward(f, f, i, w), lambda: moe.moe_dispatch_topk_backward(f, i),
                 lambda: moe.moe_route_topk_backward(f, i, w), lambda: moe.sru_scan(torch.zeros(1, 4, 24), torch.zeros(1, 4, 8)),
                 lambda: moe.moe_token_logprobs(f, i[0])):
        with pytest.raises(ValueError, match="device-resident"):
            call()
    with pytest.raises(ValueError, match="3 blocks of 8"):
        moe.sru_scan(torch.zeros(1, 4, 16), torch.zeros(1, 4, 8))
    with pytest.raises(TypeError):
        moe.sru_scan(torch.zeros(1, 4, 24, dtype=torch.float16), torch.zeros(1, 4, 8, dtype=torch.float16))
