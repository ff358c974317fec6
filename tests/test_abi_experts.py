"""Argument validation of the operators around experts through the raw C ABI (no GPU: a non-zero status, or nothing to do, launches
nothing, so the addresses are made up)."""
import ctypes

import pytest

from paper_1802_04730_amd import tc355

OK, NULL, SHAPE, ALIAS, ALIGN, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 5, 7
F32, BF16, F16 = 0, 1, 2
A, B, C, D, E_, F_, G, H = (0x10000 * i for i in range(1, 9))
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    return tc355.lib()


def test_embed(L):
    call = lambda lut=A, idx=B, o=C, E=10, D=8, T=4, t=F32: L.tc_embed(lut, idx, o, E, D, T, 1.0, t, None)  # noqa: E731
    assert call(T=0) == call(T=0, idx=None, o=None) == OK
    assert call(lut=None) == call(idx=None) == call(o=None) == NULL
    assert call(E=0) == call(D=0) == call(T=-1) == call(t=3) == call(t=-1) == SHAPE
    assert call(o=A) == call(o=B) == ALIAS
    assert call(lut=A + 4) == call(idx=B + 8) == call(o=C + 2) == ALIGN
    assert call(E=BIG) == call(D=BIG) == call(T=BIG) == UNSUPPORTED


def test_embed_grad(L):
    call = lambda d=A, idx=B, g=C, E=10, D=8, T=4, add=0, t=BF16, gt=F32, ws=D_WS, n=1 << 20: L.tc_embed_grad(  # noqa: E731
        d, idx, g, E, D, T, 1.0, -1, add, t, gt, ws, n, None)
    assert call(T=0, add=1, d=None, idx=None, ws=None, n=0) == OK
    assert call(d=None) == call(idx=None) == call(g=None) == NULL
    assert call(E=0) == call(D=-1) == call(T=-1) == call(gt=F16) == call(t=9) == SHAPE
    assert call(t=F32, gt=BF16) == SHAPE
    assert call(g=A) == call(g=B) == call(ws=A) == call(ws=B) == call(ws=C) == ALIAS
    assert call(d=A + 2) == call(idx=B + 4) == call(g=C + 8) == ALIGN
    assert call(ws=None) == call(ws=D_WS + 8) == call(n=16) == WORKSPACE
    assert call(E=BIG) == call(D=BIG) == call(T=BIG) == UNSUPPORTED
    size = L.tc_embed_grad_workspace_bytes
    assert size(10, 8, 4) > 0 and size(10, 8, 0) == size(0, 8, 4) == size(10, -8, 4) == size(BIG, 8, 4) == size(10, BIG, 4) == size(10, 8, BIG) == 0
    assert size(10, 8, 4000) > size(10, 8, 4) and call(n=size(10, 8, 4) - 1) == WORKSPACE


D_WS = 0x100000


def test_route(L):
    def call(l=A, w=B, i=C, off=D, row=E_, place=F_, T=100, E=8, k=2, t=F32, ws=G, n=1 << 20):
        return L.tc_route(l, w, i, off, row, place, T, E, k, 0, t, ws, n, None)

    assert call(l=None) == call(w=None) == call(i=None) == call(off=None) == call(row=None) == call(place=None) == NULL
    assert call(E=0) == call(k=0) == call(k=9) == call(T=-1) == call(t=5) == SHAPE
    assert call(w=A) == call(place=E_) == call(ws=A) == call(ws=C) == call(off=C) == ALIAS
    assert call(l=A + 2) == call(w=B + 4) == call(row=E_ + 4) == ALIGN
    assert call(ws=None) == call(ws=G + 4) == call(n=8) == WORKSPACE
    assert call(E=1024) == call(E=500, k=65) == call(T=BIG) == UNSUPPORTED
    size = L.tc_route_workspace_bytes
    assert size(100, 8, 2) > 0 and size(1, 8, 2) == size(0, 8, 2) == size(100, 8, 9) == size(100, 1024, 2) == size(BIG, 8, 2) == 0
    assert call(n=size(100, 8, 2) - 1) == WORKSPACE

    grad = lambda l=A, i=B, w=C, d=D, T=4, E=8, k=2, t=F32: L.tc_route_grad(l, i, w, d, T, E, k, 0, t, None)  # noqa: E731
    assert grad(T=0) == grad(T=0, l=None, d=None) == OK
    assert grad(l=None) == grad(i=None) == grad(w=None) == grad(d=None) == NULL
    assert grad(k=9) == grad(E=0) == grad(t=7) == SHAPE
    assert grad(d=A) == grad(d=B) == grad(d=C) == ALIAS
    assert grad(l=A + 8) == grad(d=D + 2) == ALIGN
    assert grad(E=2000) == grad(T=BIG) == UNSUPPORTED


def test_expert_mm(L):
    def call(x=A, w=B, off=C, row=D, y=E_, T=4, R=6, E=3, N=8, K=8, t=BF16):
        return L.tc_expert_mm(x, w, off, row, y, T, R, E, N, K, 0, t, None)

    assert call(R=0) == call(R=0, x=None, y=None) == call(R=0, T=0, row=None) == OK
    assert call(x=None) == call(w=None) == call(off=None) == call(y=None) == NULL
    assert call(row=None) == call(E=0) == call(N=0) == call(K=0) == call(R=-1) == call(T=-1) == call(t=3) == SHAPE  # (without Row, T is R)
    assert call(y=A) == call(y=B) == call(y=C) == call(y=D) == ALIAS
    assert call(x=A + 2) == call(w=B + 4) == call(off=C + 4) == call(row=D + 8) == call(y=E_ + 8) == ALIGN
    assert call(T=BIG) == call(R=BIG) == call(E=BIG) == call(N=BIG) == call(K=BIG) == call(N=1 << 22) == UNSUPPORTED

    def grad_x(d=A, w=B, off=C, gate=D, x=E_, R=6, E=3, N=8, K=8, t=F16):
        return L.tc_expert_mm_grad_x(d, w, off, gate, x, R, E, N, K, t, None)

    assert grad_x(R=0) == grad_x(R=0, d=None, x=None, gate=None) == OK
    assert grad_x(d=None) == grad_x(w=None) == grad_x(off=None) == grad_x(x=None) == NULL
    assert grad_x(E=-1) == grad_x(N=0) == grad_x(K=0) == grad_x(R=-1) == grad_x(t=4) == SHAPE
    assert grad_x(x=A) == grad_x(x=B) == grad_x(x=C) == grad_x(x=D) == ALIAS
    assert grad_x(gate=D + 2) == grad_x(x=E_ + 8) == ALIGN
    assert grad_x(R=BIG) == grad_x(K=BIG) == UNSUPPORTED

    def grad_w(d=A, x=B, off=C, row=D, w=E_, T=4, R=6, E=3, N=8, K=8, add=0, t=BF16, gt=F32, ws=F_, n=64):
        return L.tc_expert_mm_grad_w(d, x, off, row, w, T, R, E, N, K, add, t, gt, ws, n, None)

    assert grad_w(R=0, add=1) == grad_w(R=0, add=1, d=None, x=None, ws=None, n=0) == OK
    assert grad_w(d=None) == grad_w(x=None) == grad_w(off=None) == grad_w(w=None) == NULL
    assert grad_w(row=None) == grad_w(gt=F16) == grad_w(t=F32, gt=BF16) == grad_w(E=0) == grad_w(R=-1) == SHAPE
    assert grad_w(w=A) == grad_w(w=B) == grad_w(w=C) == grad_w(w=D) == grad_w(ws=A) == grad_w(ws=E_) == grad_w(ws=C) == ALIAS
    assert grad_w(w=E_ + 4) == grad_w(ws=F_ + 4) == grad_w(row=D + 4) == ALIGN
    assert grad_w(N=BIG) == grad_w(E=BIG) == UNSUPPORTED
    size = L.tc_expert_mm_grad_w_workspace_bytes
    assert size(0, 3, 8, 8) == size(6, 0, 8, 8) == size(6, 3, BIG, 8) == size(BIG, 3, 8, 8) == 0


def test_expert_sum(L):
    call = lambda y=A, w=B, p=C, o=D, T=4, R=6, k=2, N=8, t=F32: L.tc_expert_sum(y, w, p, o, T, R, k, N, t, None)  # noqa: E731
    assert call(T=0) == call(T=0, y=None, w=None, p=None, o=None) == OK
    assert call(y=None) == call(p=None) == call(o=None) == NULL
    assert call(k=0) == call(N=0) == call(T=-1) == call(R=-1) == call(t=3) == SHAPE
    assert call(o=A) == call(o=B) == call(o=C) == ALIAS
    assert call(y=A + 2) == call(w=B + 4) == call(o=D + 8) == ALIGN
    assert call(T=BIG) == call(R=BIG) == call(N=BIG) == call(k=BIG) == UNSUPPORTED

    def grad(o=A, y=B, w=C, p=D, dy=E_, dw=F_, T=4, R=6, k=2, N=8, t=F32):
        return L.tc_expert_sum_grad(o, y, w, p, dy, dw, T, R, k, N, t, None)

    assert grad(T=0) == OK
    assert grad(o=None) == grad(y=None) == grad(w=None) == grad(p=None) == grad(dy=None) == grad(dw=None) == NULL
    assert grad(k=0) == grad(N=-1) == grad(t=8) == SHAPE
    assert grad(dy=A) == grad(dy=B) == grad(dw=C) == grad(dw=D) == grad(dw=E_) == ALIAS
    assert grad(o=A + 2) == grad(dy=E_ + 4) == grad(dw=F_ + 4) == ALIGN
    assert grad(T=BIG) == grad(N=BIG) == UNSUPPORTED


def test_nothing_is_thrown_at_extremes(L):
    """Extents at the ends of 64 bits, in every place, end in a status."""
    ends = [-(1 << 63), (1 << 63) - 1, 1 << 62, (1 << 31) - 1, 1 << 31]
    for v in ends:
        for name, n in (("tc_embed_grad_workspace_bytes", 3), ("tc_route_workspace_bytes", 3), ("tc_expert_mm_grad_w_workspace_bytes", 4)):
            for at in range(n):
                args = [4] * n
                args[at] = v
                getattr(L, name)(*args)
        for at in range(3):
            s = [4, 4, 4]
            s[at] = v if v < 0 or at != 2 else 1 << 62
            if s[at] > (1 << 31):
                assert L.tc_embed(A, B, C, *s, 1.0, F32, None) == UNSUPPORTED
    assert isinstance(ctypes.c_int(L.tc355_version()).value, int)


def test_an_empty_list_of_rows_may_be_null(L):
    """A step without routed rows: a list of no elements comes as NULL, as an array without elements does, whatever X holds."""
    for T in (0, 4):
        for row in (None, D):
            assert L.tc_expert_mm(A, B, C, row, None, T, 0, 3, 8, 8, 0, BF16, None) == OK
            assert L.tc_expert_mm_grad_w(None, A, C, row, E_, T, 0, 3, 8, 8, 1, BF16, F32, None, 0, None) == OK
    assert L.tc_expert_mm(A, B, C, None, E_, 4, 6, 3, 8, 8, 0, BF16, None) == SHAPE  # (with rows, T is R without a list)
    assert L.tc_expert_mm_grad_w(A, B, C, None, E_, 4, 6, 3, 8, 8, 1, BF16, F32, None, 0, None) == SHAPE


def test_the_router_wants_a_workspace_where_two_launches_are_faster(L):
    size = L.tc_route_workspace_bytes
    for E, k in ((8, 2), (64, 4), (128, 8), (1023, 64)):
        assert size(32, E, k) == 0 and size(33, E, k) > 0 and size(64, E, k) > 0
        grows = [size(T, E, k) for T in range(1, 5000)]
        assert grows == sorted(grows)


def test_a_workspace_for_more_tokens_serves_fewer(L):
    """A program that asks for its largest batch's bytes once is not refused a smaller one."""
    size = L.tc_embed_grad_workspace_bytes
    for E, D in ((100, 1), (50000, 333), (1 << 20, 4096)):
        T = sorted({x for n in (8, 32, 1000, 2048, 8192, 14336, 16384, 57344, 65536, 1 << 20) for x in range(n - 33, n + 34) if x > 0})
        sizes = [size(E, D, t) for t in T]
        assert sizes == sorted(sizes) and sizes[0] > 0
