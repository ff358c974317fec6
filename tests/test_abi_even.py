"""Argument validation of the operators around experts of even load through the raw C ABI (no GPU: a non-zero status, or nothing to do, launches
nothing, so the addresses are made up)."""
import pytest

from paper_1802_04730_amd import tc355

OK, NULL, SHAPE, ALIAS, ALIGN, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 5, 7
F32, BF16, F16 = 0, 1, 2
A, B, C, D, E_, F_, G, H, I, J = (0x10000 * i for i in range(1, 11))
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    return tc355.lib()


def test_layer_norm(L):
    call = lambda x=A, w=B, b=C, o=D, T=4, N=8, eps=1e-5, t=BF16, wt=F32: L.tc_layer_norm(x, w, b, o, T, N, eps, t, wt, None)  # noqa: E731
    assert call(T=0) == call(T=0, x=None, o=None) == OK
    assert call(x=None) == call(w=None) == call(o=None) == NULL
    assert call(T=-1) == call(N=0) == call(N=-3) == call(t=3) == call(t=-1) == call(wt=F16) == call(wt=7) == call(eps=-1e-9) == call(eps=float("nan")) == SHAPE
    assert call(t=F32, wt=BF16) == SHAPE
    assert call(o=A) == call(o=B) == call(o=C) == ALIAS
    assert call(x=A + 4) == call(w=B + 2) == call(b=C + 8) == call(o=D + 2) == ALIGN
    assert call(T=BIG) == call(N=BIG) == call(N=1 << 26) == UNSUPPORTED


def test_layer_norm_grad(L):
    call = lambda g=A, x=B, w=C, dx=D, dw=E_, db=F_, T=4, N=8, eps=1e-5, add=0, t=BF16, wt=F32, ws=G, n=1 << 20: L.tc_layer_norm_grad(  # noqa: E731
        g, x, w, dx, dw, db, T, N, eps, add, t, wt, ws, n, None)
    assert call(T=0, add=1) == call(T=0, dw=None, db=None) == call(T=0, add=1, g=None, x=None, dx=None, ws=None, n=0) == OK
    assert call(g=None) == call(x=None) == call(w=None) == call(dx=None) == call(dw=None) == NULL
    assert call(T=-1) == call(N=0) == call(t=3) == call(wt=F16) == call(eps=-1.0) == call(eps=float("nan")) == SHAPE
    assert call(dx=A) == call(dx=B) == call(dx=C) == call(dw=C) == call(dw=D) == call(db=E_) == call(db=A) == call(ws=A) == call(ws=D) == call(ws=E_) == call(ws=F_) == ALIAS
    assert call(g=A + 2) == call(x=B + 2) == call(w=C + 4) == call(dx=D + 8) == call(dw=E_ + 4) == call(db=F_ + 4) == ALIGN
    assert call(ws=None) == call(ws=G + 8) == call(n=64) == WORKSPACE
    assert call(T=BIG) == call(N=1 << 26) == UNSUPPORTED
    size = L.tc_layer_norm_grad_workspace_bytes
    assert size(0, 8) == size(4, 0) == size(-1, 8) == size(BIG, 8) == size(4, BIG) == 0
    for N in (1, 333, 4096, 20000):  # what serves more rows serves fewer
        sizes = [size(T, N) for T in (1, 2, 16, 17, 100, 511, 5000, 8192, 8193, 100000, 1 << 30)]
        assert sizes == sorted(sizes) and sizes[0] > 0


def test_route_balanced(L):
    call = lambda l=A, b=B, w=C, i=D, off=E_, row=F_, p=G, T=4, E=8, k=2, g=4, keep=2, t=BF16, ws=H, n=1 << 20: L.tc_route_balanced(  # noqa: E731
        l, b, w, i, off, row, p, T, E, k, g, keep, 1, 1, 1.0, t, ws, n, None)
    assert call(l=None) == call(w=None) == call(i=None) == call(off=None) == call(row=None) == call(p=None) == NULL
    assert call(T=-1) == call(E=0) == call(k=0) == call(k=9) == call(t=3) == call(g=0) == call(g=3) == call(g=9) == call(keep=0) == call(keep=5) == call(g=-4) == SHAPE
    assert call(w=A) == call(w=B) == call(i=C) == call(row=E_) == call(p=F_) == call(off=A) == call(ws=A) == call(ws=B) == call(ws=G) == ALIAS
    assert call(l=A + 2) == call(b=B + 4) == call(w=C + 4) == call(i=D + 4) == call(off=E_ + 4) == call(row=F_ + 4) == call(p=G + 4) == ALIGN
    assert call(E=1024) == call(E=520, k=65) == call(T=BIG) == call(T=1 << 28) == call(E=130, g=65) == UNSUPPORTED
    assert call(T=65, ws=None) == call(T=100, ws=H + 4) == call(T=100, n=8) == WORKSPACE
    size = L.tc_route_balanced_workspace_bytes
    assert size(32, 8, 2) == 0 and size(33, 8, 2) > 0 and size(-1, 8, 2) == size(40, 0, 1) == size(40, 8, 9) == size(40, 1024, 2) == size(BIG, 8, 2) == 0
    assert size(100, 8, 2) == L.tc_route_workspace_bytes(100, 8, 2)


def test_route_balanced_grad(L):
    call = lambda l=A, i=B, d=C, g=D, T=4, E=8, k=2, t=BF16: L.tc_route_balanced_grad(l, i, d, g, T, E, k, 1, 1, 1.0, t, None)  # noqa: E731
    assert call(T=0) == call(T=0, l=None, i=None, d=None, g=None) == OK
    assert call(l=None) == call(i=None) == call(d=None) == call(g=None) == NULL
    assert call(T=-1) == call(E=0) == call(k=0) == call(k=9) == call(t=3) == SHAPE
    assert call(g=A) == call(g=B) == call(g=C) == ALIAS
    assert call(l=A + 2) == call(i=B + 4) == call(d=C + 8) == call(g=D + 2) == ALIGN
    assert call(E=1024) == call(E=520, k=65) == call(T=BIG) == UNSUPPORTED


def test_quantize_rows(L):
    call = lambda x=A, q=B, s=C, R=4, K=8, t=BF16: L.tc_quantize_rows(x, q, s, R, K, t, None)  # noqa: E731
    assert call(R=0) == call(R=0, x=None, q=None, s=None) == OK
    assert call(x=None) == call(q=None) == call(s=None) == NULL
    assert call(R=-1) == call(K=0) == call(t=3) == SHAPE
    assert call(q=A) == call(s=A) == call(s=B) == ALIAS
    assert call(x=A + 2) == call(q=B + 8) == call(s=C + 1) == ALIGN
    assert call(R=BIG) == call(K=BIG) == UNSUPPORTED


def test_quantize_weights(L):
    call = lambda w=A, q=B, s=C, qt=D, st=E_, E=2, N=4, K=8, t=BF16: L.tc_quantize_weights(w, q, s, qt, st, E, N, K, t, None)  # noqa: E731
    assert call(w=None) == call(q=None) == call(s=None) == call(qt=None) == call(st=None) == NULL
    assert call(E=0) == call(N=0) == call(K=-1) == call(t=3) == SHAPE
    assert call(q=A) == call(s=B) == call(qt=B) == call(st=D) == call(st=A) == ALIAS
    assert call(w=A + 2) == call(q=B + 8) == call(s=C + 1) == call(qt=D + 8) == call(st=E_ + 2) == ALIGN
    assert call(E=BIG) == call(N=BIG) == call(K=BIG) == call(E=1 << 29, N=1 << 20, K=1 << 20) == UNSUPPORTED


def test_expert_mm_q8(L):
    call = lambda x=A, sx=None, w=B, sw=C, off=D, row=E_, gate=F_, y=G, T=4, R=8, E=2, N=4, K=8, t=BF16, ws=H, n=1 << 20: L.tc_expert_mm_q8(  # noqa: E731
        x, sx, w, sw, off, row, gate, y, T, R, E, N, K, 0, t, ws, n, None)
    assert call(R=0) == call(R=0, T=0, x=None, y=None, ws=None, n=0) == call(R=0, E=1, off=None) == OK
    assert call(x=None) == call(w=None) == call(sw=None) == call(y=None) == NULL
    assert call(T=-1) == call(R=-1) == call(E=0) == call(N=0) == call(K=0) == call(t=3) == call(row=None) == call(off=None) == SHAPE
    assert call(y=A) == call(y=B) == call(y=C) == call(y=D) == call(y=E_) == call(y=F_) == call(y=H) == call(y=I, sx=I) == ALIAS
    assert call(ws=A) == call(ws=B) == call(ws=C) == call(ws=D) == call(ws=E_) == call(ws=F_) == call(ws=I, sx=I) == ALIAS
    assert call(x=A + 2) == call(w=B + 8) == call(sw=C + 1) == call(off=D + 4) == call(row=E_ + 4) == call(gate=F_ + 2) == call(y=G + 2) == call(sx=I + 1) == ALIGN
    assert call(ws=None) == call(ws=H + 8) == call(n=100) == WORKSPACE
    assert call(T=BIG) == call(R=BIG) == call(E=BIG) == call(N=BIG) == call(K=BIG) == call(K=1 << 22) == UNSUPPORTED
    size = L.tc_expert_mm_q8_workspace_bytes
    assert size(0, 8, 2, 4, 8) == size(4, 0, 2, 4, 8) == size(4, 8, 0, 4, 8) == size(BIG, 8, 2, 4, 8) == size(4, 8, 2, 4, -8) == 0
    sizes = [size(T, T, 2, 4, 300) for T in (1, 2, 100, 10000, 1 << 29)]
    assert sizes == sorted(sizes) and sizes[0] >= 3 * 128 + 3


def test_wrappers_refuse_what_does_not_fit():
    """Through the binding, without a GPU: tensors of the host are refused by name."""
    import torch

    X = torch.zeros(4, 8)
    with pytest.raises(TypeError, match="X must be a torch CUDA tensor"):
        tc355.tc_layer_norm(X, X[0], None, X)
    with pytest.raises(TypeError, match="X must be a torch CUDA tensor"):
        tc355.tc_quantize_rows(X, X, X)
    with pytest.raises(TypeError, match="Y must be a torch CUDA tensor"):
        tc355.tc_expert_mm_q8(X, None, X, X, None, None, None, X)
