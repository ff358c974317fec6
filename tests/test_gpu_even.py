"""Layer norm, the balanced router, blocks of 8 bits and products of them on the GPU against the float64 oracle.

Tolerances, before any run.  u: half a step of the output's type; c: 2^-24, or 2^-52 for float32 rows, whose sums are in 64 bits.
A sum of n terms that has at most d additions in a row is off by d c times its terms' magnitudes.
 - norm: d = columns of a thread + 16.  The mean is off by dm = d c mean|x|; y = (x - m) / s by |1/s| dm + |y| er, er = d c + (dm / s)^2 + 8 c (the squares'
   sum moves by the mean's error squared, since the differences sum to nothing).
 - products: float32 outputs 2 (K + 4) 2^-24 of the terms' magnitudes.  16-bit outputs besides: of 8 products the matrix core keeps the bits down to 2^-13 of
   the largest exponent, seven terms lose less than 2^-13 of that each: 2^-10 of the magnitudes.  Small whole numbers are summed exactly.
 - blocks of 8 bits: no tolerance.
"""
import numpy as np
import pytest
import torch

from oracle import even as ref
from paper_1802_04730_amd import tc355 as tc

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
STEP = {F32: 2.0 ** -126, BF16: 2.0 ** -126, F16: 2.0 ** -24}
E4, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _rand(shape, dtype, seed, std=1.0, mean=0.0):
    return (torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32)) * std + mean).to(dtype).cuda()


def _np(t):
    return None if t is None else (t.double() if t.is_floating_point() else t.long()).cpu().numpy()


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _nan(shape, dtype):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def _within(got, want, tol, what=""):
    g = _np(got)
    assert g.shape == want.shape, what
    bad = ~(np.abs(g - want) <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %g over its tolerance" % (what, bad.sum(), bad.size, np.nanmax(np.where(bad, np.abs(g - want) / tol, 0)))


# ---- layer norm ---------------------------------------------------------------------------------------------------------------


def _norm_errors(X, W, dtype, eps):
    """y, 1/s and how far they may be off."""
    _, y, r = ref.layer_norm(X, np.ones_like(W), None, eps)
    c, d = 2.0 ** (-52 if dtype is F32 else -24), max(64, X.shape[1] / 256) + 16
    dm = d * c * np.abs(X).mean(axis=1, keepdims=True)
    er = d * c + (dm * r) ** 2 + 8 * c
    return y, r, r * dm + np.abs(y) * er, er, c, d * c


def _check_norm(X, W, B, eps):
    dtype = X.dtype
    O = _nan(X.shape, dtype)
    tc.tc_layer_norm(X, W, B, O, eps)
    path = tc.last_path()
    x, w, b = _np(X), _np(W), _np(B)
    eps = float(np.float32(eps))
    want = ref.layer_norm(x, w, b, eps)[0]
    y, _, ey, _, c, _ = _norm_errors(x, w, dtype, eps)
    _within(O, want, UNIT[dtype] * np.abs(want) + np.abs(w) * ey + 2 * c * (np.abs(y * w) + (0 if b is None else np.abs(b))) + STEP[dtype], "O")
    return path


def _check_norm_grad(dO, X, W, bias, eps, add=False, ws=True):
    dtype, kind, (T, N) = X.dtype, W.dtype, X.shape
    dX = _nan(X.shape, dtype)
    dW, dB = ((_rand((N,), kind, s) if add else _nan((N,), kind)) for s in (31, 32))
    there = _np(dW) if add else 0, _np(dB) if add else 0
    tc.tc_layer_norm_grad(dO, X, W, dX, dW, dB if bias else None, _bytes(tc.tc_layer_norm_grad_workspace_bytes(T, N)), eps, add)
    path = tc.last_path()
    x, w, g = _np(X), _np(W), _np(dO)
    eps = float(np.float32(eps))
    want, gw, gb = ref.layer_norm_grad(g, x, w, eps)
    y, r, ey, er, c, e1 = _norm_errors(x, w, dtype, eps)
    h = np.abs(g * w)
    mean = lambda a: a.mean(axis=1, keepdims=True)  # noqa: E731
    c1, c2 = np.abs(mean(g * w)), np.abs(mean(g * w * y))
    tol = UNIT[dtype] * np.abs(want) + r * (4 * c * (h + c1 + np.abs(y) * c2) + e1 * mean(h) + np.abs(y) * (e1 * mean(h * np.abs(y)) + mean(h * ey)) + ey * c2) + np.abs(want) * er
    _within(dX, want, tol + STEP[dtype], "dX")
    n = -(-T // 512) + 96  # additions in a row: a thread's rows, a workgroup's, the parts'
    for got, total, mag, far, before in ((dW, gw, np.abs(g * y).sum(0), (np.abs(g) * ey).sum(0), there[0]), (dB if bias else None, gb, np.abs(g).sum(0), 0, there[1])):
        if got is not None:
            total = total + before
            _within(got, total, UNIT[kind] * np.abs(total) + n * c * (mag + np.abs(before)) + far + STEP[kind], "dW, dB")
    return path


NORM_SHAPES = [(1, 1), (3, 2), (5, 7), (1, 8), (4, 9), (40, 33), (7, 64), (130, 100), (33, 255), (1000, 333), (9, 512), (70, 1023), (5, 2048), (33, 2049), (700, 4096),
               (6, 8189), (3, 8192), (2, 12001), (40, 16400)]


@pytest.mark.parametrize("dtype,kind", [(d, k) for d in TYPES for k in dict.fromkeys((d, F32))])
@pytest.mark.parametrize("T,N", NORM_SHAPES)
def test_layer_norm(dtype, kind, T, N):
    X = _rand((T, N), dtype, T + N, 2.0, 0.5)
    W, B = _rand((N,), kind, 1, 0.3, 1.0), _rand((N,), kind, 2)
    for b in (B, None):
        path = _check_norm(X, W, b, 1e-5)
    assert path == ("layer_norm:long" if N > (4096 if dtype is F32 else 8192) else "layer_norm:rows")


@pytest.mark.parametrize("dtype,kind", [(d, k) for d in TYPES for k in dict.fromkeys((d, F32))])
@pytest.mark.parametrize("T,N", NORM_SHAPES)
@pytest.mark.parametrize("add", [False, True])
def test_layer_norm_grad(dtype, kind, T, N, add):
    X, dO = _rand((T, N), dtype, T + N, 2.0, 0.5), _rand((T, N), dtype, T + N + 1)
    W = _rand((N,), kind, 1, 0.3, 1.0)
    for bias in (True, False):
        _check_norm_grad(dO, X, W, bias, 1e-5, add)


def test_layer_norm_of_many_rows():
    """More rows than workgroups go at a time: each takes several; parts of the sums reach their largest number."""
    X, dO, W, B = _rand((20011, 72), BF16, 1), _rand((20011, 72), BF16, 2), _rand((72,), F32, 3), _rand((72,), F32, 4)
    _check_norm(X, W, B, 1e-6)
    _check_norm_grad(dO, X, W, True, 1e-6)
    X, dO = _rand((9001, 5), F32, 1), _rand((9001, 5), F32, 2)
    _check_norm_grad(dO, X, _rand((5,), F32, 3), True, 1e-6)


@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_far_from_zero(dtype):
    """Rows whose mean is far above their spread: squares of the values would lose it."""
    x = torch.arange(600, device="cuda").view(1, 600) % 7
    X = (x + torch.tensor([[0.0], [1000.0], [240.0]], device="cuda")).to(dtype)
    _check_norm(X, _rand((600,), dtype, 1), None, 1e-5)
    _check_norm_grad(_rand((3, 600), dtype, 2), X, _rand((600,), dtype, 1), True, 1e-5)


def test_layer_norm_of_equal_and_of_special_values():
    X = torch.ones(6, 40, device="cuda")
    X[1, 3], X[2, 5], X[3] = float("inf"), float("nan"), 0.0
    X[4] *= 2
    O, dX = _nan((6, 40), F32), _nan((6, 40), F32)
    W, B = _rand((40,), F32, 1), _rand((40,), F32, 2)
    tc.tc_layer_norm(X, W, B, O)
    assert torch.equal(O[[0, 3, 4, 5]], B.expand(4, 40)) and bool(O[1:3].isnan().all())
    tc.tc_layer_norm_grad(torch.ones_like(X), X, W, dX, None, None)
    assert bool(dX[1:3].isnan().all()) and not bool(dX[[0, 3, 4, 5]].isnan().any())
    tc.tc_layer_norm(X, W, B, O, 0.0)  # variance 0 and eps 0
    assert bool(O.isnan().all())


def test_layer_norm_of_a_row_of_2_25():
    """Squares and products of one size: sums of 32 bits along such a row would be off by a part in 2^9.  Along rows beyond registers they are of 64: c = 2^-24 times the 8
    neighbours that are added first, the mean's, the squares' and the results' roundings."""
    N, c = 1 << 25, 2.0 ** -24
    X = torch.full((1, N), 0.55, dtype=F16, device="cuda")
    X[:, ::2].neg_()
    W, O = torch.ones(N, dtype=F16, device="cuda"), _nan((1, N), F16)
    a = float(X[0, 1])
    tc.tc_layer_norm(X, W, None, O, 0.0)
    assert float((O[0, 1::2].float() - 1).abs().max()) <= UNIT[F16] + 24 * c and float((O[0, ::2].float() + 1).abs().max()) <= UNIT[F16] + 24 * c
    dX = _nan((1, N), F16)
    tc.tc_layer_norm_grad(torch.full_like(X, a), X, W, dX, None, None, None, 0.0)
    assert float(dX.float().abs().max()) <= 24 * c  # (h equals its mean)


def test_layer_norm_without_rows():
    X, W = torch.empty((0, 9), device="cuda"), torch.ones(9, device="cuda")
    tc.tc_layer_norm(X, W, None, X)
    for add in (False, True):
        dW, dB = torch.full((9,), 3.0, device="cuda"), torch.full((9,), 4.0, device="cuda")
        tc.tc_layer_norm_grad(X, X, W, X, dW, dB, None, add=add)
        assert bool((dW == (3.0 if add else 0.0)).all()) and bool((dB == (4.0 if add else 0.0)).all())


def test_layer_norm_grad_by_differences():
    """Central differences of sum(dO * O) in 64 bits: off by h^2 times the third derivative, well below 1e-6 for values of about one."""
    T, N, h, eps = 3, 13, 1e-4, 1e-3
    X, W, dO = _rand((T, N), F32, 1), _rand((N,), F32, 2), _rand((T, N), F32, 3)
    dX, dW, dB = _nan((T, N), F32), _nan((N,), F32), _nan((N,), F32)
    tc.tc_layer_norm_grad(dO, X, W, dX, dW, dB, _bytes(tc.tc_layer_norm_grad_workspace_bytes(T, N)), eps)
    x, w, g, b = _np(X), _np(W), _np(dO), np.zeros(N)
    loss = lambda x, w, b: (g * ref.layer_norm(x, w, b, float(np.float32(eps)))[0]).sum()  # noqa: E731

    def slope(a, j, f):
        up, down = a.copy(), a.copy()
        up[j] += h
        down[j] -= h
        return (f(up) - f(down)) / (2 * h)

    for j in np.ndindex(T, N):
        assert abs(slope(x, j, lambda v: loss(v, w, b)) - _np(dX)[j]) < 1e-5
    for j in range(N):
        assert abs(slope(w, j, lambda v: loss(x, v, b)) - _np(dW)[j]) < 1e-5
        assert abs(slope(b, j, lambda v: loss(x, w, v)) - _np(dB)[j]) < 1e-5


# ---- router -------------------------------------------------------------------------------------------------------------------


def _logits(T, E, dtype, seed, std=2.0):
    L = _rand((T, E), dtype, seed, std)
    rng = np.random.default_rng(seed)
    L[torch.from_numpy(rng.random((T, E)) < 0.1).cuda()] = float("-inf")
    L[torch.from_numpy(rng.random(T) < 0.1).cuda()] = float("-inf")
    L[torch.from_numpy(rng.random((T, E)) < 0.1).cuda()] = 0.5  # (ties)
    return L


def _route(L, Bias, k, groups, keep, sigmoid, norm, scale, ws=True):
    T, E = L.shape
    i32 = dict(dtype=torch.int32, device="cuda")
    out = [_nan((T, k), F32), torch.full((T, k), 77, **i32), torch.full((E + 1,), 77, **i32), torch.full((T * k,), 77, **i32), torch.full((T, k), 77, **i32)]
    tc.tc_route_balanced(L, Bias, *out, _bytes(tc.tc_route_balanced_workspace_bytes(T, E, k)) if ws else None, groups, keep, sigmoid, norm, scale)
    return out


def _check_route(L, Bias, k, groups=1, keep=1, sigmoid=True, norm=True, scale=1.5):
    out, want = _route(L, Bias, k, groups, keep, sigmoid, norm, scale), ref.route_balanced(_np(L), _np(Bias), k, groups, keep, sigmoid, norm, scale)
    for name, g, w in zip(("Id", "Off", "Row", "Place"), out[1:], want[1:]):
        assert np.array_equal(_np(g), w), name
    g, w = _np(out[0]), want[0]
    assert np.array_equal(np.isnan(g), np.isnan(w))
    ok = ~np.isnan(w)
    assert (np.abs(g - w)[ok] <= 2.0 ** -24 * (1 + 2.0 ** -20) * w[ok] + 2.0 ** -149).all()  # (64 bits, rounded once)
    return out


ROUTE_SHAPES = [(1, 1, 1, 1, 1), (1, 8, 2, 2, 1), (5, 3, 3, 3, 2), (64, 16, 4, 4, 2), (65, 17, 5, 1, 1), (130, 32, 1, 8, 8), (70, 36, 8, 12, 3), (200, 60, 6, 3, 2), (90, 128, 16, 8, 3),
                (67, 129, 8, 3, 1), (40, 100, 20, 50, 20), (66, 256, 64, 16, 5), (70, 256, 8, 8, 4), (35, 256, 7, 1, 1), (20, 300, 17, 20, 7), (30, 1020, 9, 60, 4), (300, 6, 2, 6, 3),
                (40, 64, 3, 64, 5)]  # T, E, k, groups, keep


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sigmoid,norm", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("T,E,k,groups,keep", ROUTE_SHAPES)
def test_route_balanced(dtype, sigmoid, norm, T, E, k, groups, keep):
    L = _logits(T, E, dtype, T * E + k)
    _check_route(L, _rand((E,), F32, E, 0.1 if sigmoid else 0.3 / E), k, groups, keep, sigmoid, norm)
    _check_route(L, None, k, groups, keep, sigmoid, norm, 1.0)


def test_route_balanced_tells_scores_apart_that_agree_in_32_bits():
    """Biases that differ by less than a step of 2^-24 at one half: the order is that of 64 bits."""
    E, T = 48, 50
    rng = np.random.default_rng(1)
    L = torch.zeros((T, E), device="cuda")
    Bias = torch.from_numpy((rng.permutation(E) * 2.0 ** -40).astype(np.float32)).cuda()
    for groups, keep in ((1, 1), (6, 2)):
        out = _check_route(L, Bias, 8, groups, keep)
    assert len(set(_np(out[1])[0])) == 8


@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("E,k,groups,keep", [(256, 4, 1, 1), (256, 4, 16, 9), (30, 4, 1, 1), (300, 20, 1, 1), (64, 1, 1, 1)])
def test_route_balanced_finds_a_larger_score_behind_equal_ones(sigmoid, E, k, groups, keep):
    """Scores far below the largest, most of them equal, one of a late expert larger by less than a part in 2^28 of the largest."""
    T = 40
    L = torch.full((T, E), -20.0, device="cuda")
    L[:, 0] = _rand((T,), F32, 5).abs()
    for t in range(T):
        L[t, E - 1 - t % 7] = -20.0 + 0.125 * (t % 9)
        L[t, E // 2] = -20.0 + 0.25 * (t % 5)
    _check_route(L, None, k, groups, keep, sigmoid, False)
    _check_route(L[:, 1:].contiguous() if groups == 1 else L, None, k, groups, keep, sigmoid, False)


@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("E,k,groups,keep", [(2, 1, 1, 1), (8, 3, 1, 1), (8, 3, 4, 2), (100, 5, 10, 3), (256, 8, 16, 5), (600, 20, 1, 1)])
def test_route_balanced_of_biases_far_beyond_the_scores(sigmoid, E, k, groups, keep):
    """An expert that every token shall have, one that none shall have: the order stays that of the formula, whatever the biases' size."""
    L = _rand((50, E), F32, E, 2.0)
    for high in (3.0, 3.0e6, 1.7e9, 2.9e15, 1.0e30, torch.finfo(F32).max):
        for at in ([E - 1], [0], [E // 2, E // 3], []):
            for low in (0.0, -high):
                Bias = _rand((E,), F32, 7, 0.1)
                Bias[E // 4] = low
                Bias[at] = high
                _check_route(L, Bias, k, groups, keep, sigmoid, True)
    _check_route(L, torch.full((E,), -3.0e9, device="cuda"), k, groups, keep, sigmoid, True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_route_balanced_of_special_logits(dtype, sigmoid, norm):
    low, nan, inf = torch.finfo(dtype).min, float("nan"), float("inf")
    L = torch.tensor([[-inf] * 6, [low] * 6, [low, -inf, low, -inf, -inf, low], [nan, 1, 2, 3, 4, 5], [1, inf, 2, 0, 0, 0], [0.0, -0.0, 0.0, -0.0, 0.0, 0], [-0.0, 0.0, -1, -inf, low, 0],
                      [nan] * 6, [nan, -inf, -inf, -inf, -inf, 1], [inf, inf, -inf, 3, nan, 0], [torch.finfo(dtype).max, low, 0, 0, 0, 90], [-90, -91, -92, -93, -94, -95]], dtype=dtype).cuda()
    for Bias in (None, torch.tensor([0.0, -1.0, 0.5, -inf, 0.25, nan], device="cuda"), torch.tensor([inf, inf, 0, 0, 0, 0], device="cuda")):
        for k, groups, keep in ((1, 1, 1), (3, 3, 2), (6, 6, 5), (2, 2, 1)):
            _check_route(L, Bias, k, groups, keep, sigmoid, norm)


def test_route_balanced_of_many_tokens():
    for T, E, k, groups, keep in ((64 * 30 + 1, 8, 3, 4, 2), (33, 12, 2, 3, 1), (32, 12, 2, 3, 1)):
        _check_route(_logits(T, E, BF16, T), _rand((E,), F32, 2, 0.1), k, groups, keep)
    _check_route(_logits(4500, 16, F32, 2), None, 2, 4, 2)
    L = _logits(64, 16, F32, 3)  # without a workspace one workgroup does it all
    for a, b in zip(_route(L, None, 4, 4, 2, True, True, 1.0, ws=False), _route(L, None, 4, 4, 2, True, True, 1.0)):
        assert torch.equal(a, b)


def test_route_balanced_without_tokens():
    assert not bool(_route(torch.empty((0, 6), device="cuda"), None, 2, 2, 1, True, True, 1.0)[2].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sigmoid,norm", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("T,E,k,groups,keep", [(1, 1, 1, 1, 1), (9, 8, 2, 2, 1), (33, 17, 5, 1, 1), (20, 64, 16, 4, 3), (21, 130, 20, 5, 2), (17, 256, 8, 8, 4), (5, 1023, 3, 1, 1), (300, 12, 4, 3, 2)])
def test_route_balanced_grad(dtype, sigmoid, norm, T, E, k, groups, keep):
    L = _logits(T, E, dtype, T + E)
    Id = _route(L, _rand((E,), F32, 1, 0.1), k, groups, keep, sigmoid, norm, 1.5)[1]
    dWt = _rand((T, k), F32, 4)
    dL = _nan((T, E), dtype)
    tc.tc_route_balanced_grad(L, Id, dWt, dL, sigmoid, norm, 1.5)
    want = ref.route_balanced_grad(_np(L), _np(Id), _np(dWt), sigmoid, norm, 1.5)
    # exponentials of 2^-21 and a sum of E of them in 32 bits, on gradients of at most 1.5 max|dWt|; chosen ones in 64
    big = 1.5 * np.abs(_np(dWt)).max()
    _within(dL, want, UNIT[dtype] * np.abs(want) + (2.0 ** -20 + (E + 16) * 2.0 ** -22) * big + STEP[dtype], "dL")


@pytest.mark.parametrize("sigmoid,norm", [(True, True), (True, False), (False, True), (False, False)])
def test_route_balanced_grad_by_differences(sigmoid, norm):
    T, E, k, h, scale = 6, 9, 3, 1e-4, 1.5
    L = _rand((T, E), F32, 12)
    Id, dWt = _route(L, None, k, 3, 2, sigmoid, norm, scale)[1], _rand((T, k), F32, 13)
    dL = torch.empty_like(L)
    tc.tc_route_balanced_grad(L, Id, dWt, dL, sigmoid, norm, scale)
    L0, ids, g = _np(L), _np(Id), _np(dWt)

    def loss(x):
        p = np.take_along_axis(ref.scores(x, sigmoid), ids, 1)
        return (g * scale * (p / p.sum(1, keepdims=True) if norm else p)).sum()

    for j in np.ndindex(T, E):
        up, down = L0.copy(), L0.copy()
        up[j] += h
        down[j] -= h
        assert abs((loss(up) - loss(down)) / (2 * h) - _np(dL)[j]) < 1e-5


@pytest.mark.parametrize("sigmoid", [True, False])
def test_route_balanced_grad_of_scores_far_below_the_others(sigmoid):
    """Chosen for their bias, with scores that 32 bits would lose: weights and gradients are those of the chosen among themselves."""
    L = torch.tensor([[-120.0, -121.0, 3.0, -122.0], [-400.0, -399.0, 5.0, -401.0]], device="cuda")
    out = _check_route(L, torch.tensor([2.0, 2.0, 0.0, 2.0], device="cuda"), 2, 1, 1, sigmoid, True, 1.0)
    dWt, dL = _rand((2, 2), F32, 1), _nan((2, 4), F32)
    tc.tc_route_balanced_grad(L, out[1], dWt, dL, sigmoid, True, 1.0)
    want = ref.route_balanced_grad(_np(L), _np(out[1]), _np(dWt), sigmoid, True, 1.0)
    assert np.abs(want).max() > 0.05
    _within(dL, want, 2.0 ** -20 * (np.abs(want) + 1e-6), "dL")


def test_route_balanced_grad_of_numbers_that_make_no_sense():
    L, dWt = _rand((3, 5), F32, 1), _rand((3, 4), F32, 2)
    for sigmoid in (False, True):
        a, b = _nan((3, 5), F32), _nan((3, 5), F32)
        tc.tc_route_balanced_grad(L, _ints([[0, -1, 7, 2 ** 31 - 1], [5, -2 ** 31, 3, 9], [-1] * 4]), dWt, a, sigmoid, True, 1.0)
        tc.tc_route_balanced_grad(L, _ints([[0, -1, -1, -1], [-1, -1, 3, -1], [-1] * 4]), dWt, b, sigmoid, True, 1.0)
        assert torch.equal(a, b) and not bool(a[2].any()) and not bool(a.isnan().any())


# ---- blocks of 8 bits -------------------------------------------------------------------------------------------------------------


def _e4(*shape):
    return torch.full(shape, 0x55, dtype=torch.uint8, device="cuda").view(E4)


def _e8(*shape):
    return torch.full(shape, 0x55, dtype=torch.uint8, device="cuda").view(E8)


def _up(n):
    return -(-n // 128) * 128


def _same(got, want):
    g = _np(got.float()) if got.dtype is E4 else _np(got.view(torch.uint8))
    assert np.array_equal(g, want, equal_nan=got.dtype is E4)
    if got.dtype is E4:
        assert not bool((got.float() == 0).logical_and(got.view(torch.uint8) != 0).logical_and(torch.from_numpy(want == 0).cuda()).logical_and(got.view(torch.uint8) != 0x80).any())


def _wild(shape, dtype, seed):
    """Values over many binades, ties among them; whole blocks of zeros, of tiny and of huge ones."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * np.exp(2 * rng.standard_normal(shape))
    x = np.where(rng.random(shape) < 0.3, rng.integers(-31, 32, shape) * 2.0 ** rng.integers(-8, 9, shape), x)
    flat = x.reshape(-1, shape[-1])
    kind = rng.integers(0, 6, len(flat))
    flat[kind == 0] = 0
    flat[kind == 1] *= 1e-6 if dtype is F16 else 1e-39
    flat[kind == 2] *= 10 if dtype is F16 else 1e35
    return torch.from_numpy(x).clamp(-torch.finfo(dtype).max, torch.finfo(dtype).max).to(dtype).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,K", [(1, 1), (3, 7), (2, 8), (5, 127), (17, 128), (40, 129), (33, 1000), (300, 256), (1, 4099), (1030, 385)])
def test_quantize_rows(dtype, R, K):
    X = _wild((R, K), dtype, R + K)
    Q, S = _e4(R, _up(K)), _e8(R, _up(K) // 128)
    tc.tc_quantize_rows(X, Q, S)
    for got, want in zip((Q, S), ref.quantize_rows(_np(X))):
        _same(got, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,N,K", [(1, 1, 1), (2, 3, 7), (1, 127, 130), (3, 128, 128), (2, 129, 255), (1, 300, 1000), (5, 256, 384), (1, 5, 2000), (1, 2000, 9)])
def test_quantize_weights(dtype, E, N, K):
    W = _wild((E, N, K), dtype, N + K)
    want = ref.quantize_weights(_np(W))
    n, k = _up(N) // 128, _up(K) // 128
    for both in (True, False):
        out = _e4(E, N, _up(K)), _e8(E, n, k), _e4(E, K, _up(N)) if both else None, _e8(E, k, n) if both else None
        tc.tc_quantize_weights(W, *out)
        for got, w in zip(out, want):
            if got is not None:
                _same(got, w)


@pytest.mark.parametrize("dtype", TYPES)
def test_blocks_that_hold_inf_or_nan(dtype):
    X = _rand((260, 300), dtype, 1)
    X[0, 5], X[1, 200], X[2, 299], X[140, 140] = float("inf"), float("-inf"), float("nan"), float("nan")
    Q, S = _e4(260, 384), _e8(260, 3)
    tc.tc_quantize_rows(X, Q, S)
    for got, want in zip((Q, S), ref.quantize_rows(_np(X))):
        _same(got, want)
    out = _e4(1, 260, 384), _e8(1, 3, 3), _e4(1, 300, 384), _e8(1, 3, 3)
    tc.tc_quantize_weights(X.view(1, 260, 300), *out)
    for got, want in zip(out, ref.quantize_weights(_np(X)[None])):
        _same(got, want)


def test_quantize_rows_without_rows():
    tc.tc_quantize_rows(torch.empty((0, 5), device="cuda"), _e4(0, 128), _e8(0, 1))


# ---- products ---------------------------------------------------------------------------------------------------------------------


def _weights8(W):
    E, N, K = W.shape
    n, k = _up(N) // 128, _up(K) // 128
    out = _e4(E, N, _up(K)), _e8(E, n, k), _e4(E, K, _up(N)), _e8(E, k, n)
    tc.tc_quantize_weights(W, *out)
    return out


def _offsets(E, R, seed, kind):
    rng = np.random.default_rng(seed)
    if kind == "one":
        off = np.where(np.arange(E + 1) > E // 2, R, 0)
    elif kind == "none":
        off = np.zeros(E + 1)
    else:
        off = np.concatenate([[0], np.sort(rng.integers(0, R + 1, E))])
        if kind == "all":
            off[-1] = R
    return off.astype(np.int64)


def _product_close(got, x, w, Off, Row, R, relu, gate, K, dtype, what):
    want, mag = ref.product(x, w, Off, Row, R, relu)
    if gate is not None:
        want, mag = np.where(gate > 0, want, 0), np.where(gate > 0, mag, 0)
    tol = UNIT[dtype] * np.abs(want) + (2 * (K + 4) * 2.0 ** -24 + (0 if dtype is F32 else 2.0 ** -10)) * mag + STEP[dtype]
    _within(got, want, tol, what)


MM_SHAPES = [(1, 1, 1, 1, 1), (3, 5, 2, 7, 9), (20, 40, 4, 64, 64), (50, 30, 3, 130, 72), (300, 410, 5, 136, 200), (60, 150, 70, 24, 40), (33, 64, 9, 129, 257),
             (128, 256, 2, 128, 128), (513, 513, 1, 257, 384), (16, 32, 8, 512, 1000), (7, 14, 130, 48, 33), (40, 260, 2, 8, 1500), (700, 900, 3, 520, 640)]  # T, R, E, N, K


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,R,E,N,K", MM_SHAPES)
@pytest.mark.parametrize("kind", ["some", "all", "one", "none"])
def test_expert_mm_q8(dtype, T, R, E, N, K, kind):
    rng = np.random.default_rng(R + E)
    Off = _offsets(E, R, R, kind)
    W, SW, _, _ = _weights8(_rand((E, N, K), dtype, 1, K ** -0.5))
    w = ref.values(_np(W.float()), _np(SW.view(torch.uint8)))[:, :, :K]
    for gather, relu, gated in ((False, False, True), (True, True, False), (True, False, False), (False, True, True)):
        n = T if gather else R
        X = _rand((n, K), dtype, 2)
        x = ref.values(*ref.quantize_rows(_np(X)))[:, :K]
        Row = rng.integers(-1, T + 1, R) if gather else None  # (a row outside is one of zeros)
        gate = _rand((R, N), dtype, 5) if gated else None
        Y = _nan((R, N), dtype)
        tc.tc_expert_mm_q8(X, None, W, SW, _ints(Off), None if Row is None else _ints(Row), gate, Y, _bytes(tc.tc_expert_mm_q8_workspace_bytes(n, R, E, N, K)), relu)
        _product_close(Y, x, w, Off, Row, R, relu, _np(gate), K, dtype, tc.last_path())
        Q, S = _e4(n, _up(K)), _e8(n, _up(K) // 128)
        tc.tc_quantize_rows(X, Q, S)
        Z = _nan((R, N), dtype)
        tc.tc_expert_mm_q8(Q, S, W, SW, _ints(Off), None if Row is None else _ints(Row), gate, Z, None, relu)
        assert torch.equal(Y, Z)


def _whole(rng, shape, top):
    return torch.from_numpy(rng.integers(-top, top + 1, shape).astype(np.float32)).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,R,E,N,K", [(1, 1, 1, 16, 128), (40, 70, 3, 200, 1000), (256, 700, 4, 640, 1152), (300, 300, 1, 1030, 515), (3000, 3000, 2, 520, 256), (16, 32, 8, 128, 2048),
                                       (9, 700, 2, 300, 1025), (1200, 1200, 1, 2050, 4000)])
def test_products_of_whole_numbers_are_exact(dtype, T, R, E, N, K):
    """Whole numbers of up to 3 bits times powers of two that differ from block to block: sums that the matrix core holds exactly, results that are rounded once."""
    rng = np.random.default_rng(K + R)
    blocks = lambda n: -(-n // 128)  # noqa: E731
    power = lambda *s: torch.from_numpy(2.0 ** rng.integers(-2, 3, s)).float().cuda()  # noqa: E731
    W = _whole(rng, (E, N, K), 7) * power(E, blocks(N), blocks(K)).repeat_interleave(128, 1).repeat_interleave(128, 2)[:, :N, :K]
    X = _whole(rng, (T, K), 7) * power(T, blocks(K)).repeat_interleave(128, 1)[:, :K]
    Off = _offsets(E, R, R, "all")
    Row = rng.permutation(R) % T if R != T else None
    Q, S, Qt, St = _weights8(W.to(dtype))
    x, w = _np(X), _np(W)
    Y = _nan((R, N), dtype)
    tc.tc_expert_mm_q8(X.to(dtype), None, Q, S, _ints(Off) if E > 1 else None, None if Row is None else _ints(Row), None, Y, _bytes(tc.tc_expert_mm_q8_workspace_bytes(T, R, E, N, K)))
    want = ref.product(x, w, Off, Row, R, False)[0]
    assert torch.equal(Y, torch.from_numpy(want).float().cuda().to(dtype)), tc.last_path()
    dY = _whole(rng, (R, N), 7) * power(R, blocks(N)).repeat_interleave(128, 1)[:, :N]
    dX = _nan((R, K), dtype)
    tc.tc_expert_mm_q8(dY.to(dtype), None, Qt, St, _ints(Off), None, None, dX, _bytes(tc.tc_expert_mm_q8_workspace_bytes(R, R, E, K, N)))
    want = ref.product(_np(dY), w.transpose(0, 2, 1), Off, None, R, False)[0]
    assert torch.equal(dX, torch.from_numpy(want).float().cuda().to(dtype)), tc.last_path()


@pytest.mark.parametrize("dtype", TYPES)
def test_scales_from_one_end_to_the_other(dtype):
    """Scales of operands handed over in 8 bits: sums of exponents count, not either one by itself; 255 is NaN."""
    bytes_of = lambda a: torch.from_numpy(np.asarray(a, np.uint8)).cuda()  # noqa: E731
    Q = torch.ones((6, 128), device="cuda").to(E4)
    SX = bytes_of([[1], [120], [127], [200], [254], [255]]).view(E8)
    W = torch.ones((6, 3, 128), device="cuda").to(E4)
    SW = bytes_of([253, 133, 127, 54, 1, 127]).view(6, 1, 1).view(E8)
    Y = _nan((6, 3), dtype)
    tc.tc_expert_mm_q8(Q, SX, W, SW, _ints(np.arange(7)), None, None, Y)
    want = torch.tensor([2.0 ** (a + b - 254 + 7) for a, b in ((1, 253), (120, 133), (127, 127), (200, 54), (254, 1))], device="cuda")
    assert torch.equal(Y[:5].float(), want.view(5, 1).expand(5, 3))
    assert bool(Y[5].isnan().all())


@pytest.mark.parametrize("dtype", TYPES)
def test_what_an_expert_does_not_read_does_not_matter(dtype):
    """NaN in rows of no expert, in other experts' rows and weights; an expert's own stay in their rows, or in the columns of their block."""
    R, E, N, K = 300, 4, 200, 256
    Off = np.array([0, 130, 130, 200, 290])
    X, W = _rand((R, K), dtype, 1), _rand((E, N, K), dtype, 2)
    X[290:], W[1] = float("nan"), float("nan")
    X[140:150, 3], W[3, 7, 9] = float("inf"), float("nan")
    Q, S, _, _ = _weights8(W)
    Y = _nan((R, N), dtype)
    tc.tc_expert_mm_q8(X, None, Q, S, _ints(Off), None, None, Y, _bytes(tc.tc_expert_mm_q8_workspace_bytes(R, R, E, N, K)))
    y = torch.isfinite(Y)
    assert not bool(y[140:150].any()) and not bool(y[200:290, :128].any()) and not bool(Y[290:].any())
    y[140:150], y[200:290, :128] = True, True
    assert bool(y.all())


def test_offsets_that_make_no_sense_stay_inside():
    for R, E, N, K in ((70, 3, 40, 256), (900, 3, 300, 256)):
        X, W = _rand((R, K), BF16, 1), _rand((E, N, K), BF16, 2)
        Q, S, _, _ = _weights8(W)
        ws = _bytes(tc.tc_expert_mm_q8_workspace_bytes(R, R, E, N, K))
        for off in ([0, 50, 20, 5000], [-9, -3, 10, 2 ** 31 - 1], [5, 4, 3, 2], [2 ** 31 - 1, -2 ** 31, 0, 70]):
            big = torch.full((R + 64, N), 7.0, dtype=BF16, device="cuda")
            tc.tc_expert_mm_q8(X, None, Q, S, _ints(off), None, None, big[:R], ws)
            assert bool((big[R:] == 7.0).all()) and not bool(big.isnan().any())
            if off[0] == 5:
                assert bool((big[:5] == 7.0).all()) and not bool(big[5:R].any())


def test_products_of_no_rows():
    Q, S, _, _ = _weights8(_rand((2, 5, 9), F32, 1))
    tc.tc_expert_mm_q8(torch.empty((0, 9), device="cuda"), None, Q, S, _ints([0, 0, 0]), None, None, torch.empty((0, 5), device="cuda"))
    Y = _nan((4, 5), F32)  # rows of nothing: every row is outside
    tc.tc_expert_mm_q8(torch.empty((0, 9), device="cuda"), None, Q, S, _ints([0, 2, 4]), _ints([0, 1, 2, 3]), None, Y)
    assert not bool(Y.any())


# ---- together ---------------------------------------------------------------------------------------------------------------------


def _layer(dtype, T, N, H, E, k, groups, keep, seed=0):
    """A layer of experts behind a norm, forward and backward, as a program runs it; returns its buffers."""
    f = lambda *s, t=dtype: _nan(s, t)  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    R = T * k
    s = dict(X=_rand((T, N), dtype, seed), W=_rand((N,), F32, seed + 1, 0.2, 1.0), B=_rand((N,), F32, seed + 2, 0.1), Wr=_rand((1, E, N), dtype, seed + 3, N ** -0.5),
             Bias=_rand((E,), F32, seed + 4, 0.05), W1=_rand((E, H, N), dtype, seed + 5, N ** -0.5), W2=_rand((E, N, H), dtype, seed + 6, H ** -0.5), dO=_rand((T, N), dtype, seed + 7),
             one=_ints([0, T]), X1=f(T, N), L=f(T, E), Wt=f(T, k, t=F32), Id=i(T, k), Off=i(E + 1), Row=i(R), Place=i(T, k), Y1=f(R, H), Y2=f(R, N), O=f(T, N), dY2=f(R, N), dWt=f(T, k, t=F32),
             dY1=f(R, H), dR=f(R, N), dX1=f(T, N), dL=f(T, E), dX=f(T, N), dW=f(N, t=F32), dB=f(N, t=F32), dW1=f(E, H, N, t=F32), dW2=f(E, N, H, t=F32), dXr=f(T, N))
    s["q1"] = _e4(E, H, _up(N)), _e8(E, _up(H) // 128, _up(N) // 128), _e4(E, N, _up(H)), _e8(E, _up(N) // 128, _up(H) // 128)
    s["q2"] = _e4(E, N, _up(H)), _e8(E, _up(N) // 128, _up(H) // 128), _e4(E, H, _up(N)), _e8(E, _up(H) // 128, _up(N) // 128)
    need = max(tc.tc_layer_norm_grad_workspace_bytes(T, N), tc.tc_route_balanced_workspace_bytes(T, E, k), tc.tc_expert_mm_q8_workspace_bytes(T, R, E, H, N),
               tc.tc_expert_mm_q8_workspace_bytes(R, R, E, N, H), tc.tc_expert_mm_q8_workspace_bytes(R, R, E, H, N), tc.tc_expert_mm_q8_workspace_bytes(R, R, E, N, H))
    s["ws"] = _bytes(need)
    s["groups"], s["keep"] = groups, keep
    return s


def _run_layer(s):
    ws = s["ws"]
    tc.tc_quantize_weights(s["W1"], *s["q1"])
    tc.tc_quantize_weights(s["W2"], *s["q2"])
    tc.tc_layer_norm(s["X"], s["W"], s["B"], s["X1"])
    tc.tc_expert_mm(s["X1"], s["Wr"], s["one"], None, s["L"])
    tc.tc_route_balanced(s["L"], s["Bias"], s["Wt"], s["Id"], s["Off"], s["Row"], s["Place"], ws, s["groups"], s["keep"], True, True, 2.0)
    tc.tc_expert_mm_q8(s["X1"], None, s["q1"][0], s["q1"][1], s["Off"], s["Row"], None, s["Y1"], ws, True)
    tc.tc_expert_mm_q8(s["Y1"], None, s["q2"][0], s["q2"][1], s["Off"], None, None, s["Y2"], ws)
    tc.tc_expert_sum(s["Y2"], s["Wt"], s["Place"], s["O"])
    tc.tc_expert_sum_grad(s["dO"], s["Y2"], s["Wt"], s["Place"], s["dY2"], s["dWt"])
    tc.tc_expert_mm_q8(s["dY2"], None, s["q2"][2], s["q2"][3], s["Off"], None, s["Y1"], s["dY1"], ws)
    tc.tc_expert_mm_q8(s["dY1"], None, s["q1"][2], s["q1"][3], s["Off"], None, None, s["dR"], ws)
    tc.tc_expert_mm_grad_w(s["dY2"], s["Y1"], s["Off"], None, s["dW2"])
    tc.tc_expert_mm_grad_w(s["dY1"], s["X1"], s["Off"], s["Row"], s["dW1"])
    tc.tc_expert_sum(s["dR"], None, s["Place"], s["dX1"])
    tc.tc_route_balanced_grad(s["L"], s["Id"], s["dWt"], s["dL"], True, True, 2.0)
    tc.tc_layer_norm_grad(s["dX1"], s["X"], s["W"], s["dX"], s["dW"], s["dB"], ws)


OUT = ("X1", "L", "Wt", "Id", "Off", "Row", "Place", "Y1", "Y2", "O", "dY1", "dR", "dX1", "dL", "dX", "dW", "dB", "dW1", "dW2")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,N,H,E,k,groups,keep", [(5, 64, 96, 4, 2, 2, 1), (150, 200, 320, 12, 3, 4, 2), (700, 256, 384, 6, 2, 1, 1)])
def test_a_layer_of_experts(dtype, T, N, H, E, k, groups, keep):
    """Each output from those that the library made before it."""
    s = _layer(dtype, T, N, H, E, k, groups, keep)
    _run_layer(s)
    n = {key: _np(v) for key, v in s.items() if isinstance(v, torch.Tensor) and key != "ws"}
    q1, q2 = (ref.quantize_weights(n[w]) for w in ("W1", "W2"))
    x, x1t, x2, x2t = (ref.values(*q)[:, :, :m] for q, m in ((q1[:2], N), (q1[2:], H), (q2[:2], H), (q2[2:], N)))
    rows = lambda name: ref.values(*ref.quantize_rows(n[name]))[:, :n[name].shape[1]]  # noqa: E731
    for a, w in zip((s["Wt"], s["Id"], s["Off"], s["Row"], s["Place"]), ref.route_balanced(n["L"], n["Bias"], k, groups, keep, True, True, 2.0)):
        _within(a, w, 2.0 ** -23 * np.abs(w))
    R = T * k
    _product_close(s["Y1"], rows("X1"), x, n["Off"], n["Row"], R, True, None, N, dtype, "Y1")
    _product_close(s["Y2"], rows("Y1"), x2, n["Off"], None, R, False, None, H, dtype, "Y2")
    _product_close(s["dY1"], rows("dY2"), x2t, n["Off"], None, R, False, n["Y1"], N, dtype, "dY1")
    _product_close(s["dR"], rows("dY1"), x1t, n["Off"], None, R, False, None, H, dtype, "dR")
    want = ref.layer_norm_grad(n["dX1"], n["X"], n["W"], float(np.float32(1e-5)))
    for a, w in zip((s["dX"], s["dW"], s["dB"]), want):
        assert np.linalg.norm(_np(a) - w) <= 2 * UNIT[a.dtype] * np.linalg.norm(w) + 2.0 ** -18 * np.linalg.norm(w)


def test_a_layer_is_the_same_each_time_on_any_stream_and_from_a_graph():
    dtype, shape = BF16, (300, 192, 256, 8, 2, 4, 2)
    s = _layer(dtype, *shape)
    _run_layer(s)
    first = {k: s[k].clone() for k in OUT}

    def same(what):
        torch.cuda.synchronize()
        for k in OUT:
            assert torch.equal(s[k], first[k]), (what, k)
            s[k].zero_()
        torch.cuda.synchronize()

    same("eager")
    _run_layer(s)
    same("again")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _run_layer(s)
    same("another stream")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _run_layer(s)
    other = _layer(dtype, *shape, seed=50)
    for turn in range(4):
        g.replay()
        same("replay %d" % turn)
        _run_layer(other)  # (other work between the replays)
        torch.cuda.synchronize()
