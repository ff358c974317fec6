"""Products grouped by expert at the extents where the larger tiles and the cut of long experts' rows are taken, against float64.

Tolerances as in test_gpu_experts.py.  test_expert_plans.py asks the library's own choice which tile each shape takes."""
import numpy as np
import pytest
import torch

from paper_1802_04730_amd import tc355 as tc
from test_gpu_experts import UNIT, _bytes, _ints, _rand

pytestmark = pytest.mark.gpu

# T, R, E, N, K: tiles of 256 forward (of 128 where K is odd), reductions of one stage, of whole ones, of a part of one
FORWARD = [(1500, 4100, 3, 3600, 200), (700, 4200, 2, 3700, 64), (4000, 4000, 1, 4096, 1000), (900, 5000, 7, 3400, 8), (1000, 4100, 3, 3601, 201)]
# T, R, E, N, K: some dozens of rows an expert
SOME_ROWS = [(100, 120, 4, 100, 136), (200, 126, 2, 33, 77), (64, 250, 5, 64, 512), (50, 20, 1, 17, 3), (300, 700, 12, 130, 1000)]
# R, E, N, K: tiles of 128 for dX
BACK_X = [(4100, 3, 200, 3600), (4000, 2, 64, 3700), (4100, 5, 1000, 3400), (4100, 3, 201, 3603)]
# T, R, E, N, K: tiles of 128 for dW
BACK_W = [(400, 1000, 3, 2000, 1000), (100, 300, 8, 1024, 1032), (500, 700, 6, 1001, 1100)]
# R, E, N, K: rows cut into parts
PARTS = [(8192, 1, 512, 512), (20000, 3, 130, 120), (3000, 2, 61, 67), (9000, 4, 64, 8)]


def _offsets(R, E, seed):
    """Uneven, an empty expert among them, some rows left over."""
    cuts = np.sort(np.random.default_rng(seed).integers(0, R - R // 50, E + 1))
    cuts[0] = 0
    if E > 2:
        cuts[2] = cuts[1]
    return cuts


def _close(got, want, mag, n, dtype):
    tol = UNIT[dtype] * want.abs() + 2 * (n + 4) * 2.0 ** -24 * mag + 2.0 ** -24
    assert bool(((got.double() - want).abs() <= tol).all()), "%s: worst %g of its tolerance" % (tc.last_path(), float(((got.double() - want).abs() / tol).max()))


def _source(X, Row):
    if Row is None:
        return X.double()
    return torch.where(((Row >= 0) & (Row < len(X))).unsqueeze(1), X[Row.clamp(0, len(X) - 1).long()].double(), 0.0)


def _by_expert(off, rows, cols, product):
    want, mag = (torch.zeros((rows, cols), dtype=torch.float64, device="cuda") for _ in range(2))
    for e in range(len(off) - 1):
        want[off[e]:off[e + 1]], mag[off[e]:off[e + 1]] = product(e, off[e], off[e + 1])
    return want, mag


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,R,E,N,K", FORWARD)
def test_forward(dtype, T, R, E, N, K):
    off = _offsets(R, E, R)
    Row = _ints(np.random.default_rng(R).integers(-1, T + 1, R))
    X, W, Y = _rand((T, K), dtype, 1), _rand((E, N, K), dtype, 2, K ** -0.5), torch.full((R, N), float("nan"), dtype=dtype, device="cuda")
    tc.tc_expert_mm(X, W, _ints(off), Row, Y, True)
    assert tc.last_path() == "expert_mm:tile"
    x, w = _source(X, Row), W.double()
    want, mag = _by_expert(off, R, N, lambda e, a, b: ((x[a:b] @ w[e].t()).clamp(min=0), x[a:b].abs() @ w[e].abs().t()))
    _close(Y, want, mag, K, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,R,E,N,K", SOME_ROWS)
@pytest.mark.parametrize("gather", [False, True])
def test_some_rows_an_expert(dtype, T, R, E, N, K, gather):
    off = _offsets(R, E, R + 4)
    Row = _ints(np.random.default_rng(R).integers(-1, T + 1, R)) if gather else None
    X, W, Y = _rand((T if gather else R, K), dtype, 1), _rand((E, N, K), dtype, 2, K ** -0.5), torch.full((R, N), float("nan"), dtype=dtype, device="cuda")
    tc.tc_expert_mm(X, W, _ints(off), Row, Y, gather)
    assert tc.last_path() == "expert_mm:rows"
    x, w = _source(X, Row), W.double()
    want, mag = _by_expert(off, R, N, lambda e, a, b: (x[a:b] @ w[e].t(), x[a:b].abs() @ w[e].abs().t()))
    _close(Y, want.clamp(min=0) if gather else want, mag, K, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R,E,N,K", BACK_X)
def test_gradient_of_the_rows(dtype, R, E, N, K):
    off = _offsets(R, E, R + 1)
    dY, W, gate, dX = _rand((R, N), dtype, 1), _rand((E, N, K), dtype, 2, N ** -0.5), _rand((R, K), dtype, 3), torch.full((R, K), float("nan"), dtype=dtype, device="cuda")
    tc.tc_expert_mm_grad_x(dY, W, _ints(off), gate, dX)
    d, w = dY.double(), W.double()
    want, mag = _by_expert(off, R, K, lambda e, a, b: (torch.where(gate[a:b] > 0, d[a:b] @ w[e], 0.0), d[a:b].abs() @ w[e].abs()))
    _close(dX, want, mag, N, dtype)


def _weights(dY, x, off, there):
    want, mag = (torch.stack(v) for v in zip(*[(dY[a:b].t() @ x[a:b], dY[a:b].abs().t() @ x[a:b].abs()) for a, b in zip(off[:-1], off[1:])]))
    return (want, mag) if there is None else (want + there, mag + there.abs())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,R,E,N,K", BACK_W)
def test_gradient_of_the_weights(dtype, T, R, E, N, K):
    off = _offsets(R, E, R + 2)
    Row = _ints(np.random.default_rng(R).integers(-1, T + 1, R))
    X, dY, dW = _rand((T, K), dtype, 1), _rand((R, N), dtype, 2), torch.full((E, N, K), float("nan"), dtype=dtype, device="cuda")
    tc.tc_expert_mm_grad_w(dY, X, _ints(off), Row, dW)
    _close(dW, *_weights(dY.double(), _source(X, Row), off, None), R, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R,E,N,K", PARTS)
@pytest.mark.parametrize("add", [False, True])
def test_rows_cut_into_parts(dtype, R, E, N, K, add):
    off = _offsets(R, E, R + 3)
    need = tc.tc_expert_mm_grad_w_workspace_bytes(R, E, N, K)
    assert need
    for grad, T in ((dtype, R), (torch.float32, 700)):
        Row = None if T == R else _ints(np.random.default_rng(R).integers(-1, T + 1, R))
        X, dY = _rand((T, K), dtype, 1), _rand((R, N), dtype, 2)
        dW = _rand((E, N, K), grad, 3) if add else torch.full((E, N, K), float("nan"), dtype=grad, device="cuda")
        want = _weights(dY.double(), _source(X, Row), off, dW.double() if add else None)
        got = [dW.clone() for _ in range(3)]
        for g, ws in zip(got, (_bytes(need), torch.full((need,), 255, dtype=torch.uint8, device="cuda"), None)):
            tc.tc_expert_mm_grad_w(dY, X, _ints(off), Row, g, ws, add)
            assert tc.last_path() == "expert_mm_grad_w:" + ("tile" if ws is None else "parts")
            _close(g, *want, R, grad)
        assert torch.equal(got[0], got[1])


def test_too_small_a_workspace_only_costs_time():
    R, E, N, K = PARTS[0]
    dY, X, dW = _rand((R, N), torch.bfloat16, 1), _rand((R, K), torch.bfloat16, 2), torch.empty((E, N, K), dtype=torch.bfloat16, device="cuda")
    tc.tc_expert_mm_grad_w(dY, X, _ints([0, R]), None, dW, _bytes(4 * E * N * K))  # (one part's)
    assert tc.last_path() == "expert_mm_grad_w:tile"
    _close(dW, *_weights(dY.double(), X.double(), [0, R], None), R, torch.bfloat16)


def test_rows_beyond_4_gb():
    """Rows taken from both ends of a matrix of more than 4 GB: no tile addresses them by 32 bits."""
    T, R, E, N, K = (1 << 20) + 9, 4100, 3, 3600, 2056
    off = _offsets(R, E, 9)
    places = torch.tensor([0, 1, 1 << 19, (1 << 20) - 1, 1 << 20, T - 1], device="cuda")
    X = torch.empty((T, K), dtype=torch.bfloat16, device="cuda")
    X[places] = _rand((len(places), K), torch.bfloat16, 1)
    Row = places[torch.from_numpy(np.random.default_rng(2).integers(0, len(places), R)).cuda()].to(torch.int32)
    W, Y, dY = _rand((E, N, K), torch.bfloat16, 3, K ** -0.5), torch.empty((R, N), dtype=torch.bfloat16, device="cuda"), _rand((R, N), torch.bfloat16, 4)
    tc.tc_expert_mm(X, W, _ints(off), Row, Y)
    x, w = X[Row.long()].double(), W.double()
    _close(Y, *_by_expert(off, R, N, lambda e, a, b: (x[a:b] @ w[e].t(), x[a:b].abs() @ w[e].abs().t())), K, torch.bfloat16)
    tc.tc_expert_mm_grad_w(dY, X, _ints(off), Row, W)
    _close(W, *_weights(dY.double(), x, off, None), R, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_results_beyond_the_type_and_far_below_one(dtype):
    """Sums that no value of the type holds become infinite, as by one rounding; products of small values are not lost on the way."""
    R, E, N, K = 200, 2, 136, 64
    big, small = (3e38, 1e-18) if dtype is torch.bfloat16 else (6e4, 1e-3)
    off = _ints([0, 90, R])
    for value, other in ((big, 1.0), (small, small)):
        X, W = torch.full((R, K), value, dtype=dtype, device="cuda"), torch.full((E, N, K), other, dtype=dtype, device="cuda")
        Y = torch.empty((R, N), dtype=dtype, device="cuda")
        tc.tc_expert_mm(X, W, off, None, Y)
        want = (X.double() @ W[0].double().t()).float().to(dtype)
        assert torch.equal(Y, want) or bool(((Y.double() - want.double()).abs() <= 2 * UNIT[dtype] * want.double().abs()).all())
        assert bool(torch.isinf(Y).all()) == (value == big)


# R, E, N, K: tiles of 256 forward, tiles of 128 for dX, rows cut into parts for dW
DECREASING = [(4100, 3, 3600, 200), (4100, 3, 200, 3600), (3000, 3, 64, 64)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_offsets_that_decrease_on_large_tiles_and_in_parts(dtype):
    """An offset below an earlier one counts as that one."""
    for R, E, N, K in DECREASING:
        raw = [0, R - 700, R // 3, R - 100]
        off = np.maximum.accumulate(raw)
        X, W, dY = _rand((R, K), dtype, 1), _rand((E, N, K), dtype, 2, K ** -0.5), _rand((R, N), dtype, 3)
        Y, dX, dW = (torch.full_like(t, float("nan")) for t in (dY, X, W))
        tc.tc_expert_mm(X, W, _ints(raw), None, Y)
        tc.tc_expert_mm_grad_x(dY, W, _ints(raw), None, dX)
        tc.tc_expert_mm_grad_w(dY, X, _ints(raw), None, dW, _bytes(tc.tc_expert_mm_grad_w_workspace_bytes(R, E, N, K)))
        x, w, d = X.double(), W.double(), dY.double()
        _close(Y, *_by_expert(off, R, N, lambda e, a, b: (x[a:b] @ w[e].t(), x[a:b].abs() @ w[e].abs().t())), K, dtype)
        _close(dX, *_by_expert(off, R, K, lambda e, a, b: (d[a:b] @ w[e], d[a:b].abs() @ w[e].abs())), N, dtype)
        _close(dW, *_weights(d, x, off, None), R, dtype)
