"""Products grouped by expert with sums that are exact, for every kernel.

One operand holds whole numbers of as many bits as its type keeps (fp32: 15 bits), the other -1, 0 and 1; with at most 500 terms every partial sum is a whole
number below 2^24, which 32 bits hold.  So a result is the exact sum rounded once to its type and has to be equal bit by bit: an operand that loses bits
on its way, or a term that is lost or counted twice, shows."""
import numpy as np
import pytest
import torch

from paper_1802_04730_amd import tc355 as tc
from test_gpu_experts import TYPES, _ints

pytestmark = pytest.mark.gpu

MOST = {torch.float32: 1 << 14, torch.bfloat16: 1 << 8, torch.float16: 1 << 7}  # (half: sums stay below its largest value)

# path of the forward product, R, E, N, K
SHAPES = [("rows", 32, 8, 512, 500), ("rows", 90, 5, 96, 333), ("rows", 40, 3, 31, 3), ("tile", 500, 8, 2048, 480), ("tile", 1400, 7, 200, 499), ("tile", 1300, 9, 77, 65), ("tile", 1500, 8, 130, 3),
          ("tile", 4500, 10, 496, 488)]


def _many_bits(shape, dtype, seed):
    m = MOST[dtype]
    return torch.from_numpy(np.random.default_rng(seed).integers(-m + 1, m, shape).astype(np.float32)).to(dtype).cuda()


def _signs(shape, dtype, seed):
    return torch.from_numpy(np.random.default_rng(seed).integers(-1, 2, shape).astype(np.float32)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("path,R,E,N,K", SHAPES)
@pytest.mark.parametrize("swap", [False, True])
def test_sums_are_exact(dtype, path, R, E, N, K, swap):
    a, b = (_signs, _many_bits) if swap else (_many_bits, _signs)
    rng = np.random.default_rng(R + N)
    share = R // E  # (at most 500 rows an expert, uneven, one without any)
    off = np.minimum(np.cumsum([0] + [0 if e == 1 else int(share * rng.uniform(0.5, 1.1)) for e in range(E)]), R)
    assert max(np.diff(off)) <= 500 and K <= 500
    X, W, dY, V = a((R, K), dtype, 1), b((E, N, K), dtype, 2), a((R, N), dtype, 3), b((R, K), dtype, 4)
    if N > 500:
        dY[:, 500:] = 0  # (no more terms than that for dX)
    Y, dX, dW = torch.full_like(dY, float("nan")), torch.full_like(X, float("nan")), torch.full_like(W, float("nan"))
    tc.tc_expert_mm(X, W, _ints(off), None, Y)
    assert tc.last_path() == "expert_mm:" + path
    tc.tc_expert_mm_grad_x(dY, W, _ints(off), None, dX)
    tc.tc_expert_mm_grad_w(dY, V, _ints(off), None, dW)
    wY, wdX, wdW = (torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (Y, dX, dW))
    for e in range(E):
        i, j = int(off[e]), int(off[e + 1])
        w = W[e].double()
        wY[i:j], wdX[i:j], wdW[e] = X[i:j].double() @ w.t().contiguous(), dY[i:j].double() @ w, dY[i:j].double().t().contiguous() @ V[i:j].double()
    assert torch.equal(Y, wY.to(dtype)) and torch.equal(dX, wdX.to(dtype)) and torch.equal(dW, wdW.to(dtype))
