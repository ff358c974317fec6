"""The gradient of the experts' weights with the rows cut into parts, with sums that are exact.

Small whole numbers: every product and every partial sum is a whole number below 2^24, which 32 bits hold, so a result is the exact sum rounded once to
its type and has to be equal bit by bit.  A row that is lost or counted twice at a part's or a stage's end shows.  test_expert_choices.py asks the
library's own choice for the tile and the number of parts."""
import numpy as np
import pytest
import torch

from paper_1802_04730_amd import tc355 as tc
from test_gpu_experts import TYPES, _bytes, _ints

pytestmark = pytest.mark.gpu

R, E = 12000, 7
# N, K: tiles of 64, in 8 or 16 parts: whole pieces, rows narrower than one, odd widths
SMALL = [(40, 72), (64, 8), (24, 5), (3, 130), (61, 67)]
# R, E, N, K: tiles of 128 in two or more parts, 16-bit storage
LARGE = [(12000, 1, 2048, 2048), (32768, 4, 1000, 1024), (30000, 2, 1501, 1503)]


def _whole(shape, dtype, seed):
    return torch.from_numpy(np.random.default_rng(seed).integers(-2, 3, shape).astype(np.float32)).to(dtype).cuda()


def _check(dtype, off, rows, N, K, gather, add, seed):
    experts, T = len(off) - 1, 900 if gather else rows
    Row = np.random.default_rng(seed).integers(-1, T + 1, rows) if gather else np.arange(rows)
    dY, X = _whole((rows, N), dtype, seed), _whole((T, K), dtype, seed + 1)
    at = torch.from_numpy(Row).cuda()
    x = torch.where(((at >= 0) & (at < T)).unsqueeze(1), X[at.clamp(0, T - 1)].double(), 0.0)
    sums = torch.stack([dY[a:b].double().t().contiguous() @ x[a:b] for a, b in zip(off[:-1], off[1:])])
    ws = _bytes(tc.tc_expert_mm_grad_w_workspace_bytes(rows, experts, N, K))
    for grad in {dtype, torch.float32}:
        there = _whole((experts, N, K), grad, seed + 2) if add else None
        dW = there.clone() if add else torch.full((experts, N, K), float("nan"), dtype=grad, device="cuda")
        tc.tc_expert_mm_grad_w(dY, X, _ints(off), _ints(Row) if gather else None, dW, ws, add)
        assert tc.last_path() == "expert_mm_grad_w:parts"
        want = (sums + there.double() if add else sums).to(grad)
        assert torch.equal(dW, want), (grad, int((dW != want).sum()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", SMALL)
@pytest.mark.parametrize("parts", [2, 4, 8, 16])
def test_rows_around_the_ends_of_parts(dtype, N, K, parts):
    """Experts with a row less than, as many as, and a row more than whole stages for all parts; fewer rows than parts; one; none."""
    whole = parts * (32 if dtype is torch.float32 else 64)
    for counts in ([3 * whole - 1, 3 * whole, 3 * whole + 1, parts - 1, 0, 1, parts + 1], [whole - 1, 0, whole + 1, 2 * whole - 31, 2 * whole + 33, 17, whole]):
        off = np.concatenate([[0], np.cumsum(counts)])
        assert off[-1] <= R and len(counts) == E
        _check(dtype, off, R, N, K, gather=False, add=False, seed=parts)
        _check(dtype, off, R, N, K, gather=True, add=True, seed=parts + 50)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,experts,N,K", LARGE)
def test_tiles_of_128_in_parts(dtype, rows, experts, N, K):
    for shift in (0, 1, 127):
        off = np.linspace(0, rows - shift, experts + 1).astype(np.int64)
        _check(dtype, off, rows, N, K, gather=shift == 1, add=shift == 127, seed=shift)
