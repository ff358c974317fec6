"""The gradient of a token table for batches around the lines between its forms, with sums that are exact.

Small whole numbers, a scale of a half: every partial sum is a multiple of 1/2 below 2^23, which 32 bits hold, so a result is the exact sum rounded
once to the storage type and has to be equal bit by bit, whatever the order.  A token that is lost or counted twice anywhere shows."""
import numpy as np
import pytest
import torch

from paper_1802_04730_amd import tc355 as tc
from test_gpu_experts import TYPES, _bytes, _ints

pytestmark = pytest.mark.gpu


def _whole(shape, dtype, seed):
    return torch.from_numpy(np.random.default_rng(seed).integers(-4, 5, shape).astype(np.float32)).to(dtype).cuda()


def _numbers(T, E, seed):
    """A run over hundreds of places, runs of some chunks, many short ones, numbers outside and a pad; shuffled."""
    rng = np.random.default_rng(seed)
    Idx = rng.integers(-1, E + 1, T)
    Idx[:T // 8] = 3
    Idx[T // 8:T // 8 + 100] = E - 1
    Idx[T // 4:T // 4 + 64] = 5  # (two whole chunks, if they fall so)
    return rng.permutation(Idx)


def _check(dtype, grad, E, D, T, add, Idx, pad, ws):
    dO = _whole((T, D), dtype, T + D)
    dLUT = _whole((E, D), grad, 1) if add else torch.full((E, D), float("nan"), dtype=grad, device="cuda")
    at = torch.from_numpy(np.where((Idx >= 0) & (Idx < E) & (Idx != pad), Idx, E)).cuda()
    want = torch.zeros((E + 1, D), dtype=torch.float64, device="cuda").index_add_(0, at, dO.double())[:E] * 0.5
    want = (want + dLUT.double() if add else want).to(grad)
    tc.tc_embed_grad(dO, _ints(Idx), dLUT, ws, 0.5, pad, add)
    assert torch.equal(dLUT, want), (T, add)


@pytest.mark.parametrize("dtype,grad", [(d, g) for d in TYPES for g in (d, torch.float32)][1:])
@pytest.mark.parametrize("E,D", [(50, 333), (3000, 24), (7, 1030), (900, 3)])
def test_around_the_lines(dtype, grad, E, D):
    ws = _bytes(tc.tc_embed_grad_workspace_bytes(E, D, 20001))  # (the largest batch's)
    for T in (8190, 8191, 8192, 8193, 14335, 14336, 16384, 20001):
        for add in (False, True):
            _check(dtype, grad, E, D, T, add, _numbers(T, E, T), 4, ws)


@pytest.mark.parametrize("T", [14336, 14336 + 32, 20000])
def test_runs_that_end_with_chunks(T):
    """Numbers in runs of whole chunks, of a chunk and one place, of one number in all."""
    E, D = 700, 40
    ws = _bytes(tc.tc_embed_grad_workspace_bytes(E, D, T))
    for run in (8, 32, 33, 64, 31, T):
        for add in (False, True):
            _check(torch.bfloat16, torch.float32, E, D, T, add, np.arange(T) // run % E, -1, ws)
