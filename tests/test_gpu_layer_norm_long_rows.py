"""Layer norm of many rows that are too long for registers: workgroups that take several rows each (more than 2048), parts of the sums for dW and dB that take several (more than 512).
Tolerances are test_gpu_even.py's: a column's sum is of ceil(T / 512) rows in turn and 48 parts, which its count of additions covers."""
import numpy as np
import pytest
import torch

from paper_1802_04730_amd import tc355 as tc
from test_gpu_even import BF16, F16, F32, _bytes, _check_norm, _check_norm_grad, _nan, _rand

pytestmark = pytest.mark.gpu

SHAPES = [(1100, 4099, F32), (2100, 4100, F32), (513, 8192, F32), (1030, 9001, F16), (2100, 8200, BF16)]


@pytest.mark.parametrize("T,N,dtype", SHAPES)
def test_norm(T, N, dtype):
    X = _rand((T, N), dtype, T + N, 2.0, 0.5)
    X *= (1 + torch.arange(T, device="cuda") % 5).to(dtype).view(T, 1)  # (rows that differ in mean and spread: one taken for another is seen)
    for kind in dict.fromkeys((dtype, F32)):
        W, B = _rand((N,), kind, 1, 0.3, 1.0), _rand((N,), kind, 2)
        for b in (B, None):
            assert _check_norm(X, W, b, 1e-5) == "layer_norm:long"


@pytest.mark.parametrize("T,N,dtype", SHAPES)
@pytest.mark.parametrize("add", [False, True])
def test_gradient(T, N, dtype, add):
    X, dO = _rand((T, N), dtype, T + N, 2.0, 0.5), _rand((T, N), dtype, T + N + 1)
    X *= (1 + torch.arange(T, device="cuda") % 5).to(dtype).view(T, 1)
    dO *= (1 + torch.arange(T, device="cuda") % 3).to(dtype).view(T, 1)
    for kind in dict.fromkeys((dtype, F32)):
        W = _rand((N,), kind, 1, 0.3, 1.0)
        for bias in (True, False):
            assert _check_norm_grad(dO, X, W, bias, 1e-5, add) == "layer_norm_grad:long"


def test_each_row_counts_once():
    """Rows of +1 and -1, whose y is that (eps 0): whole gradients are summed exactly, each row by a weight of its own."""
    T, N = 2600, 8200
    sign = torch.ones(T, N, dtype=F16, device="cuda")
    sign[:, ::2] = -1
    sign *= (1 - 2 * (torch.arange(T, device="cuda") % 3 == 0).to(F16)).view(T, 1)
    dO = (torch.arange(T, device="cuda") % 13 - 4).to(F16).view(T, 1).expand(T, N).contiguous()
    W, dX, dW, dB, O = torch.ones(N, device="cuda"), _nan((T, N), F16), _nan((N,), F32), _nan((N,), F32), _nan((T, N), F16)
    tc.tc_layer_norm(sign, W, None, O, 0.0)
    assert torch.equal(O, sign)
    tc.tc_layer_norm_grad(dO, sign, W, dX, dW, dB, _bytes(tc.tc_layer_norm_grad_workspace_bytes(T, N)), 0.0)
    assert torch.equal(dW, (dO.double() * sign.double()).sum(dim=0).float()) and torch.equal(dB, dO.double().sum(dim=0).float())
    assert np.abs(dX.float().cpu().numpy()).max() == 0  # (h equals its mean, and is nowhere along y)
