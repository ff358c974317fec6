"""Pins of the float64 oracle of the operators around experts of even load: against torch's own on the CPU, and by hand."""
import numpy as np
import torch

from oracle import even as ref
from oracle import experts


def test_layer_norm_and_its_gradient():
    rng = np.random.default_rng(1)
    X, W, B, dO = rng.standard_normal((7, 13)), rng.standard_normal(13), rng.standard_normal(13), rng.standard_normal((7, 13))
    x, w, b = (torch.from_numpy(a).requires_grad_() for a in (X, W, B))
    o = torch.nn.functional.layer_norm(x, (13,), w, b, 1e-3)
    o.backward(torch.from_numpy(dO))
    assert np.allclose(ref.layer_norm(X, W, B, 1e-3)[0], o.detach().numpy(), atol=1e-13)
    for got, want in zip(ref.layer_norm_grad(dO, X, W, 1e-3), (x, w, b)):
        assert np.allclose(got, want.grad.numpy(), atol=1e-12)


def test_router_without_groups_or_bias_is_the_plain_one():
    L = np.random.default_rng(2).standard_normal((20, 9))
    L[3, 2:] = -np.inf
    for norm in (False, True):
        for a, b in zip(ref.route_balanced(L, None, 4, 1, 1, False, norm, 1.0), experts.route(L, 4, norm)):
            assert np.allclose(a, b)
        Id, dWt = experts.route(L, 4, norm)[1], np.random.default_rng(3).standard_normal((20, 4))
        assert np.allclose(ref.route_balanced_grad(L, Id, dWt, False, norm, 1.0), experts.route_grad(L, Id, dWt, norm))


def test_router_with_groups_by_hand():
    L = np.zeros((1, 6))
    Bias = np.array([0.0, 0.3, 0.2, 0.2, 0.5, -1.0])  # scores of the groups of two: 1 + 0.3, 1 + 0.4, 1 - 0.5
    Wt, Id, Off, Row, Place = ref.route_balanced(L, Bias, 3, 3, 1, True, True, 2.0)
    assert Id.tolist() == [[2, 3, -1]] and Wt.tolist() == [[1.0, 1.0, 0.0]]
    assert Off.tolist() == [0, 0, 0, 1, 2, 2, 2] and Row.tolist() == [0, 0, -1] and Place.tolist() == [[0, 1, -1]]
    assert ref.route_balanced(L, Bias, 3, 3, 2, True, True, 2.0)[1].tolist() == [[1, 2, 3]]
    assert ref.route_balanced(L, Bias, 3, 1, 1, True, True, 2.0)[1].tolist() == [[4, 1, 2]]


def test_blocks_of_8_bits_round_as_torch_does():
    rng = np.random.default_rng(4)
    X = (rng.standard_normal((40, 300)) * np.exp(2 * rng.standard_normal((40, 300)))).astype(np.float32).astype(np.float64)
    Q, S = ref.quantize_rows(X)
    scale = 2.0 ** (np.repeat(S, 128, axis=1) - 127.0)
    x = np.zeros((40, 384))
    x[:, :300] = X
    want = torch.from_numpy(x / scale).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(Q, want)
    most = np.abs(x.reshape(40, 3, 128)).max(-1) / 2.0 ** (S - 127.0)
    assert (most <= 448).all() and (most > 224).all()
    assert (np.abs(ref.values(Q, S) - x) <= np.maximum(2.0 ** -4 * np.abs(x), scale * 2.0 ** -10)).all()


def test_scales_at_the_border_by_hand():
    X = np.zeros((5, 128))
    X[0, 3], X[1, 3], X[2, 3], X[3, 3] = 448, 449, 1e-45, np.inf
    assert ref.quantize_rows(X)[1][:, 0].tolist() == [127, 128, 1, 255, 1]


def test_transposed_weights_stand_for_the_same():
    W = np.random.default_rng(5).standard_normal((2, 150, 260))
    Q, S, Qt, St = ref.quantize_weights(W)
    assert np.array_equal(ref.values(Q, S)[:, :, :260], ref.values(Qt, St)[:, :, :150].transpose(0, 2, 1))


def test_product_is_the_plain_one():
    rng = np.random.default_rng(6)
    X, W, Off, Row = rng.standard_normal((5, 7)), rng.standard_normal((3, 4, 7)), np.array([0, 4, 4, 9]), rng.integers(-1, 6, 11)
    for relu in (False, True):
        for a, b in zip(ref.product(X, W, Off, Row, 11, relu), experts.expert_mm(X, W, Off, Row, 11, relu)):
            assert np.allclose(a, b)
