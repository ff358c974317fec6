"""The binding's native calls of the operators around experts of even load: the same call as by the general path, and -1 for what is not right."""
import numpy as np
import pytest
import torch

from paper_1802_04730_amd import tc355 as tc


def _calls(dev, dtype=torch.bfloat16):
    """(name, arguments, outputs), small."""
    g = torch.Generator().manual_seed(1)
    f = lambda *s, t=dtype: torch.randn(s, generator=g).to(t).to(dev)  # noqa: E731
    e = lambda *s, t=dtype: torch.full(s, float("nan"), dtype=t, device=dev)  # noqa: E731
    i = lambda a: torch.tensor(a, dtype=torch.int32, device=dev)  # noqa: E731
    f32, z = torch.float32, lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)  # noqa: E731
    q8 = lambda *s: torch.randint(0, 120, s, generator=g, dtype=torch.uint8).to(dev).view(torch.float8_e4m3fn)  # noqa: E731
    s8 = lambda *s: torch.randint(120, 130, s, generator=g, dtype=torch.uint8).to(dev).view(torch.float8_e8m0fnu)  # noqa: E731
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=dev)
    for t in (dtype, f32):
        for b in (None, f(8, t=t)):
            O = e(3, 8)
            yield "tc_layer_norm", [f(3, 8), f(8, t=t), b, O, 1e-5], [O]
        for bias in (False, True):
            dX, dW, dB = e(3, 8), e(8, t=t), e(8, t=t) if bias else None
            yield "tc_layer_norm_grad", [f(3, 8), f(3, 8), f(8, t=t), dX, dW, dB, ws, 1e-5, False], [dX, dW] + ([dB] if bias else [])
    dX = e(3, 8)
    yield "tc_layer_norm_grad", [f(3, 8), f(3, 8), f(8), dX, None, None, None, 1, False], [dX]
    for bias in (None, f(4, t=f32)):
        out = [e(3, 2, t=f32), z(3, 2), z(5), z(6), z(3, 2)]
        yield "tc_route_balanced", [f(3, 4), bias, *out, None, 2, 1, True, False, 2.5], out
    dL = e(3, 4)
    yield "tc_route_balanced_grad", [f(3, 4), i([[0, 1], [2, 3], [1, -1]]), f(3, 2, t=f32), dL, False, True, 1.0], [dL]
    Q, S = q8(3, 256), s8(3, 2)
    yield "tc_quantize_rows", [f(3, 130), Q, S], [Q, S]
    for both in (True, False):
        out = [q8(2, 9, 256), s8(2, 1, 2)] + ([q8(2, 130, 128), s8(2, 2, 1)] if both else [None, None])
        yield "tc_quantize_weights", [f(2, 9, 130), *out], [o for o in out if o is not None]
    for x, sx in ((f(6, 130), None), (q8(6, 256), s8(6, 2))):
        for row, gate in ((None, f(6, 9)), (i([0, 2, 1, 5, 2, -1]), None)):
            Y = e(6, 9)
            yield "tc_expert_mm_q8", [x, sx, q8(3, 9, 256), s8(3, 1, 2), i([0, 2, 2, 5]), row, gate, Y, ws, True], [Y]
    Y = e(6, 9)
    yield "tc_expert_mm_q8", [f(6, 130), None, q8(1, 9, 256), s8(1, 1, 2), None, None, None, Y, ws, False], [Y]


def _fast(name):
    return getattr(tc._FAST, name[3:])


def test_what_is_not_on_a_gpu_is_left_to_the_general_path():
    tc.lib()
    for name, args, _ in _calls("cpu"):
        assert _fast(name)(0, *args, None) == -1  # (entry 0: a call would crash)
        with pytest.raises((TypeError, ValueError)):
            getattr(tc, name)(*args)
        for bad in (3, "x", [], [None], object()):
            assert _fast(name)(0, *[bad] * len(args), None) == -1
        assert _fast(name)(0) == -1 and _fast(name)() == -1


def _bits(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_the_same_results_by_both_ways(monkeypatch, dtype):
    tc.lib()
    ways = []
    for fast in (tc._FAST, None):
        monkeypatch.setattr(tc, "_FAST", fast)
        got = []
        for name, args, outs in _calls("cuda", dtype):
            if fast is not None:
                assert _fast(name)(tc._AT[name], *args, None) == 0, name
            getattr(tc, name)(*args)
            getattr(tc, name)(*args, stream=torch.cuda.current_stream().cuda_stream)
            got += [_bits(o).clone() for o in outs]
        ways.append(got)
    assert all(torch.equal(a, b) and not bool(a.isnan().any()) for a, b in zip(*ways))


@pytest.mark.gpu
def test_wrong_arguments_are_left_to_the_general_path():
    tc.lib()
    for name, args, _ in _calls("cuda"):
        for j, a in enumerate(args):
            if not isinstance(a, torch.Tensor) or a.shape == (1 << 16,):
                continue
            b = _bits(a)
            bads = [a.cpu(), a.unsqueeze(0), b.repeat([2] * a.dim()).view(a.dtype), b.repeat([3] + [1] * (a.dim() - 1)).view(a.dtype)[:, ..., :-1] if a.dim() > 1 else b.double()]
            bads += [b.t().view(a.dtype) if a.dim() == 2 else b.double(), b.to(torch.int16)]
            for bad in bads:
                changed = list(args)
                changed[j] = bad
                with pytest.raises((TypeError, ValueError, tc.TcError)):
                    getattr(tc, name)(*changed)


@pytest.mark.gpu
def test_a_python_number_of_any_kind():
    X, W, O, P = torch.randn(4, 8, device="cuda"), torch.ones(8, device="cuda"), torch.empty(4, 8, device="cuda"), torch.empty(4, 8, device="cuda")
    tc.tc_layer_norm(X, W, None, P, 2.0)
    for eps in (2, 2.0, np.float64(2.0), np.float32(2.0)):
        tc.tc_layer_norm(X, W, None, O, eps)
        assert torch.equal(O, P)
