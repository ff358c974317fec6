"""The binding's native calls of the operators around experts: the same call as by the general path, and -1 for what is not right."""
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
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=dev)
    idx, off, row, place = i([1, 4, 1]), i([0, 2, 2, 5]), i([0, 2, 1, 0, 2, -1]), i([[0, 3], [2, -1], [1, 4]])
    O = e(3, 8)
    yield "tc_embed", [f(5, 8), idx, O, 2.0], [O]
    for t in (dtype, f32):
        G = e(5, 8, t=t)
        yield "tc_embed_grad", [f(3, 8), idx, G, ws, 0.5, -1, False], [G]
    out = [e(3, 2, t=f32), z(3, 2), z(5), z(6), z(3, 2)]
    yield "tc_route", [f(3, 4), *out, None, True], out
    dL = e(3, 4)
    yield "tc_route_grad", [f(3, 4), i([[0, 1], [2, 3], [1, -1]]), f(3, 2, t=f32), dL, False], [dL]
    for r, x in ((row, f(3, 8)), (None, f(6, 8))):
        Y = e(6, 4)
        yield "tc_expert_mm", [x, f(3, 4, 8), off, r, Y, True], [Y]
        for t, w in ((dtype, ws), (f32, None)):
            dW = e(3, 4, 8, t=t)
            yield "tc_expert_mm_grad_w", [f(6, 4), x, off, r, dW, w, False], [dW]
    for gate in (None, f(6, 8)):
        dX = e(6, 8)
        yield "tc_expert_mm_grad_x", [f(6, 4), f(3, 4, 8), off, gate, dX], [dX]
    for w in (None, f(3, 2, t=f32)):
        O = e(3, 8)
        yield "tc_expert_sum", [f(6, 8), w, place, O], [O]
    dY, dWt = torch.zeros((6, 8), dtype=dtype, device=dev), e(3, 2, t=f32)
    yield "tc_expert_sum_grad", [f(3, 8), f(6, 8), f(3, 2, t=f32), place, dY, dWt], [dY, dWt]


def _fast(name):
    return getattr(tc._FAST, name[3:])


def test_what_is_not_on_a_gpu_is_left_to_the_general_path():
    tc.lib()
    for name, args, _ in _calls("cpu"):
        assert _fast(name)(0, *args, None) == -1  # (entry 0: a call would crash)
        with pytest.raises((TypeError, ValueError)):
            getattr(tc, name)(*args)
        for bad in (None, 3, "x", [], [None], object()):
            assert _fast(name)(0, *[bad] * len(args), None) == -1
        assert _fast(name)(0) == -1 and _fast(name)() == -1


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
            got += [o.clone() for o in outs]
        ways.append(got)
    assert all(torch.equal(a, b) and not bool(a.isnan().any()) for a, b in zip(*ways))


@pytest.mark.gpu
def test_wrong_arguments_are_left_to_the_general_path():
    tc.lib()
    for name, args, _ in _calls("cuda"):
        for j, a in enumerate(args):
            if not isinstance(a, torch.Tensor) or a.dtype is torch.uint8:
                continue
            for bad in (a.double(), a.cpu(), a[:0].clone() if a.shape[0] else a.double(), a.unsqueeze(0), a.repeat([2] * a.dim()), a.t() if a.dim() == 2 else a[::2]):
                if name == "tc_embed" and j in (0,) and bad.shape[-1:] == a.shape[-1:] and bad.dtype == a.dtype and bad.is_cuda and bad.dim() == a.dim():
                    continue  # (another table is as good)
                if name == "tc_embed_grad" and j == 2 and bad.dim() == 2 and bad.shape[1] == a.shape[1] and bad.dtype == a.dtype and bad.is_cuda:
                    continue
                changed = list(args)
                changed[j] = bad
                if bad.dtype == a.dtype and bad.is_cuda and bad.dim() == a.dim() and bad.is_contiguous() and bad.numel() == 0:
                    continue  # (no elements: shapes are compared below)
                with pytest.raises((TypeError, ValueError, tc.TcError)):
                    getattr(tc, name)(*changed)


@pytest.mark.gpu
def test_a_python_number_of_any_kind():
    LUT, O = torch.randn(4, 8, device="cuda"), torch.empty(2, 8, device="cuda")
    idx = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    for scale in (2, 2.0, np.float64(2.0), np.float32(2.0)):
        tc.tc_embed(LUT, idx, O, scale)
        assert torch.equal(O, LUT[[3, 0]] * 2)
