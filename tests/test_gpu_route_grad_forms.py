"""The router's gradient in every form that the number of experts picks, each column against the size of its own terms.

dL(t,e) = [e chosen as i] w_i g_i - S_e sum_j g_j w_j.  In steps of u = 2^-24: a logit's distance from the largest is rounded once and is at most some 16
here, so that an exponential is off by 16 u and its own 4 u; a sum over at most 16 neighbours of a lane and 6 exchanges by 22 u; a quotient by 2 u: a weight or a
share by less than 48 u.  The inner sum adds 48 u of the sum of |g_j w_j| for the weights and 22 u for its own additions, and the difference 2 u.  So a result is off by less than
128 u (|w_i g_i| + S_e sum_j |g_j w_j|), and by its rounding: columns that were not chosen, where the second term is all there is, are held to it too."""
import numpy as np
import pytest
import torch

from oracle import experts as ref
from paper_1802_04730_amd import tc355 as tc
from test_gpu_experts import STEP, TYPES, UNIT, _logits, _np, _rand, _route

pytestmark = pytest.mark.gpu

# T, E, k: lanes of 16 with 1, 2, 4, 8 logits each, of 64 with 4, 8, 16; ends and beginnings of each, whole and partial last lanes
SHAPES = [(40, 16, 3), (37, 17, 2), (40, 32, 5), (19, 33, 8), (50, 64, 6), (33, 65, 4), (21, 100, 8), (70, 128, 8), (25, 127, 16), (9, 128, 40), (23, 129, 8), (21, 256, 8), (17, 257, 12),
          (18, 300, 64), (11, 512, 10), (9, 513, 10), (7, 1023, 33), (5, 1000, 1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("T,E,k", SHAPES)
def test_every_form(dtype, norm, T, E, k):
    L = _logits(T, E, dtype, T * E + 1)
    Id, dWt = _route(L, k, norm)[1], _rand((T, k), torch.float32, 9)
    dL = torch.full((T, E), float("nan"), dtype=dtype, device="cuda")
    tc.tc_route_grad(L, Id, dWt, dL, norm)
    l, ids, g = _np(L), _np(Id), _np(dWt)
    want = ref.route_grad(l, ids, g, norm)
    # the terms' sizes
    share, size = ref.softmax_rows(l), np.zeros((T, E))
    for t in range(T):
        on = ids[t] >= 0
        chosen = ids[t][on]
        if not len(chosen):
            continue
        w = ref.softmax_rows(l[t:t + 1, chosen])[0] if norm else share[t, chosen]
        second = np.zeros(E) if norm else share[t].copy()
        second[chosen] = w
        size[t] = second * np.abs(g[t][on] * w).sum()
        size[t, chosen] += np.abs(g[t][on] * w)
    assert (np.abs(_np(dL) - want) <= UNIT[dtype] * np.abs(want) + 2.0 ** -17 * size + STEP[dtype]).all()
    # what such a bound is good for: without the second term it would be missed in most columns that were not chosen
    if not norm and dtype is torch.float32 and E >= 100 and k > 1:
        other = share > 0
        np.put_along_axis(other, np.maximum(ids, 0), False, 1)  # (an empty slot's stands for expert 0)
        assert (np.abs(want) > UNIT[dtype] * np.abs(want) + 2.0 ** -17 * size + STEP[dtype])[other].mean() > 0.9
