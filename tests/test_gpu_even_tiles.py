"""Products with 8-bit weights in the large tiles, over long reductions and over rows beyond 4 GB; layer norm and blocks of 8 bits of that size.  The products' reference is taken
on the GPU in float64.  Whole numbers are summed exactly (see test_gpu_even.py): no tolerance.  test_expert_q8_plan.py holds the shapes to the kernels they are meant for."""
import numpy as np
import pytest
import torch

from paper_1802_04730_amd import tc355 as tc
from test_gpu_even import E4, E8, F32, BF16, F16, _bytes, _e4, _e8, _ints, _offsets, _nan, _up, _weights8

pytestmark = pytest.mark.gpu

# side, float32, T, R, E, N, K
SHAPES = [(256, 0, 8192, 8192, 1, 8192, 3300), (256, 0, 6000, 12200, 2, 8100, 4200), (256, 0, 12200, 12200, 2, 8004, 8500), (256, 0, 16200, 16200, 1, 8321, 3300),
          (256, 0, 9000, 16200, 2, 8184, 4300), (128, 0, 2000, 4000, 5, 1016, 700), (128, 0, 4096, 4096, 1, 1025, 8450), (128, 1, 4096, 4096, 3, 2050, 900),
          (128, 1, 4000, 6000, 2, 2048, 300), (64, 0, 600, 600, 1, 1000, 8400), (64, 1, 400, 900, 7, 1333, 8321), (0, 0, 20, 16, 1, 512, 8400), (0, 1, 16, 16, 1, 500, 8321),
          (64, 0, 90, 300, 2, 1000, 1)]


def _whole(shape, seed, dtype, block):
    """Whole numbers of up to 3 bits times powers of two that differ from block to block of the last axis."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randint(-7, 8, shape, generator=g, device="cuda").float()
    p = torch.exp2(torch.randint(-2, 3, (*block, -(-shape[-1] // 128)), generator=g, device="cuda").float())
    p = p.repeat_interleave(128, -1)[..., :shape[-1]]
    return (x * (p if len(block) == 1 else p.repeat_interleave(128, -2)[:, :shape[1]])).to(dtype)


def _product(x, w, Off, Row, R):
    y = torch.zeros((R, w.shape[1]), dtype=torch.float64, device="cuda")
    for e in range(len(Off) - 1):
        rows = slice(int(Off[e]), int(Off[e + 1]))
        if Off[e] < Off[e + 1]:
            if Row is None:
                a = x[rows].double()
            else:
                r = Row[rows].long()
                a = torch.where(((r >= 0) & (r < len(x))).unsqueeze(1), x[r.clamp(0, len(x) - 1)].double(), 0.0)
            y[rows] = a @ w[e].double().t()
    return y


@pytest.mark.parametrize("dtype,T,R,E,N,K", [(F32 if s[1] else half, *s[2:]) for s in SHAPES for half in ((F32,) if s[1] else (BF16, F16))])
def test_large_tiles_and_long_reductions(dtype, T, R, E, N, K):
    rng = np.random.default_rng(R + K)
    X, W = _whole((T, K), 1, dtype, (T,)), _whole((E, N, K), 2, dtype, (E, -(-N // 128)))
    Q, S, Qt, St = _weights8(W)
    Off = _offsets(E, R, R, "some" if E > 1 else "all")
    ws = _bytes(max(tc.tc_expert_mm_q8_workspace_bytes(T, R, E, N, K), tc.tc_expert_mm_q8_workspace_bytes(R, R, E, K, N)))
    for gather, relu, gated in ((False, False, True), (True, True, False)):
        if not gather and T != R:
            continue
        Row = _ints(rng.integers(-1, T + 1, R)) if gather else None
        gate = _whole((R, N), 3, dtype, (R,)) if gated else None
        Y = _nan((R, N), dtype)
        tc.tc_expert_mm_q8(X, None, Q, S, _ints(Off) if E > 1 else None, Row, gate, Y, ws, relu)
        want = _product(X, W, Off, Row, R)
        want = torch.where(want > 0, want, 0.0) if relu else want
        want = torch.where(gate > 0, want, 0.0) if gated else want
        assert torch.equal(Y, want.float().to(dtype)), (tc.last_path(), gather)
    if R < 13000:
        dY = _whole((R, N), 4, dtype, (R,))
        dX = _nan((R, K), dtype)
        tc.tc_expert_mm_q8(dY, None, Qt, St, _ints(Off), None, None, dX, ws)
        assert torch.equal(dX, _product(dY, W.transpose(1, 2), Off, None, R).float().to(dtype))


SHORT = [(9000, 7, 8200, 1000), (9000, 6, 8185, 300), (20000, 70, 4100, 520), (70000, 300, 1000, 650)]  # R, E, N, K


def _odd_shares(R, E, seed):
    """Offsets that leave last row tiles of a tile of 256 of every kind, rows before the first expert and behind the last."""
    rng = np.random.default_rng(seed)
    rest, off = rng.permutation(np.resize([1, 128, 0, 129, 256, 127, 255], E)), [3]
    for i, r in enumerate(rest):
        spare = (R - 40 - off[-1] - int(rest[i:].sum())) // 256
        off.append(off[-1] + int(r) + 256 * (min(spare, int(rng.integers(0, 2 * (R // 256) // E + 1))) if r or i % 2 else 0))
    assert off[-1] < R - 30
    return np.array(off)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("R,E,N,K", SHORT)
def test_last_row_tiles_of_every_kind(dtype, R, E, N, K):
    rng = np.random.default_rng(R + K)
    T = R // 2
    X, W = _whole((T, K), 1, dtype, (T,)), _whole((E, N, K), 2, dtype, (E, -(-N // 128)))
    Q, S, _, _ = _weights8(W)
    ws = _bytes(tc.tc_expert_mm_q8_workspace_bytes(T, R, E, N, K))
    Row, gate = _ints(rng.integers(-1, T + 1, R)), _whole((R, N), 3, dtype, (R,))
    for seed, gated in ((1, False), (2, True)):
        Off = _odd_shares(R, E, seed)
        Y = _nan((R, N), dtype)
        tc.tc_expert_mm_q8(X, None, Q, S, _ints(Off), Row, gate if gated else None, Y, ws)
        want = _product(X, W, Off, Row, R)
        want = torch.where(gate > 0, want, 0.0) if gated else want
        assert torch.equal(Y[Off[0]:], want[Off[0]:].float().to(dtype))
        assert bool(Y[:Off[0]].isnan().all())
    for off in (np.full(E + 1, 0), np.full(E + 1, R), np.r_[np.zeros(E), R], np.r_[0, np.full(E, R)], np.r_[np.linspace(R, 0, E), 2 ** 31 - 1], np.r_[-5, rng.integers(-R, 2 * R, E)]):
        big = torch.full((R + 64, N), 7.0, dtype=dtype, device="cuda")
        tc.tc_expert_mm_q8(X, None, Q, S, _ints(np.asarray(off, np.int64).clip(-2 ** 31, 2 ** 31 - 1)), Row, None, big[:R], ws)
        reached = np.maximum.accumulate(np.clip(off, 0, R)).astype(np.int64)
        want = _product(X, W, reached, Row, R)
        assert torch.equal(big[reached[0]:R], want[reached[0]:].float().to(dtype)) and bool((big[R:] == 7.0).all()) and bool((big[:reached[0]] == 7.0).all())


def test_a_layer_of_experts_in_large_tiles_is_the_same_each_time():
    """No wait between stages may be missing: the same bits over many calls, between calls of other sizes."""
    T, E, N, K = 8192, 1, 8192, 3300
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    X = torch.randn((T, K), generator=g, device="cuda").to(BF16)
    Q, S, _, _ = _weights8(torch.randn((E, N, K), generator=g, device="cuda").to(BF16))
    ws = _bytes(tc.tc_expert_mm_q8_workspace_bytes(T, T, E, N, K))
    Y, Z = _nan((T, N), BF16), _nan((300, N), BF16)
    tc.tc_expert_mm_q8(X, None, Q, S, None, None, None, Y, ws)
    first, small = Y.clone(), None
    for _ in range(12):
        Y.fill_(float("nan"))
        tc.tc_expert_mm_q8(X[:300].contiguous(), None, Q, S, None, None, None, Z, ws)
        tc.tc_expert_mm_q8(X, None, Q, S, None, None, None, Y, ws)
        assert torch.equal(Y, first)
        small = Z.clone() if small is None else small
        assert torch.equal(Z, small)


def test_rows_beyond_4_gb():
    """Rows in 8 bits and in 16, and outputs, whose offsets pass 32 bits."""
    T, K, N = (1 << 20) + 7, 4224, 8
    at = torch.tensor([0, 5, 1 << 19, (1 << 20) + 6, 1 << 20, -1, T], device="cuda")
    X = torch.zeros((T, K), dtype=BF16, device="cuda")
    rows = _whole((5, K), 1, BF16, (5,))
    X[at[:5]] = rows
    W = _whole((1, N, K), 2, BF16, (1, 1))
    Q, S, _, _ = _weights8(W)
    want = torch.zeros((7, N), device="cuda", dtype=torch.float64)
    want[:5] = rows.double() @ W[0].double().t()
    want = want.float().to(BF16)
    Y = _nan((7, N), BF16)
    ws = _bytes(tc.tc_expert_mm_q8_workspace_bytes(T, 7, 1, N, K))
    tc.tc_expert_mm_q8(X, None, Q, S, None, at.int(), None, Y, ws)
    assert torch.equal(Y, want)
    Xq, Xs = _e4(T, K), _e8(T, K // 128)
    tc.tc_quantize_rows(X, Xq, Xs)
    Y.fill_(float("nan"))
    tc.tc_expert_mm_q8(Xq, Xs, Q, S, None, at.int(), None, Y)
    assert torch.equal(Y, want)
    del X, ws
    everything = _nan((T, N), BF16)  # all rows, in tiles
    tc.tc_expert_mm_q8(Xq, Xs, Q, S, None, None, None, everything)
    assert torch.equal(everything[at[:5]], want[:5])
    everything[at[:5]] = 0
    assert not bool(everything.any())


def test_weights_beyond_2_31_elements():
    E, N, K = 33, 8192, 8200  # 2.2e9
    W = torch.zeros((E, N, K), dtype=BF16, device="cuda")
    W[E - 1] = _whole((1, N, K), 3, BF16, (1, N // 128))[0]
    Q, S, Qt, St = _weights8(W)
    X = _whole((70, K), 4, BF16, (70,))
    off = [0] * E + [70]
    Y = _nan((70, N), BF16)
    tc.tc_expert_mm_q8(X, None, Q, S, _ints(off), None, None, Y, _bytes(tc.tc_expert_mm_q8_workspace_bytes(70, 70, E, N, K)))
    assert torch.equal(Y, (X.double() @ W[E - 1].double().t()).float().to(BF16))
    assert torch.equal(Qt.view(torch.uint8)[E - 1, :, :N], Q.view(torch.uint8)[E - 1, :, :K].t())
    assert torch.equal(St.view(torch.uint8), S.view(torch.uint8).transpose(1, 2))


def test_layer_norm_beyond_4_gb():
    T, N = (1 << 20) + 3, 2304
    X = torch.zeros((T, N), dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    at = torch.tensor([0, 1 << 19, T - 1], device="cuda")
    X[at] = torch.randn((3, N), generator=g, device="cuda").to(BF16)
    W, B = torch.randn(N, generator=g, device="cuda"), torch.randn(N, generator=g, device="cuda")
    O = _nan((T, N), BF16)
    tc.tc_layer_norm(X, W, B, O)
    few = _nan((3, N), BF16)
    tc.tc_layer_norm(X[at].contiguous(), W, B, few)
    assert torch.equal(O[at], few) and torch.equal(O[1 << 20], B.to(BF16))
    dX, dW, dB = O, _nan((N,), F32), _nan((N,), F32)
    dO = torch.zeros((T, N), dtype=BF16, device="cuda")
    dO[at] = torch.randn((3, N), generator=g, device="cuda").to(BF16)
    tc.tc_layer_norm_grad(dO, X, W, dX, dW, dB, _bytes(tc.tc_layer_norm_grad_workspace_bytes(T, N)))
    fX, fW, fB = _nan((3, N), BF16), _nan((N,), F32), _nan((N,), F32)
    tc.tc_layer_norm_grad(dO[at].contiguous(), X[at].contiguous(), W, fX, fW, fB, _bytes(tc.tc_layer_norm_grad_workspace_bytes(3, N)))
    assert torch.equal(dX[at], fX)
    for a, b in ((dW, fW), (dB, fB)):  # sums of three terms, of which zeros take none
        assert bool(((a - b).abs() <= 2.0 ** -22 * (b.abs() + 8)).all())
    dX[at] = 0
    assert not bool(dX.any())
