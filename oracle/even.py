"""Float64 oracle of the operators around experts of even load, with weights in 8 bits (numpy, written from the formulas)."""
import numpy as np

from .experts import softmax_rows

BLOCK = 128


def layer_norm(X, W, B, eps):
    """O, y, 1/s."""
    d = X - X.mean(axis=1, keepdims=True)
    r = 1 / np.sqrt((d * d).mean(axis=1, keepdims=True) + eps)
    return d * r * W + (0 if B is None else B), d * r, r


def layer_norm_grad(dO, X, W, eps):
    """dX, dW, dB."""
    _, y, r = layer_norm(X, W, None, eps)
    h = dO * W
    return (h - h.mean(axis=1, keepdims=True) - y * (h * y).mean(axis=1, keepdims=True)) * r, (dO * y).sum(axis=0), dO.sum(axis=0)


def scores(L, sigmoid):
    if not sigmoid:
        return softmax_rows(L)
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-L))


def route_balanced(L, Bias, k, groups, keep, sigmoid, norm, scale):
    """Wt, Id, Off, Row, Place."""
    T, E = L.shape
    S = scores(L, sigmoid)
    C = np.where(L == -np.inf, -np.inf, S + (0 if Bias is None else Bias))
    size = E // groups
    Wt, Id = np.zeros((T, k)), np.full((T, k), -1, np.int64)
    first = lambda values, numbers: sorted(numbers, key=lambda e: (not np.isnan(values[e]), 0.0 if np.isnan(values[e]) else -values[e], e))  # noqa: E731
    for t in range(T):
        group = np.empty(groups)
        for g in range(groups):
            best = [C[t, e] for e in first(C[t], range(g * size, (g + 1) * size)) if C[t, e] != -np.inf][:2]
            group[g] = sum(best) if best else -np.inf
        kept = first(group, range(groups))[:keep]
        order = first(C[t], [e for g in kept for e in range(g * size, (g + 1) * size) if C[t, e] != -np.inf])[:k]
        Id[t, :len(order)] = order
        w = S[t, order]
        Wt[t, :len(order)] = scale * w / (max(w.sum(), 1e-300) if norm and not np.isnan(w.sum()) else w.sum() if norm else 1.0)
    return (Wt, Id, *places(Id, E))


def places(Id, E):
    """Off, Row, Place: the slots by expert, those of one expert in their order."""
    T, k = Id.shape
    key = np.where(Id < 0, E, Id).ravel()
    order = np.argsort(key, kind="stable")
    Off = np.concatenate([[0], np.cumsum(np.bincount(key, minlength=E + 1)[:E])])
    there = np.arange(T * k) < Off[E]
    Place = np.empty(T * k, np.int64)
    Place[order] = np.where(there, np.arange(T * k), -1)
    return Off, np.where(there, order // k, -1), Place.reshape(T, k)


def route_balanced_grad(L, Id, dWt, sigmoid, norm, scale):
    T, E = L.shape
    S = scores(L, sigmoid)
    dL = np.zeros((T, E))
    for t in range(T):
        at = [i for i in range(Id.shape[1]) if 0 <= Id[t, i] < E and L[t, Id[t, i]] != -np.inf]
        ids = Id[t, at]
        g, s = dWt[t, at], S[t, ids]
        total = max(s.sum(), 1e-300)
        ds = np.zeros(E)
        ds[ids] = scale * ((g - (g * s).sum() / total) / total if norm else g)
        dL[t] = ds * S[t] * (1 - S[t]) if sigmoid else S[t] * (ds - (ds * S[t]).sum())
    return np.where(L == -np.inf, 0.0, dL)


def _up(n):
    return -(-n // BLOCK) * BLOCK


def _quantize(blocks):
    """Blocks along the last axis: their values in e4m3 and the scales' bytes."""
    most = np.abs(blocks).max(axis=-1, keepdims=True)
    bad = ~np.isfinite(most)
    byte = np.ones(most.shape, np.int64)
    for b in range(2, 248):
        byte = np.where(most > 448 * 2.0 ** (b - 1 - 127), b, byte)
    with np.errstate(invalid="ignore", over="ignore"):
        v = np.where(bad, 0, blocks) / 2.0 ** (byte - 127.0)
        step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6))) - 3)
        q = np.rint(v / step) * step
    return np.where(bad, np.nan, q), np.where(bad, 255, byte)[..., 0]


def quantize_rows(X):
    """Q [R, K'], S [R, K'/128]."""
    R, K = X.shape
    x = np.zeros((R, _up(K)))
    x[:, :K] = X
    q, s = _quantize(x.reshape(R, -1, BLOCK))
    return q.reshape(R, -1), s


def quantize_weights(W):
    """Q [E, N, K'], S, Qt [E, K, N'], St."""
    E, N, K = W.shape
    n, k = _up(N) // BLOCK, _up(K) // BLOCK
    w = np.zeros((E, n * BLOCK, k * BLOCK))
    w[:, :N, :K] = W
    q, s = _quantize(w.reshape(E, n, BLOCK, k, BLOCK).transpose(0, 1, 3, 2, 4).reshape(E, n, k, BLOCK * BLOCK))
    q = q.reshape(E, n, k, BLOCK, BLOCK).transpose(0, 1, 3, 2, 4).reshape(E, n * BLOCK, k * BLOCK)
    return q[:, :N], s, q[:, :, :K].transpose(0, 2, 1).copy(), s.transpose(0, 2, 1).copy()


def values(Q, S):
    """What rows in 8 bits stand for; S along the last axis, and along the one before where it has fewer."""
    if S.ndim == 3:
        S = np.repeat(S, BLOCK, axis=1)[:, :Q.shape[1]]
    with np.errstate(invalid="ignore"):
        scale = np.where(S == 255, np.nan, 2.0 ** (S.astype(np.float64) - 127))
        return Q * np.repeat(scale, BLOCK, axis=-1)


def product(X, W, Off, Row, R, relu):
    """oracle.experts.expert_mm by one matrix product an expert, for offsets that go up: Y and the sums of its terms' magnitudes."""
    x = X
    if Row is not None:
        ok = (Row >= 0) & (Row < len(X))
        x = np.where(ok[:, None], X[np.where(ok, Row, 0)], 0.0)
    Y, mag = np.zeros((R, W.shape[1])), np.zeros((R, W.shape[1]))
    for e in range(len(Off) - 1):
        rows = slice(Off[e], Off[e + 1])
        Y[rows], mag[rows] = x[rows] @ W[e].T, np.abs(x[rows]) @ np.abs(W[e]).T
    return (np.where(Y > 0, Y, 0.0) if relu else Y), mag
