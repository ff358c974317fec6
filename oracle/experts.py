"""Float64 oracle of the operators around experts (numpy, loops over tokens or experts, written from the formulas).

Where a result is a sum, ``*_mag`` is the sum of its terms' magnitudes: what the error bound of a sum is stated in.
"""
import numpy as np


def embed(LUT, Idx, scale):
    E = LUT.shape[0]
    O = np.full((len(Idx), LUT.shape[1]), np.nan)
    ok = (Idx >= 0) & (Idx < E)
    O[ok] = LUT[Idx[ok]] * scale
    return O


def embed_grad(dO, Idx, E, scale, pad, there=None):
    total, mag = np.zeros((E, dO.shape[1])), np.zeros((E, dO.shape[1]))
    for t, e in enumerate(Idx):
        if 0 <= e < E and e != pad:
            total[e] += scale * dO[t]
            mag[e] += np.abs(scale * dO[t])
    if there is not None:
        total, mag = total + there, mag + np.abs(there)
    return total, mag


def softmax_rows(L):
    """Rows of nothing but -inf give zeros."""
    with np.errstate(invalid="ignore", over="ignore"):
        most = np.fmax.reduce(L, axis=1, keepdims=True)
        most = np.where(most == -np.inf, 0.0, most)
        p = np.exp(L - most)
        return p / np.where((p == 0).all(axis=1, keepdims=True), 1.0, p.sum(axis=1, keepdims=True))


def route(L, k, norm):
    """Wt, Id, Off, Row, Place."""
    T, E = L.shape
    share = softmax_rows(L)
    Wt, Id = np.zeros((T, k)), np.full((T, k), -1, np.int64)
    for t in range(T):
        # NaN first, then by size, equal ones by number; -inf never
        order = sorted((e for e in range(E) if L[t, e] != -np.inf), key=lambda e: (not np.isnan(L[t, e]), 0.0 if np.isnan(L[t, e]) else -L[t, e], e))
        n = min(k, len(order))
        Id[t, :n] = order[:n]
        Wt[t, :n] = share[t, order[:n]]
        if norm and n:
            Wt[t, :n] = softmax_rows(L[t:t + 1, order[:n]])[0]
    Off, Row, Place = np.zeros(E + 1, np.int64), np.full(T * k, -1, np.int64), np.full((T, k), -1, np.int64)
    at = 0
    for e in range(E):
        Off[e] = at
        for t, i in zip(*np.nonzero(Id == e)):
            Row[at], Place[t, i] = t, at
            at += 1
    Off[E] = at
    return Wt, Id, Off, Row, Place


def route_grad(L, Id, dWt, norm):
    T, E = L.shape
    dL = np.zeros((T, E))
    share = softmax_rows(L)
    for t in range(T):
        on = Id[t] >= 0
        ids, g = Id[t][on], dWt[t][on]
        if not len(ids):
            continue
        if norm:
            w = softmax_rows(L[t:t + 1, ids])[0]
            dL[t, ids] = w * (g - (g * w).sum())
        else:
            w = share[t, ids]
            dL[t] = -share[t] * (g * w).sum()
            dL[t, ids] += w * g
    return dL


def _source(X, Row, r):
    if Row is None:
        return X[r]
    return X[Row[r]] if 0 <= Row[r] < len(X) else np.zeros(X.shape[1])


def _experts(Off, R):
    """(expert, its rows): offsets clamped to [0, R], and from where they decrease on as they were, so that no row has two experts."""
    at = np.maximum.accumulate(np.clip(Off, 0, R))
    return [(e, range(at[e], at[e + 1])) for e in range(len(Off) - 1)]


def expert_mm(X, W, Off, Row, R, relu):
    Y, mag = np.zeros((R, W.shape[1])), np.zeros((R, W.shape[1]))
    for e, rows in _experts(Off, R):
        for r in rows:
            x = _source(X, Row, r)
            Y[r], mag[r] = W[e] @ x, np.abs(W[e]) @ np.abs(x)
    return (np.where(Y > 0, Y, 0.0) if relu else Y), mag


def expert_mm_grad_x(dY, W, Off, gate):
    R = len(dY)
    dX, mag = np.zeros((R, W.shape[2])), np.zeros((R, W.shape[2]))
    for e, rows in _experts(Off, R):
        for r in rows:
            dX[r], mag[r] = dY[r] @ W[e], np.abs(dY[r]) @ np.abs(W[e])
            if gate is not None:
                dX[r] = np.where(gate[r] > 0, dX[r], 0.0)
    return dX, mag


def expert_mm_grad_w(dY, X, Off, Row, there=None):
    R, N = dY.shape
    E, K = len(Off) - 1, X.shape[1]
    dW, mag = np.zeros((E, N, K)), np.zeros((E, N, K))
    for e, rows in _experts(Off, R):
        for r in rows:
            x = _source(X, Row, r)
            dW[e] += np.outer(dY[r], x)
            mag[e] += np.abs(np.outer(dY[r], x))
    if there is not None:
        dW, mag = dW + there, mag + np.abs(there)
    return dW, mag


def expert_sum(Y, Wt, Place):
    T, k = Place.shape
    O, mag = np.zeros((T, Y.shape[1])), np.zeros((T, Y.shape[1]))
    for t in range(T):
        for i in range(k):
            if 0 <= Place[t, i] < len(Y):
                term = (1.0 if Wt is None else Wt[t, i]) * Y[Place[t, i]]
                O[t] += term
                mag[t] += np.abs(term)
    return O, mag


def expert_sum_grad(dO, Y, Wt, Place, dY):
    """dY (rows of no place stay as they are), dWt, the magnitude of dWt."""
    dY, dWt, mag = dY.copy(), np.zeros(Place.shape), np.zeros(Place.shape)
    for t, i in np.ndindex(*Place.shape):
        r = Place[t, i]
        if 0 <= r < len(Y):
            dY[r] = Wt[t, i] * dO[t]
            dWt[t, i], mag[t, i] = dO[t] @ Y[r], np.abs(dO[t]) @ np.abs(Y[r])
    return dY, dWt, mag
