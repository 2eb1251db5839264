"""Plain 64-bit forms (numpy) of the gated linear recurrence, the gated
feed-forward product and the 4-bit product, written from their definitions;
used by the tests of the three."""
import numpy as np


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1 / (1 + e), e / (1 + e))


def recurrence(g, h0, lengths):
    """g [T,B,2H], h0 [B,H], lengths [B] -> h [T,B,H] (0 in padding), last [B,H]."""
    T, B, H2 = g.shape
    H = H2 // 2
    h, out = h0.astype(np.float64).copy(), np.zeros((T, B, H))
    for t in range(T):
        on = lengths > t
        z, n = sigmoid(g[t, on, :H]), g[t, on, H:]
        h[on] = z * h[on] + sigmoid(-g[t, on, :H]) * n
        out[t, on] = h[on]
    return out, h


def recurrence_backward(g, h0, lengths, h_out, dh_out, dh_last):
    T, B, H2 = g.shape
    H = H2 // 2
    dg, e = np.zeros((T, B, H2)), dh_last.astype(np.float64).copy()
    for t in range(T - 1, -1, -1):
        on = lengths > t
        z, r, n = sigmoid(g[t, on, :H]), sigmoid(-g[t, on, :H]), g[t, on, H:]
        before = h_out[t - 1, on] if t else h0[on]
        d = dh_out[t, on] + e[on]
        dg[t, on, :H] = d * (before - n) * z * r
        dg[t, on, H:] = d * r
        e[on] = z * d
    return dg, e


_erf = np.vectorize(__import__("math").erf, otypes=[np.float64])


def act(a, kind):
    if kind == "relu":
        return np.maximum(a, 0), (a > 0).astype(np.float64)
    if kind == "gelu":
        p = 0.5 * (1 + _erf(a / np.sqrt(2)))
        return a * p, p + a * np.exp(-a * a / 2) / np.sqrt(2 * np.pi)
    s = sigmoid(a)
    if kind == "sigmoid":
        return s, s * (1 - s)
    return a * s, s * (1 + a * (1 - s))


def glu(x, W, kind):
    F = W.shape[0] // 2
    return act(x @ W[:F].T, kind)[0] * (x @ W[F:].T)


def glu_backward(x, W, dh, kind):
    """dx, dW and d = [dh u act'(g) | dh act(g)]."""
    F = W.shape[0] // 2
    a, da = act(x @ W[:F].T, kind)
    d = np.concatenate([dh * (x @ W[F:].T) * da, dh * a], axis=1)
    return d @ W, d.T @ x, d


def dequantised(q, scales, group):
    """q [N,K] in 0..15, scales [N,ceil(K/group)]."""
    return (q.astype(np.float64) - 8) * np.repeat(scales, group, axis=1)[:, : q.shape[1]]


def pack_rows(q):
    """[N,K] codes -> [N,K/2] bytes, the even k in the low half."""
    return (q[:, 0::2] | (q[:, 1::2] << 4)).astype(np.uint8)


def tiled_word(q, nb, kb, half, r, t, j):
    """The 32-bit word of the tiled order, from its documented formula."""
    w = 0
    for i, e in enumerate((0, 2, 4, 6, 1, 3, 5, 7)):
        n, k = 16 * nb + 8 * half + r, 128 * kb + 32 * j + 8 * t + e
        c = int(q[n, k]) if n < q.shape[0] and k < q.shape[1] else 8
        w |= c << (4 * i)
    return w
