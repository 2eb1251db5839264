"""Plain 64-bit forms (numpy) of the root-mean-square norm, the causal
convolution, the selective scan and beam search's selection, written from their
definitions, with bounds of what 32-bit arithmetic may add; used by their tests."""
import numpy as np

U = 2.0 ** -24  # half a step of fp32
HALF = {"fp32": U, "bf16": 2.0 ** -8}


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1 / (1 + e), e / (1 + e))


def silu(x):
    return x * sigmoid(x)


def norm(x, res, w, eps):
    """y and r."""
    r = x if res is None else x + res
    return r / np.sqrt((r * r).mean(axis=1, keepdims=True) + eps) * w, r


def norm_backward(r, w, eps, dy, dres):
    """dx, dw, and sums of magnitudes that rounding is relative to."""
    k = 1 / np.sqrt((r * r).mean(axis=1, keepdims=True) + eps)
    n, d = r * k, w * dy
    dx = k * (d - n * (d * n).mean(axis=1, keepdims=True)) + dres
    size = k * (np.abs(d) + np.abs(n) * np.abs(d * n).mean(axis=1, keepdims=True)) + np.abs(dres)
    return dx, (dy * n).sum(axis=0), size, np.abs(dy * n).sum(axis=0)


def e4m3(byte):
    """The values of E4M3 bytes."""
    b = byte.astype(np.int64)
    s, e, m = np.where(b & 128, -1.0, 1.0), (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    return np.where((b & 127) == 127, np.nan, s * v)


def conv(x, w, bias, act, state, lengths):
    """x [T,B,C], state [B,W-1,C] -> y, new state, size (what rounding is relative to)."""
    T, B, C = x.shape
    W = w.shape[0]
    y, size, new = np.zeros((T, B, C)), np.zeros((T, B, C)), np.zeros((B, W - 1, C))
    for b in range(B):
        n = int(np.clip(lengths[b], 0, T))
        line = np.concatenate([state[b], x[:n, b]])
        for t in range(n):
            v = bias + (w * line[t: t + W]).sum(axis=0)
            y[t, b] = silu(v) if act else v
            size[t, b] = np.abs(bias) + np.abs(w * line[t: t + W]).sum(axis=0)
        new[b] = line[n:]
    return y, new, size


def conv_bound(y, size, width, act, kind):
    """Sums: width + 1 roundings of terms no larger than `size`; SiLU (slope at most 1.1) to 2^-20 of itself."""
    return 1.1 * (width + 1) * U * size + (2.0 ** -20 * np.abs(y) if act else 0) + HALF[kind] * np.abs(y) + 1e-38


def softplus(x):
    return np.maximum(x, 0) + np.log1p(np.exp(-np.abs(x)))


def scan(u, dt, dt_bias, A, B, Cm, D, z, h0, lengths, kind):
    """u, dt, z [T,b,C], A [C,N], B, Cm [T,b,N] -> y, last, and bounds of both in 32 bits.

    The bound follows each rounding: delta to (16 + 3|x|) half steps (x its
    argument: exp's own error is relative to |x|), a decay to that times its exponent and 4 more, inputs
    and sums to one a step.  A sequence that is cut in time rounds its runs' sums of delta and starts as
    well: four times the bound covers a start for each state."""
    T, b, C = u.shape
    N = A.shape[1]
    h, err = h0.copy(), np.zeros_like(h0)
    y, ey = np.zeros((T, b, C)), np.zeros((T, b, C))
    for t in range(T):
        on = lengths > t
        x = dt[t, on] + dt_bias
        delta = softplus(x)
        e_delta = (16 + 3 * (np.abs(dt[t, on]) + np.abs(dt_bias))) * U
        power = delta[..., None] * A
        a = np.exp(power)
        e_a = np.abs(power) * (e_delta[..., None] + 3 * U) + 4 * U
        add = (delta * u[t, on])[..., None] * B[t, on][:, None, :]
        err[on] = a * err[on] + np.abs(a * h[on]) * e_a + np.abs(add) * (e_delta[..., None] + 3 * U)
        h[on] = a * h[on] + add
        err[on] += U * np.abs(h[on])
        c = Cm[t, on][:, None, :]
        v = (h[on] * c).sum(axis=2) + D * u[t, on]
        ev = (err[on] * np.abs(c)).sum(axis=2) + (N + 4) * U * ((np.abs(h[on] * c)).sum(axis=2) + np.abs(D * u[t, on]))
        g = silu(z[t, on]) if z is not None else 1.0
        y[t, on] = v * g
        ey[t, on] = 4 * ev * np.abs(g) + 2.0 ** -20 * np.abs(v * g) + HALF[kind] * np.abs(v * g)
    return y, h, ey + 1e-37, 4 * err + 1e-37


def select(logits, scores, eos, finished, count):
    """[(score, parent, token, finished)] of one sequence, best first: by score, then
    beam, then logit, then token; logits [beams,V] and scores [beams] in 64 bits."""
    found = []
    for k in range(logits.shape[0]):
        if not np.isfinite(scores[k]):
            continue
        if finished is not None and finished[k]:
            found.append((scores[k], k, eos, True, 0.0))
            continue
        l = np.where(np.isnan(logits[k]), -np.inf, logits[k])
        top = l.max()
        if not np.isfinite(top):
            continue
        lse = top + np.log(np.exp(l - top).sum())
        best = np.lexsort((np.arange(l.size), -l))[:count]
        found += [(scores[k] + l[v] - lse, k, int(v), bool(v == eos), l[v]) for v in best if l[v] > -np.inf]
    found.sort(key=lambda f: (-f[0], f[1], -f[4], f[2]))
    return [f[:4] for f in found[:count]] + [(-np.inf, 0, 0, False)] * (count - len(found))
