"""Plain 64-bit forms of the operators around a decoding step, for the tests:
numpy, from the formulas, sharing nothing with the library."""
import numpy as np


def unpack(q, K):
    """4-bit values (N, K) from bytes (N, ceil(K / 2)), even k in the low half."""
    k = np.arange(K)
    return (q[:, k // 2] >> (4 * (k % 2))) & 15


def quant(x, q, scales, zeros, group, K):
    """(y, S) with S[m, n] = sum over k of |x s| (16 + q) + |x s| (16 + z): what
    the products summed for y add up to at most."""
    k = np.arange(K) // group
    v = unpack(q, K).astype(np.float64)
    z = zeros.astype(np.float64)[:, k] if zeros is not None else np.full(v.shape, 8.0)
    s = scales.astype(np.float64)[:, k]
    x = x.astype(np.float64)
    return x @ ((v - z) * s).T, np.abs(x) @ (np.abs(s) * (32.0 + v + z)).T


def choices(scores, top):
    """(T, top) experts of the largest scores, equal ones in ascending order;
    a NaN counts as the largest."""
    s = np.where(np.isnan(scores), np.inf, scores.astype(np.float64))
    first = np.isnan(scores)
    order = [sorted(range(s.shape[1]), key=lambda e: (not first[t, e], -s[t, e], e))[:top] for t in range(s.shape[0])]
    return np.array(order, dtype=np.int64).reshape(s.shape[0], top)


def experts(x, scores, up, down, top, renormalize):
    """(y, S, chosen): S[t, n] is the sum of the absolute products of the second
    product, weighted, with |h| replaced by the bound on what h is made of."""
    T, H = x.shape
    E, _, I = down.shape
    x, up, down, s = (np.asarray(a, dtype=np.float64) for a in (x, up, down, scores))
    ids = choices(scores, top)
    y, S = np.zeros((T, H)), np.zeros((T, H))
    for t in range(T):
        m = np.max(np.where(np.isnan(s[t]), -np.inf, s[t]))
        with np.errstate(invalid="ignore"):
            e = np.where(s[t] == -np.inf, 0.0, np.exp(s[t] - m))
        total = e[ids[t]].sum() if renormalize else e.sum()
        for j in ids[t]:
            w = 0.0 if total == 0 else e[j] / total
            g, u = up[j, :I] @ x[t], up[j, I:] @ x[t]
            with np.errstate(over="ignore"):
                h = g / (1 + np.exp(-g)) * u
            ag, au = np.abs(up[j, :I]) @ np.abs(x[t]), np.abs(up[j, I:]) @ np.abs(x[t])
            y[t] += w * (down[j] @ h)
            # |silu'| <= 1.1 and |silu(g)| <= |g|
            S[t] += abs(w) * (np.abs(down[j]) @ (1.1 * ag * np.abs(u) + np.abs(g) * au + np.abs(h)))
    return y, S, ids
