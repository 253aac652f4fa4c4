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


def logprobs(x, targets, top):
    """lse, logprob, entropy, top_logprob, top_id of rows x in 64 bits."""
    R, V = x.shape
    x = x.astype(np.float64)
    bad = np.isnan(x).any(1) | (x == np.inf).any(1)
    m = np.max(np.where(np.isnan(x), -np.inf, x), axis=1)
    ref = np.where(np.isfinite(m), m, 0.0)[:, None]
    with np.errstate(all="ignore"):
        t = x - ref
        e = np.exp(t)
        S = e.sum(1)
        logS = np.log(S)
        lse = m + logS
        empty = m == -np.inf
        lse[empty] = -np.inf
        entropy = np.where(empty, 0.0, logS - np.where(e > 0, e * t, 0.0).sum(1) / S)
        hit = x[np.arange(R), np.clip(targets, 0, V - 1)]
        logprob = np.where(empty, -np.inf, (hit - m) - logS)
    lse[bad], entropy[bad], logprob[bad] = np.nan, np.nan, np.nan
    logprob = np.where(targets < 0, 0.0, np.where(targets >= V, np.nan, logprob))
    ids, vals = np.full((R, top), -1, dtype=np.int64), np.full((R, top), np.nan)
    for r in range(R):
        order = np.lexsort((np.arange(V), -np.where(np.isnan(x[r]), -np.inf, x[r])))
        order = order[~np.isnan(x[r, order])]
        n = min(top, len(order))
        ids[r, :n] = order[:n]
        if not bad[r]:
            vals[r, :n] = -np.inf if empty[r] else (x[r, order[:n]] - m[r]) - logS[r]
    return lse, logprob, entropy, vals, ids


def logprobs_grad(x, targets, d_logprob, d_entropy, d_lse):
    """The gradient in x of sum d_logprob logprob + d_entropy entropy + d_lse lse,
    and the sum of its terms' absolute values."""
    R, V = x.shape
    zero = np.zeros(R)
    gl, ge, gs = (zero if d is None else d.astype(np.float64) for d in (d_logprob, d_entropy, d_lse))
    lse, _, entropy, _, _ = logprobs(x, targets, 0)
    with np.errstate(invalid="ignore"):
        logp = np.where((lse == -np.inf)[:, None], -np.inf, x.astype(np.float64) - lse[:, None])
    p = np.exp(logp)
    logp = np.where(p > 0, logp, 0.0)
    hot = np.zeros((R, V))
    on = (targets >= 0) & (targets < V)
    hot[np.arange(R)[on], targets[on]] = 1.0
    gl = np.where(targets >= V, np.nan if d_logprob is not None else 0.0, np.where(targets < 0, 0.0, gl))
    gl, ge, gs = gl[:, None], ge[:, None], gs[:, None]
    d = gl * (hot - p) - ge * p * (logp + entropy[:, None]) + gs * p
    S = np.abs(gl) * (hot + p) + np.abs(ge) * p * (np.abs(logp) + np.abs(entropy[:, None])) + np.abs(gs) * p
    empty = (lse == -np.inf)[:, None]
    return np.where(empty, 0.0, d), np.where(empty, 0.0, S), logp
