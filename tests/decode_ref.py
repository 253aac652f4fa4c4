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
