"""Plain 64-bit forms of the products whose ends are fused, for the tests, with
the bounds of their errors: torch in float64, from the formulas, sharing nothing
with the library.

Bounds.  u = 2^-24 is half a step of fp32.  A sum of n products in fp32, however
it is grouped, is off by at most (n + 16) u times the sum of their absolute
values.  half(t) is half a step of the type t of an output relative to its value,
and tiny(t) half of its smallest number."""
import math

import torch

U = 2.0 ** -24


def half(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def dot(a, b):
    """a @ b.T in 64 bits and the sum of the products' absolute values."""
    a, b = a.double(), b.double().t().contiguous()
    return a @ b, a.abs() @ b.abs()


def rounded(value, bound, dtype):
    """The bound after a rounding to dtype."""
    return bound + half(dtype) * (value.abs() + bound) + tiny(dtype)


def check(got, value, bound, what):
    got = got.double()
    ok = ((got - value).abs() <= bound) | (got == value) | (got.isnan() & value.isnan())
    if not bool(ok.all()):
        at = (~ok).nonzero()[0].tolist()
        i = tuple(at)
        raise AssertionError("%s: %d of %d off, first at %r: %r for %r, bound %r"
                             % (what, int((~ok).sum()), ok.numel(), at, float(got[i]), float(value[i]), float(bound[i])))


def scaled_rows(x):
    """(q, scales): the quotient in fp32, as the definition has it (numpy's
    division and rounding are correctly rounded on the CPU)."""
    import numpy as np
    x = x.float().cpu().numpy()
    with np.errstate(invalid="ignore", divide="ignore"):
        most = np.abs(x).max(1, initial=0)
        good = np.isfinite(x).all(1)
        scales = np.maximum(most * np.float32(np.float32(1) / np.float32(127)), np.float32(2.0 ** -126))
        q = np.rint((x / scales[:, None]).astype(np.float32))
    q = np.where(good[:, None], np.clip(np.nan_to_num(q), -127, 127), 0).astype(np.int8)
    return torch.from_numpy(q), torch.from_numpy(np.where(good, scales, np.float32(np.nan)).astype(np.float32))


def scaled(x, w, x_scales, w_scales, dtype):
    """(y, bound): the sum rounded to fp32, two products, the output."""
    y = (x.double() @ w.double().t().contiguous()) * x_scales.double()[:, None] * w_scales.double()
    return y, rounded(y, 3.01 * U * y.abs() + 2.0 ** -148, dtype)


def act(name, a):
    """(act(a), act'(a)) in 64 bits."""
    if name == "silu":
        s = torch.sigmoid(a)
        return a * s, s * (1 + a * torch.sigmoid(-a))
    if name == "gelu":
        p = 0.5 * torch.special.erfc(-a / math.sqrt(2))
        return a * p, p + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    z = math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)
    p = torch.sigmoid(2 * z)
    return a * p, p + 2 * a * p * torch.sigmoid(-2 * z) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * a * a)


def act_error(a, value):
    """How far fp32's act(a) may be from `value`: the exponent's rounding, at most
    2 |a| + a^2 in size, moves the exponential by as many 2^-23, and some ulps of
    the functions (erfc: 16)."""
    return value.abs() * (2.0 ** -19 + (a.abs() + a * a) * 2.0 ** -22) + 2.0 ** -126


def slope_error(a):
    """The same for act'(a), whose terms are at most 1.2 in size: where |a| is large
    the exponentials are as small, so that |a| and a^2 times them stay below 1."""
    return torch.full_like(a, 2.0 ** -18)


def gated(x, up, name, dtype):
    """(y, bound, pre, bound of pre in x's dtype)."""
    I = up.shape[0] // 2
    a, S = dot(x, up)
    e = (x.shape[1] + 16) * U * S
    g, u, eg, eu = a[:, :I], a[:, I:], e[:, :I], e[:, I:]
    v, _ = act(name, g)
    ev = 1.2 * eg + act_error(g.abs() + eg, v)
    y = v * u
    b = ev * u.abs() + v.abs() * eu + ev * eu + 2 * U * y.abs()
    return y, rounded(y, b, dtype), a, rounded(a, e, x.dtype)


def step_of_slopes(dtype, rows):
    """Up to 128 rows have slopes in two parts: half a step of what half a step leaves."""
    return half(dtype) ** 2 if rows <= 128 else half(dtype)


def gated_slopes(pre, d, name, dtype):
    """(the slopes [d_gate d_lift], their bound after their rounding to dtype)."""
    g, u = pre.double().chunk(2, 1)
    d = d.double()
    v, s = act(name, g)
    left, right = d * u * s, d * v
    bound = torch.cat(((d * u).abs() * slope_error(g) + 3 * U * left.abs(), d.abs() * act_error(g, v) + 2 * U * right.abs()), 1)
    t = torch.cat((left, right), 1)
    bound = bound + step_of_slopes(dtype, len(d)) * (t.abs() + bound)
    if dtype == torch.float16:
        # (2^-25 of what the largest is scaled to, 2^14)
        bound = bound + 2.0 ** -39 * t.abs().nan_to_num().max()
    return t, bound + 2.0 ** -133


def product_of_slopes(t, e, m, dtype):
    """(t @ m, its bound) for a t that is off by e."""
    m = m.double().contiguous()
    y = t @ m
    b = e @ m.abs() + (t.shape[1] + 32) * U * ((t.abs() + e) @ m.abs())
    return y, rounded(y, b, dtype)


def gated_grad(x, up, pre, d, name, dtype):
    """((d_x, bound), (d_up, bound))."""
    t, e = gated_slopes(pre, d, name, x.dtype)
    return (product_of_slopes(t, e, up, dtype),
            product_of_slopes(t.t().contiguous(), e.t().contiguous(), x, dtype))


def head(x, w, targets):
    """{"lse": (value, bound), "logprob": (value, bound)}."""
    a, S = dot(x, w)
    e = ((x.shape[1] + 16) * U * S).amax(1)
    T, V = a.shape
    bad = (~(a < math.inf)).any(1)
    lse = torch.logsumexp(a, 1)
    p = torch.softmax(a, 1)
    # a term is off by |a - lse| 2^-23 and some ulps; sums of up to 16 tiles' terms, tiles / 16 of them, and 64 more
    spread = (p * torch.where(p > 0, (a - lse[:, None]).abs(), 0.0)).sum(1) + 8
    rel = e + (spread + 96 + V / 2048) * 2.0 ** -23
    t = targets.clamp(0, V - 1)
    lp = a.gather(1, t[:, None])[:, 0] - lse
    out = {"lse": (torch.where(bad, math.nan, lse), rel + (lse.abs() + 8) * 2.0 ** -23),
           "logprob": (torch.where(targets < 0, 0.0, torch.where((targets >= V) | bad, math.nan, lp)),
                       rel + e + (lp.abs() + 8) * 2.0 ** -23)}
    return out


def head_slopes(x, w, targets, lse, d_logprob, d_lse):
    """(the gradient in the logits, its bound after its rounding to x's dtype)."""
    a, S = dot(x, w)
    T, V = a.shape
    e = (x.shape[1] + 16) * U * S
    zero = torch.zeros(T, dtype=torch.float64, device=x.device)
    gl = zero if d_logprob is None else d_logprob.double()
    gs = zero if d_lse is None else d_lse.double()
    hot = torch.zeros_like(a)
    if d_logprob is not None:
        gl = torch.where(targets < 0, 0.0, torch.where(targets >= V, math.nan, gl))
        hot.scatter_(1, targets.clamp(0, V - 1)[:, None], 1.0)
    t = a - lse.double()[:, None]
    p = torch.exp(t)
    d = gl[:, None] * (hot - p) + gs[:, None] * p
    size = gl.abs()[:, None] * (hot + p) + gs.abs()[:, None] * p
    bound = size * (e + (t.abs() + lse.double().abs()[:, None] + 8) * 2.0 ** -23)
    bound = bound + step_of_slopes(x.dtype, T) * (d.abs() + bound)
    if x.dtype == torch.float16:
        bound = bound + 2.0 ** -39 * (gl.abs() + gs.abs()).nan_to_num().max()
    return d, bound + 2.0 ** -126


def head_grad(x, w, targets, lse, d_logprob, d_lse, dtype):
    """((d_x, bound), (d_head, bound))."""
    d, e = head_slopes(x, w, targets, lse, d_logprob, d_lse)
    return (product_of_slopes(d, e, w, dtype),
            product_of_slopes(d.t().contiguous(), e.t().contiguous(), x, dtype))


def matrix(rows, cols, dtype, seed, pad=0, offset=0, scale=1.0, device="cuda"):
    """A random matrix whose rows lie pad apart, `offset` values into memory that
    otherwise holds NaN (int8: -128)."""
    g = torch.Generator().manual_seed(seed)
    ld = cols + pad
    whole = dtype == torch.int8
    buf = torch.full((offset + rows * ld + 16,), -128 if whole else math.nan, dtype=dtype, device=device)
    m = buf.as_strided((rows, cols), (ld, 1), offset)
    if whole:
        m.copy_(torch.randint(-127, 128, (rows, cols), generator=g, dtype=torch.int8))
    else:
        m.copy_((torch.randn(rows, cols, generator=g) * scale).to(dtype))
    return m


def inside(rows, cols, dtype, pad=0, offset=0):
    """A matrix inside a larger buffer filled with a pattern, and a check that what
    lies around it is as it was."""
    ld = cols + pad
    fill = 77 if dtype == torch.int8 else 1234.0
    buf = torch.full((offset + rows * ld + 64,), fill, dtype=dtype, device="cuda")
    m = buf.as_strided((rows, cols), (ld, 1), offset)

    def untouched():
        rest = buf.clone()
        rest.as_strided((rows, cols), (ld, 1), offset).fill_(fill)
        assert bool((rest == fill).all()), "written outside the matrix"
    return m, untouched
