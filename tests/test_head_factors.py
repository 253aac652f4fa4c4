"""Factors of a head's gradient (d_logprob, d_lse) of any size, and of different sizes
in one call."""
import pytest
import torch

import fused_ref
from paper_2609_16389_amd import xgemm as xg


def inputs(T, V, H, dtype, seed=1):
    x, w = fused_ref.matrix(T, H, dtype, seed), fused_ref.matrix(V, H, dtype, seed + 1, scale=0.3)
    targets = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(seed + 2)).cuda()
    return x, w, targets, xg.head_logprobs(x, w)["lse"]


def gradient(x, w, targets, lse, d, z):
    new = lambda t: torch.empty(t.shape, device="cuda")  # noqa: E731
    return xg.head_logprobs_grad(x, w, targets, lse, d, z, out=(new(x), new(w)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [50, 300])
@pytest.mark.parametrize("power", [-110, -60, 60, 115])
def test_factors_of_any_size(T, dtype, power):
    """A power of two in all factors is one in the results, bit for bit."""
    x, w, targets, lse = inputs(T, 900, 48, dtype)
    g = torch.Generator().manual_seed(5)
    d, z = (torch.rand(T, generator=g) + 0.5).cuda(), (torch.rand(T, generator=g) - 0.5).cuda()
    d[0] = 1.75
    one = gradient(x, w, targets, lse, d, z)
    got = gradient(x, w, targets, lse, d * 2.0 ** power, z * 2.0 ** power)
    for a, b in zip(got, one):
        # (what is no normal number there has fewer bits)
        keep = b.double().abs() * 2.0 ** power >= 2.0 ** -120
        assert int(keep.sum()) > 0.9 * keep.numel()
        assert torch.equal(a[keep].double(), b[keep].double() * 2.0 ** power)


def sizes(T, low, seed):
    """Positive factors from 2^low to 1, even over their logarithm, the first 1."""
    f = (torch.rand(T, generator=torch.Generator().manual_seed(seed)) * low).exp2()
    f[0] = 1.0
    return f.cuda()


def bounds_of_rows(x, w, targets, lse, d, z, dtype):
    """fused_ref.head_grad for binary16 slopes that are raised row by row: beside half a
    step, a slope is off by 2^-28 of its row's largest factor, not of all rows'; in d_head
    a row's x is off by 2^-25 where its slopes are at most 2^6 of what the largest factor is
    2^14 of, 2^-33 of that times what the slope is to its row's factor."""
    a, S = fused_ref.dot(x, w)
    e = (x.shape[1] + 16) * fused_ref.U * S
    kept = targets >= 0
    gl = torch.where(kept, d.double(), 0.0)
    gs = torch.zeros_like(gl) if z is None else z.double()
    size = torch.maximum(gl.abs(), gs.abs())[:, None]
    hot = torch.zeros_like(a).scatter_(1, targets.clamp(min=0)[:, None], 1.0)
    t = a - lse.double()[:, None]
    p = torch.exp(t)
    slopes = gl[:, None] * (hot - p) + gs[:, None] * p
    terms = gl.abs()[:, None] * (hot + p) + gs.abs()[:, None] * p
    off = terms * (e + (t.abs() + lse.double().abs()[:, None] + 8) * 2.0 ** -23)
    off = off + fused_ref.step_of_slopes(x.dtype, len(x)) * (slopes.abs() + off) + 2.0 ** -28 * size
    d_x = fused_ref.product_of_slopes(slopes, off, w, dtype)
    value, bound = fused_ref.product_of_slopes(slopes.t().contiguous(), off.t().contiguous(), x, dtype)
    share = torch.where(size > 0, terms / size, 0.0)
    lost = (2.0 ** -33 * size.max() * share.sum(0))[:, None]
    return d_x, (value, bound + lost * (1 + fused_ref.half(dtype)))


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,H", [(2, 60, 8), (50, 900, 48), (128, 301, 43), (129, 900, 48), (300, 700, 33), (700, 4100, 72), (66001, 120, 16)])
@pytest.mark.parametrize("low", [-8, -20, -45, -90])
def test_rows_of_different_size_in_binary16(T, V, H, low):
    """Each row of d_x keeps its bits, however small its factors beside another's."""
    x, w, targets, lse = inputs(T, V, H, torch.float16)
    targets[1 :: 7] = -1
    d = -sizes(T, low, 5)
    for z in (None, sizes(T, low, 6) * 0.01):
        for dtype in (torch.float32, torch.float16):
            if dtype == torch.float16 and low < -20:
                continue   # (they would be zeros of that type)
            out = (torch.empty(T, H, dtype=dtype, device="cuda"), torch.empty(V, H, dtype=dtype, device="cuda"))
            got = xg.head_logprobs_grad(x, w, targets, lse, d, z, out=out)
            for t, (value, bound), name in zip(got, bounds_of_rows(x, w, targets, lse, d, z, dtype), ("d_x", "d_head")):
                fused_ref.check(t, value, bound, name)
            one = xg.head_logprobs_grad(x, w, targets, lse, d, z, out=(torch.empty_like(out[0]), None))[0]
            assert torch.equal(one, got[0])


@pytest.mark.gpu
def test_a_small_row_beside_a_large_one():
    """Factors 1 and 1e-12: the small row's gradient is that of the row alone."""
    for T in (2, 200):
        x, w, targets, lse = inputs(T, 900, 48, torch.float16)
        d = torch.full((T,), -1.0, device="cuda")
        d[1] = -1e-12
        alone = torch.zeros(T, device="cuda")
        alone[1] = d[1]
        got, ref = (gradient(x, w, targets, lse, v, None)[0][1].double() for v in (d, alone))
        # (both are off by half a step of binary16 in each slope, of two parts half of half a step)
        p = torch.exp(x[1].double() @ w.double().t().contiguous() - lse[1].double())
        p[targets[1]] += 1
        step = fused_ref.step_of_slopes(torch.float16, T) * p + 2.0 ** -28
        assert float(ref.abs().max()) > 1e-14
        assert bool(((got - ref).abs() <= 1e-12 * (2 * step @ w.double().abs() + 2.0 ** -20 * (p @ w.double().abs()))).all())
