"""The gradient of a gated block with rows of different size in one call."""
import pytest
import torch

import fused_ref
from paper_2609_16389_amd import xgemm as xg


def inputs(M, H, I, low, act):
    """Rows whose slopes reach from 2^low of the largest to it: by d's size down to what
    binary16 holds of it, and by the block's inner values."""
    x, up = fused_ref.matrix(M, H, torch.float16, 1), fused_ref.matrix(2 * I, H, torch.float16, 2, scale=0.2)
    power = torch.rand(M, 1, generator=torch.Generator().manual_seed(5)) * low
    power[0] = 0
    power = power.cuda()
    pre = fused_ref.matrix(M, 2 * I, torch.float16, 3).float()
    d = fused_ref.matrix(M, I, torch.float16, 4).float()
    by_d = power.clamp(min=-10)
    # gelu and silu of values near 0 are half of them: the lift and the gate together
    d *= by_d.exp2()
    pre *= ((power - by_d) / 1).clamp(min=-22).exp2()
    return x, up, pre.half(), d.half()


def bounds_of_rows(x, up, pre, d, act, dtype):
    """fused_ref.gated_grad for binary16 slopes that are raised row by row (as the head's
    bounds in test_head_factors.py)."""
    g, u = pre.double().chunk(2, 1)
    d64 = d.double()
    v, s = fused_ref.act(act, g)
    left, right = d64 * u * s, d64 * v
    off = torch.cat(((d64 * u).abs() * fused_ref.slope_error(g) + 3 * fused_ref.U * left.abs(),
                     d64.abs() * fused_ref.act_error(g, v) + 2 * fused_ref.U * right.abs()), 1)
    t = torch.cat((left, right), 1)
    size = t.abs().amax(1, keepdim=True)
    off = off + fused_ref.step_of_slopes(x.dtype, len(d)) * (t.abs() + off) + 2.0 ** -28 * size
    d_x = fused_ref.product_of_slopes(t, off, up, dtype)
    value, bound = fused_ref.product_of_slopes(t.t().contiguous(), off.t().contiguous(), x, dtype)
    share = torch.where(size > 0, t.abs() / size, 0.0)
    lost = (2.0 ** -33 * size.max() * share.sum(0))[:, None]
    return d_x, (value, bound + lost * (1 + fused_ref.half(dtype)))


@pytest.mark.gpu
@pytest.mark.parametrize("M,H,I", [(2, 8, 5), (9, 40, 1030), (128, 43, 70), (129, 48, 130), (333, 100, 701), (2053, 40, 520), (66001, 16, 20)])
@pytest.mark.parametrize("low", [-8, -20, -32])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_rows_of_different_size_in_binary16(M, H, I, low, act):
    x, up, pre, d = inputs(M, H, I, low, act)
    out = (torch.empty(M, H, device="cuda"), torch.empty(2 * I, H, device="cuda"))
    got = xg.gated_grad(x, up, pre, d, act, out=out)
    for t, (value, bound), name in zip(got, bounds_of_rows(x, up, pre, d, act, torch.float32), ("d_x", "d_up")):
        fused_ref.check(t, value, bound, name)
    for at in (0, 1):
        one = [torch.empty_like(t) for t in out]
        one[1 - at] = None
        xg.gated_grad(x, up, pre, d, act, out=tuple(one))
        assert torch.equal(one[at], got[at])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M", [5, 300])
def test_rows_of_zeros(M, dtype):
    """Rows without a gradient, and a gradient of nothing but such rows."""
    x, up = fused_ref.matrix(M, 40, dtype, 1), fused_ref.matrix(140, 40, dtype, 2, scale=0.2)
    pre, d = fused_ref.matrix(M, 140, dtype, 3), fused_ref.matrix(M, 70, dtype, 4)
    d[1] = 0
    ref = fused_ref.gated_grad(x, up, pre, d, "silu", dtype)
    got = xg.gated_grad(x, up, pre, d)
    for t, (value, bound), name in zip(got, ref, ("d_x", "d_up")):
        fused_ref.check(t, value, bound, name)
    assert bool((got[0][1] == 0).all())
    for t in xg.gated_grad(x, up, pre, torch.zeros_like(d)):
        assert bool((t == 0).all())
