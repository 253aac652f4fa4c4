"""Products with 4-bit weights of bfloat16 values near the ends of fp32's range.

The bound is that of tests/test_quant.py: no intermediate result is outside
fp32's range as long as the output is inside.
"""
import pytest
import torch

from paper_2609_16389_amd import xgemm as xg
from test_quant import TORCH, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [1, 2, 5, 20, 64])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, True), (128, True), (128, False), (384, True)])
def test_large_values(M, group, zeros):
    """x up to 3.3e38: sums of x (16 + q) would overflow, those of the scaled differences do not."""
    K, N = 1100, 72
    x, q, s, z = make(M, N, K, "bf16", group, zeros, 41, pad=3)
    x.clamp_(-3.9, 3.9).mul_(2.0 ** 126)
    assert bool(torch.isfinite(x).all()) and float(x.abs().max()) > 3e38
    s.mul_(2.0 ** -14)
    if zeros:
        z.copy_(torch.randint(0, 256, z.shape, device="cuda", dtype=torch.uint8))
    for out in (torch.float32, TORCH["bf16"]):
        y = xg.gemv_quant(x, q, s, z, group, out=torch.empty((M, N), dtype=out, device="cuda"))
        assert bool(torch.isfinite(y).all())
        check(y, x, q, s, z, group, K, "bf16", out)


@pytest.mark.parametrize("M", [1, 5, 20, 64])
def test_small_values(M):
    """x around 2^-90 against scales that bring the output back."""
    x, q, s, z = make(M, 72, 1100, "bf16", 64, True, 42)
    x.mul_(2.0 ** -90)
    s.mul_(2.0 ** 90)
    check(xg.gemv_quant(x, q, s, z, 64), x, q, s, z, 64, 1100, "bf16", "small")
