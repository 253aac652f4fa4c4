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
