"""Log probabilities from a head's weights for logits of any size: products of one
term, which fp32 holds exactly, so that what is left is the statistics' own error."""
import math

import pytest
import torch

import fused_ref
from paper_2609_16389_amd import xgemm as xg


def logits_of(size, T, V, dtype, seed):
    """x (T, 1) and w (V, 1) whose products are up to `size`, of both signs, and some
    rows' a hair's breadth apart."""
    g = torch.Generator().manual_seed(seed)
    w = (torch.rand(V, 1, generator=g) * 2 - 1).to(dtype)
    w[0], w[V // 2], w[V - 1] = 1.0, 1.0 - torch.finfo(dtype).eps / 2, -1.0
    x = (torch.rand(T, 1, generator=g) + 0.5).log2().exp2() * size
    x[:: 2] *= -1
    return x.to(dtype).cuda(), w.cuda()


SIZES = {torch.bfloat16: [1.0, 30.0, 900.0, 1100.0, 2.0 ** 18, 2.0 ** 20, 2.0 ** 24, 2.0 ** 31, 2.0 ** 40, 1e20, 1e37],
         torch.float16: [1.0, 30.0, 900.0, 1100.0, 2.0 ** 15]}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,size", [(t, s) for t in SIZES for s in SIZES[t]])
@pytest.mark.parametrize("T,V", [(3, 700), (70, 1031), (600, 5000)])
def test_logits_of_any_size(T, V, dtype, size):
    x, w = logits_of(size, T, V, dtype, 1)
    targets = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(2)).cuda()
    targets[0], targets[1], targets[2] = 0, V - 1, V // 2
    a = x.double() @ w.double().t().contiguous()
    assert torch.equal(a, a.float().double())
    # (lse - logit cancels all that 64 bits hold where logits are large: from the largest)
    most = a.amax(1)
    log_sum = torch.log(torch.exp(a - most[:, None]).sum(1))
    lse, p = most + log_sum, torch.exp(a - most[:, None] - log_sum[:, None])
    # as in fused_ref.head, of logits without an error: a term is off by |a - lse| 2^-23 and some ulps
    rel = ((p * torch.where(p > 0, (a - most[:, None] - log_sum[:, None]).abs(), 0.0)).sum(1) + 104 + V / 2048) * 2.0 ** -23
    lp = (a.gather(1, targets[:, None])[:, 0] - most) - log_sum
    out = xg.head_logprobs(x, w, targets)
    fused_ref.check(out["lse"], lse, rel + lse.abs() * 2.0 ** -23, "lse")
    fused_ref.check(out["logprob"], lp, rel + (lp.abs() + 8) * 2.0 ** -23, "logprob")


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 300])
def test_the_largest_binary16_values(T):
    """Sums of products of 65504."""
    H, V = 64, 900
    x = torch.full((T, H), 65504.0, dtype=torch.float16, device="cuda")
    w = torch.zeros(V, H, dtype=torch.float16, device="cuda")
    for v, n in ((0, 64), (7, 63), (500, 64), (899, 1)):
        w[v, :n] = 65504.0
    w[3] = -65504.0
    targets = torch.arange(T, device="cuda") % 2 * 500
    out = xg.head_logprobs(x, w, targets)
    # two logits are the largest, 65504^2 64 (exact in fp32 but for its last bits), the others nowhere near
    most = 65504.0 ** 2 * 64
    assert bool(((out["lse"].double() - most).abs() <= most * 2.0 ** -20).all())
    assert bool(((out["logprob"] + math.log(2)).abs() <= 2.0 ** -20).all())
