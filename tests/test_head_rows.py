"""Rows of a head's gradient: those that take no part in it, whatever they hold."""
import math

import pytest
import torch

import fused_ref
from paper_2609_16389_amd import xgemm as xg

INF = float("inf")


@pytest.mark.gpu
@pytest.mark.parametrize("out", [None, torch.float32])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,V,H,pad", [(1, 40, 8, 0), (20, 700, 40, 0), (300, 700, 40, 0), (300, 701, 43, 0), (130, 9001, 24, 5),
                                       (700, 3000, 128, 8)])
def test_rows_without_part_do_not_reach_the_weights(T, V, H, pad, dtype, out):
    """A prompt, padding, a token of weight 0, a row whose logits are all -inf: their
    hidden states may hold anything, also what 0 times it is not 0."""
    x, w = fused_ref.matrix(T, H, dtype, 1, pad), fused_ref.matrix(V, H, dtype, 2, pad, scale=0.3)
    targets = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(3)).cuda()
    d = torch.full((T,), -1.0 / T, device="cuda")
    clean = x.clone()
    if T == 1:
        rows = [0]
        targets[0], x[0] = -100, math.nan
    else:
        rows = [0, 3, 7, 8, 11, T - 1]
        targets[0] = targets[3] = targets[T - 1] = -100
        d[7] = d[8] = 0.0
        x[0], x[3, H - 1], x[7], x[8, 1], x[T - 1, 0] = math.nan, INF, -INF, math.nan, -INF
        x[11, 0] = -INF   # every logit -inf
        w[:, 0] = w[:, 0].abs() + 0.01
    clean[rows] = 0
    lse = xg.head_logprobs(x, w)["lse"]
    if T > 1:
        assert lse[11] == -INF
    new = lambda: (torch.empty(T, H, dtype=out or dtype, device="cuda"), torch.empty(V, H, dtype=out or dtype, device="cuda"))  # noqa: E731
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[rows] = False
    lse_clean = torch.where(keep, lse, 0.0)
    ref = fused_ref.head_grad(clean, w, targets, lse_clean, torch.where(keep, d, 0.0), None, out or dtype)
    got = xg.head_logprobs_grad(x, w, targets, lse, d, out=new())
    for t, (value, bound), name in zip(got, ref, ("d_x", "d_head")):
        fused_ref.check(t, value, bound, name)
    assert bool((got[0][rows] == 0).all())
    one = xg.head_logprobs_grad(x, w, targets, lse, d, out=(None, new()[1]))[1]
    assert torch.equal(one, got[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [20, 300])
def test_rows_with_part_do(T, dtype):
    """A row without a target that has a d_lse, and one whose target does not exist."""
    x, w = fused_ref.matrix(T, 40, dtype, 1), fused_ref.matrix(500, 40, dtype, 2, scale=0.3)
    targets = torch.randint(0, 500, (T,), generator=torch.Generator().manual_seed(3)).cuda()
    d, z = torch.full((T,), -1.0 / T, device="cuda"), torch.zeros(T, device="cuda")
    targets[4], z[4] = -1, 0.5
    lse = xg.head_logprobs(x, w)["lse"]
    ref = fused_ref.head_grad(x, w, targets, lse, d, z, torch.float32)
    got = xg.head_logprobs_grad(x, w, targets, lse, d, z, out=(torch.empty(T, 40, device="cuda"), torch.empty(500, 40, device="cuda")))
    for t, (value, bound), name in zip(got, ref, ("d_x", "d_head")):
        fused_ref.check(t, value, bound, name)
    targets[4] = 500
    got = xg.head_logprobs_grad(x, w, targets, lse, d, z)
    assert bool(got[0][4].isnan().all()) and bool(got[1].isnan().all())
    assert not bool(got[0][5:].isnan().any())
