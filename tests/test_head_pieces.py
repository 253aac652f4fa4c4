"""The gradient of a head for few rows and more columns than are taken at a time."""
import pytest
import torch

import fused_ref
from paper_2609_16389_amd import xgemm as xg


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_few_rows_of_a_vocabulary_in_pieces(dtype):
    """Slopes in two parts, with more columns than are taken at a time."""
    T, V, H = 128, (1 << 20) + 1001, 16
    x, w = fused_ref.matrix(T, H, dtype, 1), fused_ref.matrix(V, H, dtype, 2, scale=0.3)
    targets = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(3)).cuda()
    lse = xg.head_logprobs(x, w)["lse"]
    targets[3], targets[4], targets[5] = V - 1, 1 << 20, (1 << 20) - 1
    d = torch.full((T,), -1.0 / T, device="cuda")
    for out in (dtype, torch.float32):
        got = xg.head_logprobs_grad(x, w, targets, lse, d, out=(torch.empty(T, H, dtype=out, device="cuda"),
                                                                torch.empty(V, H, dtype=out, device="cuda")))
        ref = fused_ref.head_grad(x, w, targets, lse, d, None, out)
        for t, (value, bound), name in zip(got, ref, ("d_x", "d_head")):
            fused_ref.check(t, value, bound, name)
        del ref, got
