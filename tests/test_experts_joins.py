"""Layers of experts whose second product is cut over workgroups, joined by the last of them.

The shapes are those for which waves take ranges of their own, for one or two
tokens and for a few more, in two parts or more on 256 CUs, with inner sizes
that are and are not multiples of 8.
"""
import pytest
import torch

from paper_2609_16389_amd import xgemm as xg
from test_experts import TORCH, check, make

pytestmark = pytest.mark.gpu

SHAPES = [(1, 16, 8, 200, 1024), (1, 16, 8, 72, 2047), (2, 16, 8, 72, 1001), (2, 32, 8, 40, 1536), (5, 16, 6, 136, 640),
          (5, 16, 6, 136, 647), (16, 16, 2, 40, 1030)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("out", ["fp32", "same"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%dt%de%dk%dx%d" % s)
def test_joined_parts(shape, out, dtype):
    T, E, top, H, I = shape
    for pad in (0, 3):
        args = make(T, E, H, I, dtype, 61 + T + H + I, pad)
        y = xg.experts(*args, top, out=torch.empty((T, H), dtype=torch.float32 if out == "fp32" else TORCH[dtype],
                                                   device="cuda"))
        check(y, args, top, True, dtype, "pad %d" % pad)
        for _ in range(5):                                 # whoever comes last
            assert torch.equal(xg.experts(*args, top, out=torch.empty_like(y)), y)
