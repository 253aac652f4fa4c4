"""What the second product of the layer of experts gets of h, whatever h's size and the output's type.

Bound: that of tests/test_experts.py without its absolute term, with what
binary16 parts leave out of h where blocks of 16 columns are brought to one
scale: 2^-39 of the largest h of a token's 64 columns (64 j .. 64 j + 63), times
|w down|.  A 16-bit output adds half its last place, at least 2^-25 in binary16.
"""
import numpy as np
import pytest
import torch

import decode_ref
from paper_2609_16389_amd import xgemm as xg
from test_experts import EPS, TORCH, host, make

pytestmark = pytest.mark.gpu


def left_out(x, scores, up, down, top):
    """(T, H) sums of |w down| times the largest |h| of the 64 columns around."""
    T, H = x.shape
    E, _, I = down.shape
    x, up, down, s = (a.astype(np.float64) for a in (x, up, down, scores))
    ids, out = decode_ref.choices(scores, top), np.zeros((T, H))
    for t in range(T):
        e = np.exp(s[t, ids[t]] - s[t].max())
        for w, j in zip(e / e.sum(), ids[t]):
            g, u = up[j, :I] @ x[t], up[j, I:] @ x[t]
            with np.errstate(over="ignore"):
                h = np.abs(g / (1 + np.exp(-g)) * u)
            most = np.array([h[k // 64 * 64:k // 64 * 64 + 64].max() for k in range(I)])
            out[t] += w * (np.abs(down[j]) @ most)
    return out


def check(args, top, dtype, out):
    y = xg.experts(*args, top, out=torch.empty(args[0].shape, dtype=out, device="cuda"))
    x, scores, up, down = (host(t) for t in args)
    ref, S, _ = decode_ref.experts(x, scores, up, down, top, True)
    tol = ((x.shape[1] + down.shape[2]) / 32 + 128) * 2.0 ** -24 * S + 2.0 ** -39 * left_out(x, scores, up, down, top)
    if out != torch.float32:
        tol = tol * (1 + EPS[dtype]) + EPS[dtype] * np.abs(ref) + (2.0 ** -25 if dtype == "fp16" else 0.0)
    err = np.abs(y.cpu().double().numpy() - ref)
    assert np.all(err <= tol), "off by %.3g of the bound" % np.max(err / tol)


@pytest.mark.parametrize("out", ["fp32", "same"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("I", [200, 201])
@pytest.mark.parametrize("T", [1, 6, 20, 40])
@pytest.mark.parametrize("scale", [(-10, 12), (-13, 14), (0, 0), (9, -9)], ids=lambda s: "2^%d,2^%d" % s)
def test_any_size(scale, T, I, dtype, out):
    """h from 2^-26 to 2^20, `down` scaled so that y is an ordinary number."""
    args = make(T, 4, 96, I, dtype, 21)
    args[0].mul_(2.0 ** scale[0])
    args[3].mul_(2.0 ** scale[1])
    check(args, 2, dtype, torch.float32 if out == "fp32" else TORCH[dtype])


@pytest.mark.parametrize("out", ["fp32", "same"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("I", [200, 201])
@pytest.mark.parametrize("T", [1, 6, 40])
@pytest.mark.parametrize("every", [1, 16])
def test_sizes_beside_each_other(every, T, I, dtype, out):
    """Columns of h of very different size in one block of 16, or blocks in one
    unit of 64, each with as much weight in y as the others."""
    args = make(T, 4, 96, I, dtype, 22)
    down = torch.arange(I, device="cuda") // every % 4 * 5.0 - 5.0   # -5 .. 10
    for half, sign in ((args[2][:, I:], -1.0), (args[3].transpose(1, 2), 1.0)):
        half.mul_(torch.exp2(sign * down)[None, :, None])
    check(args, 2, dtype, torch.float32 if out == "fp32" else TORCH[dtype])


@pytest.mark.parametrize("T", [1, 6, 40])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_tokens_of_different_size(T, dtype):
    """Each row of a slot has its own scale, zeros among them."""
    args = make(T, 4, 96, 200, dtype, 23)
    args[0].mul_(torch.exp2(-(torch.arange(T, device="cuda") % 5 * 3.0))[:, None])
    args[0][T // 2].zero_()
    args[3].mul_(2.0 ** 8)
    check(args, 2, dtype, torch.float32)


def test_infinities_stay_in_their_row():
    args = make(6, 4, 96, 200, "fp16", 24)
    clean = xg.experts(*args, 2)
    args[0][3, 7] = float("inf")
    y = xg.experts(*args, 2)
    assert not bool(torch.isfinite(y[3]).any())
    keep = [t for t in range(6) if t != 3]
    assert torch.equal(y[keep], clean[keep])
