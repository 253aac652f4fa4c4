"""The gradient of rows whose log-sum-exp is large: masks of a large finite value, shifted rows, high scales.

Bound: that of tests/test_logprobs.py, with what the rounding of lse leaves in
log p: |lse| 2^-24 where |lse| is below 256 (fp32) or 1024 (16 bits), else
nothing, since the row is summed again.  An error of log p counts relative to p
in every term, and once more, absolute, in that of the entropy.
"""
import numpy as np
import pytest
import torch

import decode_ref
from paper_2609_16389_amd import xgemm as xg
from test_logprobs import EPS, TORCH, close, grads, host, make

pytestmark = pytest.mark.gpu

LIMIT = {"fp32": 256.0, "bf16": 1024.0, "fp16": 1024.0}


def check(got, x, targets, d, dtype, what):
    t, h = targets.cpu().numpy(), [v.cpu().numpy() for v in d]
    # (the gradient does not change with a row's offset, which 64 bits would round too)
    x64 = host(x).astype(np.float64)
    ref, S, logp = decode_ref.logprobs_grad(x64 - x64.max(1, keepdims=True), t, *h)
    lse = decode_ref.logprobs(host(x), t, 0)[0]
    held = np.where(np.abs(lse) < LIMIT[dtype], np.abs(lse) * 2.0 ** -24, 0.0)[:, None]
    spread = np.log(x.shape[1]) + x.shape[1] / 512 + 60
    of_log = (2 * np.abs(logp) + spread) * 2.0 ** -23 + held
    tol = (S + np.abs(h[1])[:, None] * np.exp(logp)) * of_log + 2.0 ** -120
    if dtype != "fp32":
        tol = tol * 2 + EPS[dtype] * np.abs(ref) + (2.0 ** -24 if dtype == "fp16" else 0.0)
    close(got, ref, tol, what)


VALUES = {"fp32": [-1e4, -1e9, -1e30, 1e4, 3e37], "bf16": [-1e4, -1e9, -1e30, 1e4], "fp16": [-1e4, -6e4, 3e4]}


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [1, 7, 700, 4096, 5000, 40001, 140000])
def test_rows_of_one_value_and_shifted_rows(V, dtype):
    values = VALUES[dtype]
    n = len(values)
    x, targets = make(2 * n + 6, V, dtype, V, pad=3)
    for i, v in enumerate(values):
        x[i] = v                                           # every token masked alike
        x[n + i] = (x[n + i].double() + v).to(x.dtype)     # shifted
    x[2 * n, : V // 2] = values[0]                         # part of a row masked, as ever
    x[2 * n + 1] *= 40                                     # high scales
    x[2 * n + 2] *= 200
    x[2 * n + 3] += 255
    x[2 * n + 4] -= 1030
    f = xg.logprobs(x, targets)
    d = grads(x.shape[0], 31)
    got = xg.logprobs_grad(x, targets, f["lse"], f["entropy"], *d)
    check(got, x, targets, d, dtype, "V %d" % V)
    uniform = xg.logprobs_grad(x, targets, f["lse"], d_lse=torch.ones(x.shape[0], device="cuda"))
    for i in range(n):
        if -1e37 < values[i]:
            assert torch.allclose(uniform[i].double(), torch.full((), 1.0 / V, dtype=torch.float64, device="cuda"),
                                  rtol=2 * EPS[dtype] + 1e-5, atol=2.0 ** -24)
    # into the logits themselves: the same bits
    buf = x.clone()
    assert torch.equal(xg.logprobs_grad(buf, targets, f["lse"], f["entropy"], *d, out=buf), got)
    for row in (0, n, 2 * n + 2):                          # and in any company
        one = slice(row, row + 1)
        assert torch.equal(xg.logprobs_grad(x[one], targets[one], f["lse"][one], f["entropy"][one],
                                            *(v[one] for v in d)), got[one])


def test_no_token_gains_or_loses():
    """The gradient of a log probability sums to 0 over the row."""
    x, targets = make(6, 30000, "fp32", 5)
    for i, c in enumerate((0.0, 200.0, 300.0, -5000.0, 1e5, -1e7)):
        x[i] += c
    f = xg.logprobs(x, targets)
    g = xg.logprobs_grad(x, targets, f["lse"], d_logprob=torch.ones(6, device="cuda"))
    assert bool((g.double().sum(1).abs() < 2e-5).all())


def test_a_part_of_a_longer_row_keeps_its_own_sum():
    """An lse that is not the row's (a vocabulary in two parts) is taken as given."""
    x, targets = make(2, 1000, "fp32", 6)
    x += 512.0
    lse = torch.logsumexp(x.double(), 1).float()
    d = torch.ones(2, device="cuda")
    g = xg.logprobs_grad(x[:, :600], targets, lse, d_lse=d)
    p = torch.exp(x[:, :600].double() - lse.double()[:, None])
    assert torch.allclose(g.double(), p, rtol=1e-5, atol=1e-12)
