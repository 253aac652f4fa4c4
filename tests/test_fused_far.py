"""The products whose ends are fused with more rows than a launch takes, and with
matrices of more than 2^32 bytes."""
import pytest
import torch

import fused_ref
from paper_2609_16389_amd import xgemm as xg

ROWS = 65536 + 300   # (a launch takes 65536 rows of a result)


@pytest.mark.gpu
@pytest.mark.parametrize("K", [48, 33])
def test_scaled_rows_of_two_launches(K):
    a, w = fused_ref.matrix(ROWS, K, torch.int8, 1), fused_ref.matrix(70, K, torch.int8, 2)
    xs, ws = torch.rand(ROWS, device="cuda"), torch.rand(70, device="cuda")
    y, bound = fused_ref.scaled(a, w, xs, ws, torch.bfloat16)
    fused_ref.check(xg.gemm_scaled(a, w, ws, xs, out=torch.empty(ROWS, 70, dtype=torch.bfloat16, device="cuda")), y, bound, "y")


@pytest.mark.gpu
@pytest.mark.parametrize("H", [24, 13])
def test_gated_rows_of_two_launches(H):
    x = fused_ref.matrix(ROWS, H, torch.bfloat16, 1)
    up = fused_ref.matrix(80, H, torch.bfloat16, 2, scale=0.3)
    pre = torch.empty(ROWS, 80, dtype=x.dtype, device="cuda")
    y, bound, a, pre_bound = fused_ref.gated(x, up, "gelu_tanh", x.dtype)
    fused_ref.check(xg.gated(x, up, "gelu_tanh", pre=pre), y, bound, "out")
    fused_ref.check(pre, a, pre_bound, "pre")
    d = fused_ref.matrix(ROWS, 40, x.dtype, 3, scale=0.05)
    (dx, bx), (du, bu) = fused_ref.gated_grad(x, up, pre, d, "gelu_tanh", x.dtype)
    got = xg.gated_grad(x, up, pre, d, "gelu_tanh")
    fused_ref.check(got[0], dx, bx, "d_x")
    fused_ref.check(got[1], du, bu, "d_up")


@pytest.mark.gpu
def test_head_rows_of_two_launches():
    x = fused_ref.matrix(ROWS, 16, torch.float16, 1)
    w = fused_ref.matrix(300, 16, torch.float16, 2, scale=0.5)
    targets = torch.randint(-1, 300, (ROWS,), generator=torch.Generator().manual_seed(3)).cuda()
    out = xg.head_logprobs(x, w, targets)
    for name, (value, bound) in fused_ref.head(x, w, targets).items():
        fused_ref.check(out[name], value, bound, name)
    d = torch.full((ROWS,), -1.0 / ROWS, device="cuda")
    ref = fused_ref.head_grad(x, w, targets, out["lse"], d, None, x.dtype)
    for t, (value, bound), name in zip(xg.head_logprobs_grad(x, w, targets, out["lse"], d), ref, ("d_x", "d_head")):
        fused_ref.check(t, value, bound, name)


@pytest.mark.gpu
def test_results_past_32_bits():
    """5.3 GB of results: the rows on either side of 2^32 bytes, and the last ones."""
    M, N, K = 40000, 33000, 32
    a, w = fused_ref.matrix(M, K, torch.int8, 1), fused_ref.matrix(N, K, torch.int8, 2)
    xs, ws = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    out = xg.gemm_scaled(a, w, ws, xs, out=torch.empty(M, N, device="cuda"))
    at = 2 ** 32 // (4 * N)
    for rows in (slice(0, 40), slice(at - 20, at + 20), slice(M - 40, M)):
        y, bound = fused_ref.scaled(a[rows], w, xs[rows], ws, torch.float32)
        fused_ref.check(out[rows], y, bound, "rows %r" % rows)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 200])
def test_weights_past_32_bits(T):
    """A head of 4.6 GB whose last rows hold the targets."""
    V, H = 140000, 16384
    g = torch.Generator("cuda").manual_seed(1)
    w = torch.empty(V, H, dtype=torch.bfloat16, device="cuda")
    for v in range(0, V, 20000):
        w[v:v + 20000] = torch.randn(20000, H, device="cuda", generator=g).mul_(0.02).to(w.dtype)
    x = fused_ref.matrix(T, H, w.dtype, 2)
    targets = torch.arange(V - T, V, device="cuda")
    out = xg.head_logprobs(x, w, targets)
    parts = [fused_ref.dot(x, w[v:v + 10000]) for v in range(0, V, 10000)]
    a, S = torch.cat([p[0] for p in parts], 1), torch.cat([p[1] for p in parts], 1)
    lse = torch.logsumexp(a, 1)
    e = (H + 16) * fused_ref.U * S.amax(1) + (96 + V / 2048 + 16) * 2.0 ** -23   # (as fused_ref.head)
    fused_ref.check(out["lse"], lse, e + (lse.abs() + 8) * 2.0 ** -23, "lse")
    lp = a.gather(1, targets[:, None])[:, 0] - lse
    fused_ref.check(out["logprob"], lp, 2 * e + (lp.abs() + 8) * 2.0 ** -23, "logprob")
    d = torch.full((T,), -1.0 / T, device="cuda")
    _, got = xg.head_logprobs_grad(x, w, targets, out["lse"], d, out=(None, torch.empty_like(w)))
    # the last rows of the gradient, from the formula
    rows = slice(V - T, V)
    p = torch.exp(a[:, rows] - out["lse"].double()[:, None])
    s = (p - torch.eye(T, dtype=torch.float64, device="cuda")) / T
    step = fused_ref.step_of_slopes(w.dtype, T)
    bound = (p + 1) / T * ((H + 16) * fused_ref.U * S[:, rows] + 60 * 2.0 ** -23) + step * s.abs()
    value, b = fused_ref.product_of_slopes(s.t().contiguous(), bound.t().contiguous(), x, w.dtype)
    fused_ref.check(got[rows], value, b, "d_head")
