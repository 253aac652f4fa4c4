"""Products in 8-bit integers and the rows they are made of, against 64 bits."""
import math

import pytest
import torch

import fused_ref
from paper_2609_16389_amd import xgemm as xg

TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "int8": torch.int8}
INF = float("inf")


def inputs(M, N, K, x="int8", seed=0, pad=(0, 0), offset=(0, 0)):
    dt = TORCH[x]
    a = fused_ref.matrix(M, K, dt, seed, pad[0], offset[0])
    w = fused_ref.matrix(N, K, torch.int8, seed + 1, pad[1], offset[1])
    g = torch.Generator().manual_seed(seed + 2)
    scale = lambda n: (torch.rand(n, generator=g) * 0.01 + 1e-4).cuda()  # noqa: E731
    return a, w, scale(N), scale(M) if x == "int8" else None


def check(a, w, ws, xs, out, what=""):
    if xs is None:
        q, xs = fused_ref.scaled_rows(a)
        a, xs = q.cuda(), xs.cuda()
    y, bound = fused_ref.scaled(a, w, xs, ws, out.dtype)
    fused_ref.check(out, y, bound, what)


# few rows; K within one chunk, at its end, past it; sizes at the ends of tiles;
# split sums; large tiles
SHAPES = [(1, 1, 1), (1, 5, 16), (2, 3, 17), (3, 129, 127), (1, 64, 128), (16, 256, 129), (17, 33, 255), (64, 65, 1000),
          (65, 300, 64), (100, 127, 2048), (129, 257, 400), (1, 700, 4096), (8, 96, 5001), (300, 500, 4100), (2053, 4100, 272),
          (2304, 4096, 128), (1, 8200, 512), (4, 4200, 2048), (5, 4200, 2064), (16, 100, 8192), (1, 40, 16400), (1, 33, 16384),
          (3, 12345, 272), (37, 1003, 2047), (333, 700, 1001), (4096, 5001, 1024), (2100, 9100, 512)]


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("x", ["int8", "bf16", "fp16", "fp32"])
def test_shapes(M, N, K, x):
    a, w, ws, xs = inputs(M, N, K, x, M + N + K)
    for out in ("fp32", "bf16", "fp16"):
        check(a, w, ws, xs, xg.gemm_scaled(a, w, ws, xs, out=torch.empty(M, N, dtype=TORCH[out], device="cuda")), out)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 50, 96), (5, 70, 333), (40, 200, 512), (200, 260, 1030), (2100, 2300, 48)])
@pytest.mark.parametrize("pad,offset", [((0, 16), (0, 0)), ((3, 0), (0, 0)), ((0, 5), (1, 3)), ((16, 16), (16, 32)),
                                        ((1, 1), (7, 8))])
def test_layouts(M, N, K, pad, offset):
    for x in ("int8", "fp16"):
        a, w, ws, xs = inputs(M, N, K, x, K, pad, offset)
        for dt in (torch.float32, torch.bfloat16):
            out, untouched = fused_ref.inside(M, N, dt, pad[0], offset[0])
            xg.gemm_scaled(a, w, ws, xs, out=out)
            check(a, w, ws, xs, out)
            untouched()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 20, 300])
def test_extremes_are_exact(M):
    """The largest sums that 32 bits hold: -128 * -128 in every place."""
    for K, N in ((131071, 9), (131056, 40)):
        a = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
        w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
        w[1::2] = 127
        ones = torch.ones(max(M, N), device="cuda")
        out = xg.gemm_scaled(a, w, ones[:N], ones[:M])
        expect = torch.full((N,), 16384.0 * K, dtype=torch.float64, device="cuda")
        expect[1::2] = -16256.0 * K
        assert torch.equal(out, expect.float().expand(M, N))


@pytest.mark.gpu
@pytest.mark.parametrize("x", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("R,K", [(1, 1), (2, 7), (3, 8), (5, 1001), (300, 64), (7, 4096), (3, 20001), (1, 40000)])
def test_rows(R, K, x):
    for pad, offset in ((0, 0), (3, 1), (16, 8)):
        a = fused_ref.matrix(R, K, TORCH[x], K, pad, offset, 3.0)
        q, scales = fused_ref.scaled_rows(a)
        out, untouched = fused_ref.inside(R, K, torch.int8, pad, offset)
        xg.scaled_rows(a, out=(out, torch.empty(R, device="cuda")))
        untouched()
        got = xg.scaled_rows(a)
        assert torch.equal(out.cpu(), q) and torch.equal(got[0].cpu(), q) and torch.equal(got[1].cpu(), scales)
        back = got[0].double() * got[1].double()[:, None]
        assert bool(((back - a.double()).abs() <= got[1].double()[:, None] * (0.5 + 127 * 2.0 ** -22)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("x", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("K", [5, 300, 5000])
def test_rows_without_a_scale(x, K):
    a = fused_ref.matrix(8, K, TORCH[x], 1)
    a[0] = 0.0
    a[1, K // 2] = INF
    a[2, K - 1] = math.nan
    a[3] = -INF
    a[4] = torch.finfo(TORCH[x]).smallest_normal * torch.finfo(TORCH[x]).eps     # the type's smallest number
    a[5] = torch.finfo(TORCH[x]).max
    a[6, 1:] = torch.finfo(TORCH[x]).min
    q, scales = xg.scaled_rows(a)
    eq, es = fused_ref.scaled_rows(a)
    assert torch.equal(q.cpu(), eq)
    assert bool(((scales.cpu() == es) | (scales.cpu().isnan() & es.isnan())).all())
    assert q[1:4].count_nonzero() == 0 and bool(scales[1:4].isnan().all())
    w, ws = fused_ref.matrix(33, K, torch.int8, 2), torch.ones(33, device="cuda")
    y = xg.gemm_scaled(a, w, ws, out=torch.empty(8, 33, device="cuda"))
    assert bool(y[1:4].isnan().all()) and bool((y[0] == 0).all()) and not bool(y[7].isnan().any())


@pytest.mark.gpu
def test_ties_go_to_the_even_number():
    a = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5]], device="cuda")
    for t in (torch.float32, torch.float16):
        q, s = xg.scaled_rows(a.to(t))
        assert q.cpu().tolist() == [[127, 0, 2, 2, 0, -2, -2, 126]] and float(s) == 1.0


@pytest.mark.gpu
def test_empty():
    for M, N, K in ((0, 4, 8), (4, 0, 8), (3, 5, 0)):
        a, w, ws, xs = inputs(M, N, K)
        out = torch.full((M, N), 7.0, device="cuda")
        xg.gemm_scaled(a, w, ws, xs, out=out)
        assert bool((out == 0).all())
        xg.gemm_scaled(a.float(), w, ws, out=out)
        assert bool((out == 0).all())
    q, s = xg.scaled_rows(torch.empty(0, 5, device="cuda"))
    assert q.shape == (0, 5) and s.shape == (0,)
    q, s = xg.scaled_rows(torch.empty(4, 0, device="cuda"))
    assert torch.equal(s.cpu(), torch.full((4,), 2.0 ** -126))


def test_refusals():
    a, w = torch.zeros(2, 8, dtype=torch.int8), torch.zeros(3, 8, dtype=torch.int8)
    s2, s3 = torch.zeros(2), torch.zeros(3)
    with pytest.raises(ValueError, match="one GPU"):
        xg.gemm_scaled(a, w, s3, s2)
    for args in ((a, w, s3, None), (a.float(), w, s3, s2), (a, w[:, 1:], s3, s2), (a[0], w, s3, s2)):
        with pytest.raises(ValueError):
            xg.gemm_scaled(*args)
    for args in ((a.int(), w, s3, s2), (a, w.float(), s3, s2), (a.double(), w, s3)):
        with pytest.raises(TypeError):
            xg.gemm_scaled(*args)
    with pytest.raises(ValueError, match="131071"):
        xg.gemm_scaled(torch.zeros(1, 131072, dtype=torch.int8), torch.zeros(1, 131072, dtype=torch.int8), s3[:1], s2[:1])
    with pytest.raises(TypeError):
        xg.gemm_scaled(a, w, s3, s2, out=torch.zeros(2, 3, dtype=torch.float64))
    with pytest.raises(TypeError):
        xg.scaled_rows(a)
    with pytest.raises(ValueError):
        xg.scaled_rows(s2)


def test_status_without_a_gpu():
    """Checked before anything is launched."""
    bad = xg.XGEMM_ERR_INVALID_ARG
    assert xg.xgemm_scaled_run(None, 1, 1, 1, None, 1, None, None, 1, None, None, 1, 3, 2, None) == bad
    assert xg.xgemm_scaled_rows(None, 1, 1, None, 1, None, 1, None, 2, None) == bad


@pytest.mark.gpu
def test_statuses():
    h = xg.handle(0)
    t = torch.zeros(4096, device="cuda")
    p = t.data_ptr()
    ok = [h, 4, 5, 16, p, 16, p, p, 16, p, p, 5, xg.XGEMM_INT8, xg.XGEMM_FP32, None]
    assert xg.xgemm_scaled_run(*ok) == xg.XGEMM_OK
    for at, value in ((1, -1), (2, -1), (3, -1), (3, 131072), (1, 2 ** 30 + 1), (2, 2 ** 22 + 1), (4, None), (5, 15), (6, None),
                      (7, None), (8, 15), (9, None), (10, None), (11, 4), (12, 4), (12, -1), (12, xg.XGEMM_BF16), (13, 3)):
        args = list(ok)
        args[at] = value
        assert xg.xgemm_scaled_run(*args) == xg.XGEMM_ERR_INVALID_ARG, (at, value)
    ok = [h, 4, 8, p, 8, p, 8, p, xg.XGEMM_FP16, None]
    assert xg.xgemm_scaled_rows(*ok) == xg.XGEMM_OK
    for at, value in ((1, -1), (2, -1), (3, None), (4, 7), (5, None), (6, 7), (7, None), (8, 3), (8, -1)):
        args = list(ok)
        args[at] = value
        assert xg.xgemm_scaled_rows(*args) == xg.XGEMM_ERR_INVALID_ARG, (at, value)
    torch.cuda.synchronize()
