"""Products with 4-bit weights against the plain form in 64 bits.

Bound: |y - exact| <= (K / 32 + 96) 2^-24 S + rounding of the output, S the
sum of the absolute products (16 + q) x s and (16 + z) x s.  The products are
exact; an output passes through at most K / 32 / 8 + 8 sequential
accumulations of matrix products, whose 32 terms add at most 32 roundings
each time counted on their own part of S (hence 32 + 64 for the chain's and
the joins' own), three operations a group and 8 joins of waves.
"""
import numpy as np
import pytest
import torch

import decode_ref
from paper_2609_16389_amd import xgemm as xg

TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def make(M, N, K, dtype, group, zeros, seed, pad=0, device="cuda"):
    """x, q, scales, zeros as GPU views of wider arrays filled with what must
    not be read."""
    rng = np.random.default_rng(seed)
    dt, width, G = TORCH[dtype], (K + 1) // 2, -(-K // group)

    def view(t, fill):
        buf = torch.full((t.shape[0] * (t.shape[1] + pad) + pad,), fill, dtype=t.dtype, device=device)
        v = buf.as_strided(t.shape, (t.shape[1] + pad, 1), pad)
        v.copy_(t)
        return v

    x = view(torch.from_numpy(rng.normal(size=(M, K)).astype(np.float32)).to(dt).to(device), float("nan"))
    q = view(torch.from_numpy(rng.integers(0, 256, size=(N, width), dtype=np.uint8)).to(device), 255)
    s = view(torch.from_numpy(rng.uniform(0.5, 1.5, size=(N, G)).astype(np.float32)).to(dt).to(device), float("nan"))
    z = None
    if zeros:
        z = view(torch.from_numpy(rng.integers(0, 16, size=(N, G), dtype=np.uint8)).to(device), 255)
    return x, q, s, z


def host(t):
    return None if t is None else t.cpu().float().numpy() if t.is_floating_point() else t.cpu().numpy()


def check(y, x, q, s, z, group, K, dtype, what):
    ref, S = decode_ref.quant(host(x), host(q), host(s), host(z), group, K)
    got = y.cpu().double().numpy()
    tol = (K / 32 + 96) * 2.0 ** -24 * S
    if y.dtype != torch.float32:
        tol = tol * (1 + EPS[dtype]) + EPS[dtype] * np.abs(ref) + 2.0 ** -24
    assert np.all(np.abs(got - ref) <= tol), "%s: off by %.3g of the bound" % (what, np.max(np.abs(got - ref) / tol))


SHAPES = [(1, 1, 1), (1, 16, 32), (2, 17, 33), (1, 64, 127), (3, 100, 128), (1, 33, 255), (5, 47, 257), (16, 64, 512),
          (17, 40, 513), (32, 33, 1000), (33, 80, 2047), (64, 130, 2049), (65, 31, 300), (130, 48, 4100), (1, 5, 70001)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True), (128, False), (384, True)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%dx%dx%d" % s)
def test_shapes(shape, group, zeros, dtype):
    M, N, K = shape
    for pad in (0, 3):
        x, q, s, z = make(M, N, K, dtype, group, zeros, M + 2 * N + 3 * K, pad)
        for out in (torch.float32, TORCH[dtype]):
            buf = torch.full((M + 1, N + 5), 77.0, dtype=out, device="cuda")
            y = xg.gemv_quant(x, q, s, z, group, out=buf[:M, 2:N + 2])
            check(y, x, q, s, z, group, K, dtype, "pad %d %s" % (pad, out))
            # nothing beside y is written
            assert torch.all(buf[M] == 77) and torch.all(buf[:, :2] == 77) and torch.all(buf[:, N + 2:] == 77)


@pytest.mark.gpu
def test_default_output_and_determinism():
    x, q, s, z = make(7, 500, 3000, "bf16", 64, True, 5)
    y = xg.gemv_quant(x, q, s, z, 64)
    assert y.dtype == torch.float32
    for _ in range(3):
        assert torch.equal(xg.gemv_quant(x, q, s, z, 64), y)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_exact_where_sums_are_whole_numbers(dtype):
    """Every value of q against every zero point, x and s powers of two."""
    K = 512
    q = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(256, 1)
    z = torch.arange(256, dtype=torch.uint8, device="cuda")[:, None].repeat(1, K // 32).contiguous()
    s = torch.full((256, K // 32), 0.5, dtype=TORCH[dtype], device="cuda")
    x = torch.ones((2, K), dtype=TORCH[dtype], device="cuda")
    x[1, ::2] = -2.0
    ref, _ = decode_ref.quant(host(x), host(q), host(s), host(z), 32, K)
    assert np.array_equal(xg.gemv_quant(x, q, s, z, 32).cpu().double().numpy(), ref)


@pytest.mark.gpu
def test_rows_with_nan_and_infinity_stay_apart():
    x, q, s, z = make(4, 100, 1000, "bf16", 128, False, 6)
    clean = xg.gemv_quant(x, q, s, z)
    x[1, 999], x[2, 0] = float("nan"), float("inf")
    y = xg.gemv_quant(x, q, s, z)
    assert torch.equal(y[0], clean[0]) and torch.equal(y[3], clean[3])
    assert torch.all(torch.isnan(y[1])) and torch.all(torch.isnan(y[2]))


@pytest.mark.gpu
def test_empty():
    x, q, s, z = make(3, 5, 40, "fp16", 32, True, 7)
    out = torch.full((3, 5), float("nan"), device="cuda")
    assert torch.all(xg.gemv_quant(x[:, :0], q[:, :0], s[:, :0], z[:, :0], 32, out=out) == 0)
    assert xg.gemv_quant(x[:0], q, s, z, 32).shape == (0, 5)
    assert xg.gemv_quant(x, q[:0], s[:0], z[:0], 32).shape == (3, 0)


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Rows of q, x and y whose byte offsets pass 2^32."""
    K, N = 256, 5
    x, q, s, z = make(3, N, K, "bf16", 128, False, 8)
    far = torch.empty(((N - 1) * (1 << 30) + 200,), dtype=torch.uint8, device="cuda").as_strided((N, K // 2), (1 << 30, 1), 7)
    far.copy_(q)
    out = torch.empty((2 * (1 << 30) + 10,), dtype=torch.float32, device="cuda").as_strided((3, N), (1 << 30, 1), 1)
    assert torch.equal(xg.gemv_quant(x, far, s, out=out), xg.gemv_quant(x, q, s))


@pytest.mark.gpu
def test_on_another_stream():
    x, q, s, z = make(8, 300, 2000, "fp16", 64, True, 9)
    y = xg.gemv_quant(x, q, s, z, 64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2 = xg.gemv_quant(x, q, s, z, 64, stream=side)
    side.synchronize()
    assert torch.equal(y, y2)


@pytest.mark.gpu
def test_replayed_from_a_graph():
    x, q, s, z = make(4, 300, 2000, "bf16", 128, False, 10)
    out = torch.empty((4, 300), device="cuda")
    xg.gemv_quant(x, q, s, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xg.gemv_quant(x, q, s, out=out)
    for seed in range(3):
        x.copy_(torch.randn(4, 2000, device="cuda"))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, xg.gemv_quant(x, q, s))


def test_refusals_without_a_gpu():
    x, q, s, z = make(2, 5, 70, "bf16", 32, True, 1, device="cpu")
    with pytest.raises(ValueError):
        xg.gemv_quant(x, q, s, z, 32)                         # not on a GPU
    with pytest.raises(TypeError):
        xg.gemv_quant(x.float(), q, s, z, 32)
    with pytest.raises(ValueError):
        xg.gemv_quant(x, q, s, z, 48)                         # no group size
    with pytest.raises(ValueError):
        xg.gemv_quant(x, q, s, z, 64)                         # scales of another group
    with pytest.raises(ValueError):
        xg.gemv_quant(x, q[:, 1:], s, z, 32)
    with pytest.raises(ValueError):
        xg.gemv_quant(x, q, s.half(), z, 32)
    with pytest.raises(ValueError):
        xg.gemv_quant(x, q, s, z.int(), 32)
    with pytest.raises(ValueError):
        xg.gemv_quant(x, q, s, z, 32, out=torch.empty(5, 2))
    assert xg.xgemv_quant_run(None, 1, 1, 1, 16, 1, 16, 1, 16, 1, None, 0, 32, 16, 1, 0, 0, None) == \
        xg.XGEMM_ERR_INVALID_ARG


@pytest.mark.gpu
def test_refusals_of_the_c_call():
    h = xg.handle()
    x, q, s, z = make(2, 5, 70, "bf16", 32, True, 1)
    y = torch.full((2, 5), 7.0, device="cuda")

    def call(M=2, N=5, K=70, x_=x.data_ptr(), ldx=70, q_=q.data_ptr(), ldq=35, s_=s.data_ptr(), lds=3,
             z_=z.data_ptr(), ldz=3, group=32, y_=y.data_ptr(), ldy=5, dtype=0, out=0):
        return xg.xgemv_quant_run(h, M, N, K, x_, ldx, q_, ldq, s_, lds, z_, ldz, group, y_, ldy, dtype, out, None)

    bad = [dict(M=-1), dict(N=-1), dict(K=-1), dict(M=1 << 31), dict(x_=None), dict(q_=None), dict(s_=None),
           dict(y_=None), dict(ldx=69), dict(ldq=34), dict(lds=2), dict(ldz=2), dict(ldy=4), dict(group=0),
           dict(group=96), dict(group=-128), dict(group=200), dict(dtype=2), dict(out=2), dict(ldx=1 << 62)]
    for b in bad:
        assert call(**b) == xg.XGEMM_ERR_INVALID_ARG, b
    torch.cuda.synchronize()
    assert torch.all(y == 7)
    assert call() == xg.XGEMM_OK and call(z_=None, ldz=0) == xg.XGEMM_OK and call(M=0, y_=None, x_=None) == xg.XGEMM_OK
    with pytest.raises(ValueError):
        xg.gemv_quant(x, q.t().contiguous().t(), s, z, 32)    # rows not contiguous


def test_kernels_use_no_scratch(tmp_path):
    """None of the library's kernels has a private segment, those of every
    source file included (a code object each): the runtime allocates scratch
    memory at the first launch of one that does."""
    import os
    import re
    import shutil
    import subprocess
    bundler = "/opt/rocm/llvm/bin/clang-offload-bundler"
    readelf = "/opt/rocm/llvm/bin/llvm-readelf"
    if not (shutil.which("objcopy") and os.path.exists(bundler) and os.path.exists(readelf)):
        pytest.skip("objcopy / clang-offload-bundler / llvm-readelf not available")
    fat = tmp_path / "fat.bin"
    subprocess.run(["objcopy", "-O", "binary", "--only-section=.hip_fatbin", xg._LIB_PATH, str(fat)], check=True)
    data = fat.read_bytes()
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)]
    names = []
    for i, (a, b) in enumerate(zip(starts, starts[1:] + [len(data)])):
        part, co = tmp_path / ("part%d" % i), tmp_path / ("%d.co" % i)
        part.write_bytes(data[a:b])
        subprocess.run([bundler, "--unbundle", "--type=o", "--input=" + str(part),
                        "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", "--output=" + str(co)], check=True)
        notes = subprocess.run([readelf, "--notes", str(co)], check=True, capture_output=True, text=True).stdout
        symbols = re.findall(r"\.symbol:\s+(\S+)\.kd", notes)
        sizes = [int(v) for v in re.findall(r"\.private_segment_fixed_size:\s+(\d+)", notes)]
        assert len(sizes) == len(symbols)
        assert all(v == 0 for v in sizes), [(n, v) for n, v in zip(symbols, sizes) if v]
        names += symbols
    for part in ("quant_kernel", "route_up", "down_sum", "logprob_rows", "logprob_grad", "gemm_kernel_dma"):
        assert any(part in n for n in names), part


@pytest.mark.gpu
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True), (256, False)])
@pytest.mark.parametrize("shape", [(2, 8300, 300), (3, 8300, 257), (16, 8209, 700), (30, 12290, 640), (17, 12305, 129),
                                   (64, 12289, 1100), (40, 12301, 96), (100, 6200, 515)], ids=lambda s: "%dx%dx%d" % s)
def test_many_columns(shape, group, zeros):
    """The kernels that share rows between waves over columns."""
    M, N, K = shape
    for dtype, pad in (("bf16", 0), ("fp16", 3)):
        x, q, s, z = make(M, N, K, dtype, group, zeros, M + 2 * N + 3 * K, pad)
        check(xg.gemv_quant(x, q, s, z, group), x, q, s, z, group, K, dtype, "pad %d" % pad)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 20])
def test_rows_far_apart(M):
    """Rows of weights at distances past 27 and past 32 bits."""
    x, q, s, z = make(M, 3, 700, "bf16", 64, True, 8)
    for ld in (2 ** 27 + 8, 2 ** 31 + 24):
        far = torch.empty(2 * ld + 350, dtype=torch.uint8, device="cuda").as_strided((3, 350), (ld, 1))
        far.copy_(q)
        check(xg.gemv_quant(x, far, s, z, 64), x, q, s, z, 64, 700, "bf16", "ld %d" % ld)
        del far
