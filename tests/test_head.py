"""Log probabilities from a head's weights and their gradient against 64 bits
(bounds: fused_ref.py)."""
import math

import pytest
import torch

import fused_ref
from paper_2609_16389_amd import xgemm as xg

TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16}
INF = float("inf")


def inputs(T, V, H, dtype, seed=0, pad=(0, 0), offset=(0, 0)):
    dt = TORCH[dtype]
    x = fused_ref.matrix(T, H, dt, seed, pad[0], offset[0])
    w = fused_ref.matrix(V, H, dt, seed + 1, pad[1], offset[1], 2.0 / math.sqrt(max(H, 1)))
    targets = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(seed + 2)).cuda()
    return x, w, targets


SHAPES = [(1, 1, 1), (1, 2, 8), (2, 127, 7), (3, 129, 64), (1, 4099, 65), (16, 300, 130), (64, 1000, 200), (77, 5001, 72),
          (130, 257, 520), (300, 700, 33), (2053, 4100, 72), (1024, 8192, 64), (333, 3001, 1001), (20, 2003, 515)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,H", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_shapes(T, V, H, dtype):
    x, w, targets = inputs(T, V, H, dtype, T + V + H)
    targets[:: 5] = -100
    if T > 2:
        targets[1], targets[2] = V, V - 1
    ref = fused_ref.head(x, w, targets)
    out = xg.head_logprobs(x, w, targets)
    for name in ("lse", "logprob"):
        fused_ref.check(out[name], *ref[name], name)
    assert list(xg.head_logprobs(x, w)) == ["lse"]
    for name in ("lse", "logprob"):
        one = {name: torch.empty(T, device="cuda")}
        xg.head_logprobs(x, w, targets, out=one)
        assert torch.equal(one[name].nan_to_num(3.0), out[name].nan_to_num(3.0))


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,H", [(5, 333, 71), (40, 1000, 96), (200, 130, 333)])
@pytest.mark.parametrize("pad,offset", [((3, 5), (1, 3)), ((8, 16), (8, 16)), ((0, 1), (7, 0)), ((0, 8), (0, 0))])
def test_layouts(T, V, H, pad, offset):
    for dtype in ("bf16", "fp16"):
        x, w, targets = inputs(T, V, H, dtype, H, pad, offset)
        ref = fused_ref.head(x, w, targets)
        out = xg.head_logprobs(x, w, targets)
        for name in ref:
            fused_ref.check(out[name], *ref[name], name)
        d = torch.full((T,), -1.0 / T, device="cuda")
        grad = fused_ref.head_grad(x, w, targets, out["lse"], d, None, x.dtype)
        got = [fused_ref.inside(T, H, x.dtype, pad[0], offset[0]), fused_ref.inside(V, H, x.dtype, pad[1], offset[1])]
        xg.head_logprobs_grad(x, w, targets, out["lse"], d, out=(got[0][0], got[1][0]))
        for (t, untouched), (value, bound), name in zip(got, grad, ("d_x", "d_head")):
            fused_ref.check(t, value, bound, name)
            untouched()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T", [4, 600])
def test_rows_that_are_not_ordinary(T, dtype):
    """Logits of -inf, +inf and NaN, of one sign and of both."""
    V, H = 1500, 16
    x = torch.zeros(T, H, dtype=TORCH[dtype], device="cuda")
    w = torch.zeros(V, H, dtype=TORCH[dtype], device="cuda")
    w[:, 0], w[3, 0], w[:, 1] = 1.0, 2.0, torch.arange(V, device="cuda") % 2
    x[0, 0] = -INF                # every logit -inf (0 * inf is left out: the other columns of w are zeros)
    w[:, 2:] = 1.0
    x[1, 0] = INF
    x[2, 1] = -INF                # 0 * -inf: NaN
    x[3, 5] = math.nan
    targets = torch.full((T,), 3, device="cuda")
    out = xg.head_logprobs(x, w, targets)
    lse, lp = out["lse"].cpu(), out["logprob"].cpu()
    assert lse[0] == -INF and lp[0] == -INF
    assert bool(lse[1:4].isnan().all()) and bool(lp[1:4].isnan().all())
    if T > 4:
        assert bool((lse[4:] - math.log(V)).abs().max() < 1e-5) and bool((lp[4:] + math.log(V)).abs().max() < 1e-5)
    d = torch.ones(T, device="cuda")
    dx, dw = xg.head_logprobs_grad(x, w, targets, out["lse"], d, d)
    assert bool((dx[0] == 0).all()) and bool(dx[1:4].isnan().all())
    assert not bool(dx[4:].isnan().any())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("size", [40.0, 3000.0])
def test_large_logits(dtype, size):
    """Logits far from zero, of which one carries nearly everything."""
    T, V, H = 33, 700, 40
    x, w, targets = inputs(T, V, H, dtype, 5)
    x = (x.float() * size).to(x.dtype)
    ref = fused_ref.head(x, w, targets)
    out = xg.head_logprobs(x, w, targets)
    for name in ref:
        fused_ref.check(out[name], *ref[name], name)


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,H", [(1, 1, 1), (2, 127, 7), (3, 129, 64), (77, 5001, 72), (130, 257, 520), (300, 700, 33),
                                   (1030, 4100, 72), (4100, 2309, 40), (64, 3001, 2048), (333, 3001, 1001)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gradient(T, V, H, dtype):
    x, w, targets = inputs(T, V, H, dtype, T + V + H)
    targets[:: 5] = -100
    lse = xg.head_logprobs(x, w)["lse"]
    g = torch.Generator().manual_seed(3)
    d = (torch.randn(T, generator=g) / T).cuda()
    z = (torch.randn(T, generator=g) * 1e-3 / T).cuda()
    for dl, ds in ((d, None), (None, z), (d, z)):
        for out in (x.dtype, torch.float32):
            ref = fused_ref.head_grad(x, w, targets, lse, dl, ds, out)
            got = xg.head_logprobs_grad(x, w, targets if dl is not None else None, lse, dl, ds,
                                        out=(torch.empty(T, H, dtype=out, device="cuda"),
                                             torch.empty(V, H, dtype=out, device="cuda")))
            for t, (value, bound), name in zip(got, ref, ("d_x", "d_head")):
                fused_ref.check(t, value, bound, name)
    both = xg.head_logprobs_grad(x, w, targets, lse, d, z)
    for at in (0, 1):
        one = [torch.empty_like(t) for t in both]
        one[1 - at] = None
        xg.head_logprobs_grad(x, w, targets, lse, d, z, out=tuple(one))
        assert torch.equal(one[at], both[at])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gradient_in_pieces(dtype):
    """So many rows that the vocabulary is taken in several pieces, the last odd."""
    T, V, H = 40000, 9001, 24
    x, w, targets = inputs(T, V, H, dtype, 4)
    targets[:: 7] = -1
    lse = xg.head_logprobs(x, w)["lse"]
    d = torch.full((T,), -1.0 / T, device="cuda")
    for out in (x.dtype, torch.float32):
        ref = fused_ref.head_grad(x, w, targets, lse, d, None, out)
        got = xg.head_logprobs_grad(x, w, targets, lse, d, out=(torch.empty(T, H, dtype=out, device="cuda"),
                                                                torch.empty(V, H, dtype=out, device="cuda")))
        # (d_x is summed over the pieces: some roundings more than one sum has, which its n + 32 covers)
        for t, (value, bound), name in zip(got, ref, ("d_x", "d_head")):
            fused_ref.check(t, value, bound, name)
        del ref, got


@pytest.mark.gpu
def test_many_rows():
    """More rows than their statistics are kept for at a time."""
    T, V, H = 16384 * 2 + 3, 300, 16
    x, w, targets = inputs(T, V, H, "bf16", 8)
    ref = fused_ref.head(x, w, targets)
    out = xg.head_logprobs(x, w, targets)
    for name in ref:
        fused_ref.check(out[name], *ref[name], name)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** -20, 2.0 ** 20])
def test_gradient_of_any_size_in_binary16(size):
    x, w, targets = inputs(50, 900, 48, "fp16", 9)
    lse = xg.head_logprobs(x, w)["lse"]
    d = torch.full((50,), size, device="cuda")
    ref = fused_ref.head_grad(x, w, targets, lse, d, None, torch.float32)
    got = xg.head_logprobs_grad(x, w, targets, lse, d, out=(torch.empty(50, 48, device="cuda"), torch.empty(900, 48, device="cuda")))
    for t, (value, bound), name in zip(got, ref, ("d_x", "d_head")):
        fused_ref.check(t, value, bound, name)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T", [20, 300])
def test_rows_without_a_target_leave_no_trace(T, dtype):
    """Whatever their d_logprob holds."""
    x, w, targets = inputs(T, 700, 40, dtype, 6)
    targets[:: 3] = -100
    lse = xg.head_logprobs(x, w)["lse"]
    clean = torch.full((T,), -1.0 / T, device="cuda")
    d = clean.clone()
    d[0], d[3], d[6], d[9] = 1e30, -INF, math.nan, 1e-30
    ref = xg.head_logprobs_grad(x, w, targets, lse, clean)
    got = xg.head_logprobs_grad(x, w, targets, lse, d)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    assert bool((got[0][:: 3] == 0).all())


@pytest.mark.gpu
def test_gradient_against_differences():
    T, V, H = 11, 60, 24
    x, w, targets = inputs(T, V, H, "bf16", 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(s, dtype=torch.float64, device="cuda", generator=g)  # noqa: E731
    d, z, vx, vw = rand(T), rand(T), rand(T, H), rand(V, H)
    lse = xg.head_logprobs(x, w)["lse"]
    dx, dw = xg.head_logprobs_grad(x, w, targets, lse, d.float(), z.float(),
                                   out=(torch.empty(T, H, device="cuda"), torch.empty(V, H, device="cuda")))

    def total(t):
        a = (x.double() + t * vx) @ (w.double() + t * vw).t().contiguous()
        lse = torch.logsumexp(a, 1)
        return float((d * (a.gather(1, targets[:, None])[:, 0] - lse) + z * lse).sum())

    t = 1e-5
    slope = (total(t) - total(-t)) / (2 * t)
    got = float((dx.double() * vx).sum() + (dw.double() * vw).sum())
    size = float((dx.double() * vx).abs().sum() + (dw.double() * vw).abs().sum())
    assert abs(got - slope) <= 2 * 2.0 ** -8 * size   # (d is rounded to bfloat16, its terms of either sign)


@pytest.mark.gpu
def test_empty():
    new = lambda *s: torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert xg.head_logprobs(new(0, 8), new(5, 8), none)["lse"].shape == (0,)
    out = xg.head_logprobs(new(3, 0), new(5, 0), torch.tensor([0, -1, 4], device="cuda"))
    assert bool((out["lse"] - math.log(5)).abs().max() < 1e-6)
    assert bool((out["logprob"].cpu() - torch.tensor([-math.log(5), 0.0, -math.log(5)])).abs().max() < 1e-6)
    f = torch.empty(0, device="cuda")
    dx, dw = xg.head_logprobs_grad(new(0, 8), new(5, 8), none, f, f, out=(new(0, 8), new(5, 8)))
    assert bool((dw == 0).all())
    dx, dw = xg.head_logprobs_grad(new(2, 8), new(5, 8), None, torch.ones(2, device="cuda"), out=(new(2, 8), new(5, 8)))
    assert bool((dx == 0).all()) and bool((dw == 0).all())


def test_refusals():
    b = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    x, w, t, f = b(2, 8), b(5, 8), torch.zeros(2, dtype=torch.int64), torch.zeros(2)
    with pytest.raises(ValueError, match="one GPU"):
        xg.head_logprobs(x, w, t)
    for args in ((x, w[:, 1:]), (x[0], w), (x, w[:0])):
        with pytest.raises(ValueError):
            xg.head_logprobs(*args)
    with pytest.raises(ValueError, match="targets"):
        xg.head_logprobs(x, w, out={"logprob": f})
    for args in ((x.float(), w.float()), (x, w.half())):
        with pytest.raises(TypeError):
            xg.head_logprobs(*args)
    for args in ((x, w, t, None, f), (x, w, None, f, f)):
        with pytest.raises(ValueError):
            xg.head_logprobs_grad(*args)
    with pytest.raises(ValueError):
        xg.head_logprobs_grad(x, w, t, f, f, out=(None, None))


def test_status_without_a_gpu():
    bad = xg.XGEMM_ERR_INVALID_ARG
    assert xg.xgemm_head_run(None, 1, 1, 1, None, 1, None, 1, None, None, None, 0, None) == bad
    assert xg.xgemm_head_grad(None, 1, 1, 1, None, 1, None, 1, None, None, None, None, None, 1, None, 1, 0, 0, None) == bad


@pytest.mark.gpu
def test_shapes_and_statuses_are_checked():
    b = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    x, w, t, f = b(2, 8), b(5, 8), torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(2, device="cuda")
    for kw in ({"targets": t[:1]}, {"targets": t.int()}, {"out": {"lse": f[:1]}}, {"out": {"lse": f.half()}}):
        with pytest.raises(ValueError):
            xg.head_logprobs(x, w, **kw)
    for out in ((b(2, 7), None), (None, b(4, 8)), (b(8, 2).t(), None)):
        with pytest.raises(ValueError):
            xg.head_logprobs_grad(x, w, t, f, f, out=out)
    h, p = xg.handle(0), torch.zeros(4096, device="cuda").data_ptr()
    ok = [h, 2, 5, 8, p, 8, p, 8, p, p, p, 0, None]
    assert xg.xgemm_head_run(*ok) == xg.XGEMM_OK
    for at, value in ((1, -1), (2, 0), (2, 2 ** 22 + 1), (3, -1), (4, None), (5, 7), (6, None), (7, 7), (8, None), (11, 2)):
        args = list(ok)
        args[at] = value
        assert xg.xgemm_head_run(*args) == xg.XGEMM_ERR_INVALID_ARG, (at, value)
    ok = [h, 2, 5, 8, p, 8, p, 8, p, p, p, p, p, 8, p, 8, 0, 1, None]
    assert xg.xgemm_head_grad(*ok) == xg.XGEMM_OK
    for at, value in ((1, -1), (2, 0), (3, -1), (4, None), (5, 7), (6, None), (7, 7), (8, None), (9, None), (13, 7), (15, 7),
                      (16, 2), (17, 2)):
        args = list(ok)
        args[at] = value
        assert xg.xgemm_head_grad(*args) == xg.XGEMM_ERR_INVALID_ARG, (at, value)
    torch.cuda.synchronize()
