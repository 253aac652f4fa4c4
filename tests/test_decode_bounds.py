"""What the operators around a decoding step leave alone: outputs lie as views
inside larger buffers of a known pattern, of which everything but the views has
to be unchanged after the call, and the views written whole."""
import pytest
import torch

from paper_2609_16389_amd import xgemm as xg

MARK = {torch.float32: 12345.0, torch.bfloat16: 12352.0, torch.float16: 12344.0, torch.int64: 1234567890123}


class Inside:
    """Views inside buffers of MARK, and the check that the rest still holds it."""

    def __init__(self):
        self.made = []

    def view(self, rows, cols, dtype, ld=None, before=64, after=4096):
        ld = ld or cols
        buf = torch.full((before + rows * ld + after,), MARK[dtype], dtype=dtype, device="cuda")
        v = buf.as_strided((rows, cols), (ld, 1), before)
        self.made.append((buf, v, before, rows, cols, ld))
        return v

    def vector(self, n, dtype=torch.float32):
        return self.view(1, n, dtype)[0]

    def check(self):
        torch.cuda.synchronize()
        for buf, v, before, rows, cols, ld in self.made:
            outside = torch.ones(buf.shape, dtype=torch.bool, device="cuda")
            outside.as_strided((rows, cols), (ld, 1), before).fill_(False)
            assert torch.all(buf[outside] == MARK[buf.dtype])
            assert not torch.any(v == MARK[buf.dtype])


def rand(*shape, dtype, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,group", [(1, 17, 300, 32), (2, 8209, 130, 64), (16, 33, 257, 128), (5, 9001, 96, 32),
                                         (17, 129, 511, 64), (33, 65, 1000, 128), (40, 12301, 64, 32), (64, 12289, 200, 128),
                                         (30, 12290, 129, 64)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_quant(M, N, K, group, out):
    x = rand(M, K, dtype=torch.bfloat16)
    q = torch.randint(0, 256, (N, (K + 1) // 2), dtype=torch.uint8, device="cuda")
    s = rand(N, -(-K // group), dtype=torch.bfloat16, seed=1)
    inside = Inside()
    xg.gemv_quant(x, q, s, None, group, out=inside.view(M, N, out, ld=N + 3))
    inside.check()


@pytest.mark.gpu
@pytest.mark.parametrize("T,E,top,H,I", [(1, 5, 2, 65, 33), (2, 40, 4, 130, 64), (7, 13, 3, 101, 77), (16, 9, 4, 250, 136),
                                         (20, 6, 2, 67, 5), (33, 8, 8, 513, 70), (64, 3, 1, 1000, 257)])
@pytest.mark.parametrize("out", [torch.float32, torch.float16])
def test_experts(T, E, top, H, I, out):
    x, scores = rand(T, H, dtype=torch.float16), rand(T, E, dtype=torch.float32, seed=1)
    up, down = rand(E, 2 * I, H, dtype=torch.float16, seed=2), rand(E, H, I, dtype=torch.float16, seed=3) / 64
    inside = Inside()
    y = inside.view(T, H, out, ld=H + 5)
    xg.experts(x, scores, up, down, top, out=y)
    inside.check()


@pytest.mark.gpu
@pytest.mark.parametrize("R,V,top", [(1, 1, 1), (1, 70001, 32), (3, 999, 7), (40, 20000, 5), (700, 130, 3)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_logprobs_and_gradient(R, V, top, dtype):
    logits, targets = rand(R, V, dtype=dtype), torch.randint(0, V, (R,), device="cuda")
    inside = Inside()
    out = {k: inside.vector(R) for k in ("lse", "logprob", "entropy")}
    out["top_logprob"], out["top_id"] = inside.view(R, top, torch.float32), inside.view(R, top, torch.int64)
    xg.logprobs(logits, targets, top=top, out=out)
    inside.check()
    ones = torch.ones(R, device="cuda")
    xg.logprobs_grad(logits, targets, out["lse"], out["entropy"], ones, ones, ones, out=inside.view(R, V, dtype, ld=V + 7))
    inside.check()


@pytest.mark.gpu
def test_experts_far_apart():
    """Matrices, and rows of them, at distances past 32 bits of bytes."""
    T, E, H, I = 3, 3, 130, 70
    x, scores = rand(T, H, dtype=torch.float16), rand(T, E, dtype=torch.float32, seed=1)
    up, down = rand(E, 2 * I, H, dtype=torch.float16, seed=2), rand(E, H, I, dtype=torch.float16, seed=3) / 64
    ref = xg.experts(x, scores, up, down, 3)
    far = 2 ** 31 + 8
    stride = 2 * I * H
    buf = torch.empty(far * 2 + stride, dtype=torch.float16, device="cuda")
    u = buf.as_strided(up.shape, (far, H, 1))
    u.copy_(up)
    assert torch.equal(xg.experts(x, scores, u, down, 3), ref)
    row = far // 100
    d = buf.as_strided(down.shape, (I, row, 1))   # rows far apart, matrices side by side
    d.copy_(down)
    assert torch.equal(xg.experts(x, scores, up, d, 3), ref)


@pytest.mark.gpu
def test_logprobs_far_apart():
    """Rows at a distance past 32 bits of bytes, read and written."""
    R, V, ld = 3, 5000, 2 ** 31 + 24
    logits, targets, ones = rand(R, V, dtype=torch.bfloat16), torch.tensor([0, 7, V - 1], device="cuda"), torch.ones(3, device="cuda")
    ref = xg.logprobs(logits, targets, top=4)
    grad = xg.logprobs_grad(logits, targets, ref["lse"], ref["entropy"], ones, ones, ones)
    far = torch.empty(2 * ld + V, dtype=torch.bfloat16, device="cuda").as_strided((R, V), (ld, 1))
    far.copy_(logits)
    got = xg.logprobs(far, targets, top=4)
    assert all(torch.equal(got[k], ref[k]) for k in ref)
    xg.logprobs_grad(far, targets, ref["lse"], ref["entropy"], ones, ones, ones, out=far)
    assert torch.equal(far, grad)
