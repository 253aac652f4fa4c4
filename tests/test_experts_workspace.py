"""The workspace that a layer of experts asks for is what the call uses."""
import pytest
import torch

from paper_2609_16389_amd import xgemm as xg
from test_experts import check, make

pytestmark = pytest.mark.gpu


def run(h, args, top, out):
    x, scores, up, down = args
    (T, H), (E, _, I) = x.shape, down.shape
    return xg.xgemm_experts_run(h, T, E, top, H, I, x.data_ptr(), H, scores.data_ptr(), E, up.data_ptr(), H, 2 * I * H,
                                down.data_ptr(), I, H * I, out.data_ptr(), H, 1, xg.XGEMM_BF16, xg.XGEMM_OUT_FP32, None)


@pytest.mark.parametrize("shape,limit", [
    # one part, no partial sums: 2 x 2 x 64 inner values of 6 bytes and tables
    ((2, 4, 2, 20, 12), 8192),
    # 3 tokens, 2 x 64 inner values each, 3000 columns that fill the GPU in one part
    ((3, 8, 2, 3000, 64), 16384),
    # a full chunk and one token after it
    ((65, 4, 1, 2048, 20), 1 << 20),
])
def test_a_limit_that_the_call_keeps(shape, limit):
    T, E, top, H, I = shape
    args = make(T, E, H, I, "bf16", 51)
    out = torch.empty((T, H), device="cuda")
    torch.cuda.synchronize()
    h = xg.xgemm_create()
    assert xg.xgemm_set_workspace_limit(h, limit) == xg.XGEMM_OK
    assert run(h, args, top, out) == xg.XGEMM_OK, xg.xgemm_last_error(h)
    torch.cuda.synchronize()
    check(out, args, top, True, "bf16", "limit")
    assert xg.xgemm_destroy(h) == xg.XGEMM_OK


@pytest.mark.parametrize("shape", [(1, 16, 8, 200, 1024), (64, 8, 2, 512, 512), (70, 8, 2, 200, 1500), (130, 16, 8, 64, 600)])
def test_chunks_with_partial_sums(shape):
    """Chunks of another size than the first, each cut into parts of its own."""
    T, E, top, H, I = shape
    args = make(T, E, H, I, "bf16", 52)
    out = torch.empty((T, H), device="cuda")
    for _ in range(2):
        assert torch.equal(xg.experts(*args, top, out=out), xg.experts(*args, top, out=torch.empty_like(out)))
    check(out, args, top, True, "bf16", "parts")
