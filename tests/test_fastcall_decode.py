"""The native call path of the operators around a decoding step: it declines
what is not plain, and gives what the ctypes path gives."""
import pytest
import torch

from paper_2609_16389_amd import _fastcall
from paper_2609_16389_amd import xgemm as xg


def test_declines_what_is_not_plain():
    a, b = torch.zeros(2, 8).bfloat16(), torch.zeros(2, 8)
    q = torch.zeros(2, 4, dtype=torch.uint8)
    assert _fastcall.gemv_quant(a, q, a[:, :1], None, 32, b[:, :2]) is None            # not on a GPU
    assert _fastcall.gemv_quant(a, q, a[:, :1], None, 32.0, b[:, :2]) is None
    assert _fastcall.gemv_quant(a, q) is None
    assert _fastcall.experts(a, b, a[None], a[None], 1, True, b) is None
    assert _fastcall.experts(a, b, a[None], a[None], 2 ** 70, True, b) is None
    assert _fastcall.logprobs(b, None, 0, {"lse": b[:, 0]}) is None
    assert _fastcall.logprobs(b, None, 0, None) is None
    assert _fastcall.logprobs_grad(b, None, b[:, 0], None, None, None, None, b) is None


@pytest.fixture
def slow(monkeypatch):
    def calls(f):
        with monkeypatch.context() as m:
            for name in ("gemv_quant", "experts", "logprobs", "logprobs_grad"):
                m.setattr(_fastcall, name, lambda *a: None)
            return f()
    return calls


@pytest.mark.gpu
def test_same_as_the_other_path(slow):
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    xg.handle(0, torch.cuda.current_stream())
    x = rand(5, 300).half()[:, :257]
    q = torch.randint(0, 256, (70, 129), dtype=torch.uint8, device="cuda", generator=g)
    s, z = rand(70, 9).half(), torch.randint(0, 16, (70, 9), dtype=torch.uint8, device="cuda", generator=g)
    for zeros in (z, None):
        for dt in (torch.float32, torch.float16):
            call = lambda: xg.gemv_quant(x, q, s, zeros, 32, out=torch.empty(5, 70, dtype=dt, device="cuda"))  # noqa: E731
            assert _fastcall.gemv_quant(x, q, s, zeros, 32, torch.empty(5, 70, dtype=dt, device="cuda")) == xg.XGEMM_OK
            assert torch.equal(call(), slow(call))
    # shapes, types and layouts that do not fit are left to the checks in Python
    out = torch.empty(5, 70, device="cuda")
    for bad in ((x, q, s, z, 48, out), (x, q, s, z, 64, out), (x, q, s.float(), z, 32, out), (x, q, s, z.int(), 32, out),
                (x, q[:, 1:], s, z, 32, out), (x, q, s, z, 32, out[:, 1:]), (x, q, s, z, 32, out.double()),
                (x.float(), q, s, z, 32, out), (x, q, s, z[:1], 32, out)):
        assert _fastcall.gemv_quant(*bad) is None

    x, scores = rand(6, 40).bfloat16(), rand(6, 9)
    up, down = rand(9, 48, 40).bfloat16(), rand(9, 40, 24).bfloat16()
    for flag in (True, False):
        call = lambda: xg.experts(x, scores, up, down, 3, flag, out=torch.empty(6, 40, device="cuda"))  # noqa: E731
        assert _fastcall.experts(x, scores, up, down, 3, flag, torch.empty(6, 40, device="cuda")) == xg.XGEMM_OK
        assert torch.equal(call(), slow(call))
    out = torch.empty(6, 40, device="cuda")
    for bad in ((x, scores, up, down, 10, True, out), (x, scores, up, down, 3, 1, out), (x, scores.half(), up, down, 3, True, out),
                (x, scores, up.half(), down, 3, True, out), (x, scores, up[:, 1:], down, 3, True, out),
                (x, scores, up, down[:8], 3, True, out), (x, scores, up, down, 3, True, out[:5])):
        assert _fastcall.experts(*bad) is None

    logits, t = rand(7, 500), torch.randint(0, 500, (7,), device="cuda", generator=g)
    new = lambda *s, **k: torch.empty(*s, device="cuda", **k)  # noqa: E731
    outs = lambda: {"lse": new(7), "logprob": new(7), "entropy": new(7), "top_logprob": new(7, 4),  # noqa: E731
                    "top_id": new(7, 4, dtype=torch.int64)}
    call = lambda: xg.logprobs(logits, t, 4, out=outs())  # noqa: E731
    assert _fastcall.logprobs(logits, t, 4, outs()) == xg.XGEMM_OK
    a, b = call(), slow(call)
    assert all(torch.equal(a[k], b[k]) for k in b)
    for bad in ((logits, t.int(), 4, outs()), (logits, t, 5, outs()), (logits, None, 4, outs()), (logits, t, 0, outs()),
                (logits, t, 4, {**outs(), "more": new(7)}), (logits.t(), t, 4, outs()),
                (logits, t, 4, {**outs(), "lse": new(14)[::2]})):
        assert _fastcall.logprobs(*bad) is None
    d = rand(7)
    call = lambda: xg.logprobs_grad(logits, t, a["lse"], a["entropy"], d, d, None, out=new(7, 500))  # noqa: E731
    assert _fastcall.logprobs_grad(logits, t, a["lse"], a["entropy"], d, d, None, new(7, 500)) == xg.XGEMM_OK
    assert torch.equal(call(), slow(call))
    for bad in ((logits, t, None, a["entropy"], d, d, d, new(7, 500)), (logits, t, a["lse"], None, d, d, d, new(7, 500)),
                (logits, None, a["lse"], None, d, None, None, new(7, 500)),
                (logits, t, a["lse"], a["entropy"], d, d, d, new(7, 501)),
                (logits, t, a["lse"], a["entropy"], d.half(), d, d, new(7, 500))):
        assert _fastcall.logprobs_grad(*bad) is None


@pytest.mark.gpu
def test_a_failure_is_raised():
    x, scores = torch.zeros(1, 64, device="cuda").bfloat16(), torch.zeros(1, 2, device="cuda")
    up, down = torch.zeros(2, 64, 64, device="cuda").bfloat16(), torch.zeros(2, 64, 32, device="cuda").bfloat16()
    h = xg.handle(0, torch.cuda.current_stream())
    assert xg.xgemm_set_workspace_limit(h, 4100) == xg.XGEMM_OK
    try:
        with pytest.raises(xg.XgemmError) as e:
            xg.experts(x, scores, up, down, 1, out=torch.empty(1, 64, device="cuda"))
        assert e.value.status == xg.XGEMM_ERR_ALLOC and "limit" in str(e.value)
    finally:
        assert xg.xgemm_set_workspace_limit(h, 0) == xg.XGEMM_OK
