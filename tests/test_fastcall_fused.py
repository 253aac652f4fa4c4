"""The native call path of the products whose ends are fused: it declines what is
not plain, and gives what the ctypes path gives."""
import pytest
import torch

from paper_2609_16389_amd import _fastcall
from paper_2609_16389_amd import xgemm as xg

NAMES = ("scaled_rows", "gemm_scaled", "gated", "gated_grad", "head_logprobs", "head_logprobs_grad")


def test_declines_what_is_not_plain():
    b, f, i = torch.zeros(2, 8).bfloat16(), torch.zeros(2, 8), torch.zeros(2, 8, dtype=torch.int8)
    v = torch.zeros(2)
    assert _fastcall.scaled_rows(f, i, v) is None                     # not on a GPU
    assert _fastcall.scaled_rows(f, i) is None and _fastcall.scaled_rows(None, i, v) is None
    assert _fastcall.gemm_scaled(i, i, v, v, f[:, :2]) is None
    assert _fastcall.gated(b, b, 0, b[:, :1], None) is None and _fastcall.gated(b, b, "silu", b[:, :1], None) is None
    assert _fastcall.gated_grad(b, b, b[:, :2], b[:, :1], 0, b, b) is None
    assert _fastcall.gated_grad(b, b, b[:, :2], b[:, :1], 0, None, None) is None
    assert _fastcall.head_logprobs(b, b, None, {"lse": v}) is None and _fastcall.head_logprobs(b, b, None, None) is None
    assert _fastcall.head_logprobs_grad(b, b, None, v, None, v, b, b) is None
    for name in NAMES:
        assert getattr(_fastcall, name)() is None


@pytest.fixture
def both(monkeypatch):
    """The results of a call either way, and that the first was a native one."""
    def calls(name, f, *tensors):
        native = getattr(_fastcall, name)
        done = []
        with monkeypatch.context() as m:
            m.setattr(_fastcall, name, lambda *a: done.append(native(*a)) or done[-1])
            first = f()
            assert done == [xg.XGEMM_OK], name
            m.setattr(_fastcall, name, lambda *a: None)
            second = f()
        for a, b in zip(first, second):
            assert torch.equal(a, b), name
    return calls


@pytest.mark.gpu
def test_same_as_the_other_path(both):
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    new = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    xg.handle(0, torch.cuda.current_stream())
    for M in (5, 70):
        for t in (torch.bfloat16, torch.float16, torch.float32):
            x = rand(M, 300).to(t)[:, :257]
            both("scaled_rows", lambda: xg.scaled_rows(x, out=(new(M, 257, dtype=torch.int8), new(M))))
            w, ws = xg.scaled_rows(rand(70, 257))
            both("gemm_scaled", lambda: [xg.gemm_scaled(x, w, ws, out=new(M, 70, dtype=t))])
            q, xs = xg.scaled_rows(x)
            both("gemm_scaled", lambda: [xg.gemm_scaled(q, w, ws, xs, out=new(M, 70))])
        x, up = rand(M, 40).bfloat16(), rand(48, 40).bfloat16()
        pre = new(M, 48, dtype=x.dtype)
        for act in ("silu", "gelu", "gelu_tanh"):
            both("gated", lambda: [xg.gated(x, up, act, out=new(M, 24), pre=pre), pre.clone()])
            both("gated", lambda: [xg.gated(x, up, act, out=new(M, 24, dtype=x.dtype))])
            d = rand(M, 24).bfloat16()
            both("gated_grad", lambda: xg.gated_grad(x, up, pre, d, act, out=(new(M, 40), new(48, 40))))
            both("gated_grad", lambda: xg.gated_grad(x, up, pre, d, act, out=(None, new(48, 40)))[1:])
        head, targets = rand(99, 40).bfloat16(), torch.randint(0, 99, (M,), device="cuda", generator=g)
        both("head_logprobs", lambda: xg.head_logprobs(x, head, targets, out={"lse": new(M), "logprob": new(M)}).values())
        both("head_logprobs", lambda: xg.head_logprobs(x, head, out={"lse": new(M)}).values())
        lse, dl, ds = xg.head_logprobs(x, head)["lse"], rand(M), rand(M)
        both("head_logprobs_grad", lambda: xg.head_logprobs_grad(x, head, targets, lse, dl, ds, out=(new(M, 40), new(99, 40))))
        both("head_logprobs_grad",
             lambda: xg.head_logprobs_grad(x, head, None, lse, None, ds, out=(new(M, 40, dtype=x.dtype), None))[:1])


@pytest.mark.gpu
def test_leaves_what_does_not_fit_to_the_checks():
    b = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int8, device="cuda")  # noqa: E731
    t = torch.zeros(2, dtype=torch.int64, device="cuda")
    xg.handle(0, torch.cuda.current_stream())
    for bad in ((b(2, 8), i(2, 7), f(2)), (b(2, 8), f(2, 8), f(2)), (b(2, 8), i(2, 8), f(3)), (b(2, 8), i(2, 8), None),
                (f(2, 8).double(), i(2, 8), f(2)), (f(8, 2).t(), i(2, 8), f(2))):
        assert _fastcall.scaled_rows(*bad) is None
    for bad in ((i(2, 8), i(3, 8), f(3), None, f(2, 3)), (f(2, 8), i(3, 8), f(3), f(2), f(2, 3)), (i(2, 8), i(3, 7), f(3), f(2), f(2, 3)),
                (i(2, 8), f(3, 8), f(3), f(2), f(2, 3)), (i(2, 8), i(3, 8), f(2), f(2), f(2, 3)), (i(2, 8), i(3, 8), f(3), f(2), i(2, 3)),
                (i(2, 8), i(3, 8), None, f(2), f(2, 3)), (i(2, 8), i(3, 8), f(3), f(2), f(3, 2).t())):
        assert _fastcall.gemm_scaled(*bad) is None
    for bad in ((b(2, 8), b(5, 8), 0, b(2, 2), None), (b(2, 8), b(6, 8), 3, b(2, 3), None), (b(2, 8), b(6, 8), 0, i(2, 3), None),
                (b(2, 8), b(6, 8), 0, b(2, 3), f(2, 6)), (b(2, 8), f(6, 8), 0, b(2, 3), None), (b(2, 8), b(6, 8), 0.0, b(2, 3), None),
                (b(2, 8), b(6, 8), None, b(2, 3), None)):
        assert _fastcall.gated(*bad) is None
    for bad in ((b(2, 8), b(6, 8), b(2, 6), b(2, 3), 0, None, None), (b(2, 8), b(6, 8), b(2, 6), b(2, 3), 0, b(2, 8), f(6, 8)),
                (b(2, 8), b(6, 8), b(2, 5), b(2, 3), 0, b(2, 8), None), (b(2, 8), b(6, 8), b(2, 6), f(2, 3), 0, b(2, 8), None),
                (b(2, 8), b(6, 8), b(2, 6), b(2, 3), 0, b(2, 7), None)):
        assert _fastcall.gated_grad(*bad) is None
    for bad in ((b(2, 8), b(5, 8), None, {"logprob": f(2)}), (b(2, 8), b(5, 8), t.int(), {"lse": f(2)}),
                (b(2, 8), b(5, 7), t, {"lse": f(2)}), (b(2, 8), b(5, 8), t, {"entropy": f(2)}), (b(2, 8), b(0, 8), t, {"lse": f(2)})):
        assert _fastcall.head_logprobs(*bad) is None
    for bad in ((b(2, 8), b(5, 8), t, None, f(2), None, b(2, 8), None), (b(2, 8), b(5, 8), None, f(2), f(2), None, b(2, 8), None),
                (b(2, 8), b(5, 8), t, f(2), f(2), None, None, None), (b(2, 8), b(5, 8), t, f(2), f(3), None, b(2, 8), None)):
        assert _fastcall.head_logprobs_grad(*bad) is None
