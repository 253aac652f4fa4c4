"""How the products whose ends are fused share the machine: recorded into graphs,
on streams of their own, with a capped workspace, the same bits each time."""
import pytest
import torch

from paper_2609_16389_amd import xgemm as xg


def calls(M, H, I, V, dtype, seed=0):
    """Every operator on one set of inputs: a function that runs them all and returns
    their outputs, the same buffers each time."""
    g = torch.Generator("cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, up = rand(M, H).to(dtype), (rand(2 * I, H) / H ** 0.5).to(dtype)
    head, targets = (rand(V, H) / H ** 0.5).to(dtype), torch.randint(0, V, (M,), device="cuda", generator=g)
    w, ws = xg.scaled_rows(rand(V, H))
    d = rand(M, I).to(dtype)
    weight = torch.full((M,), -1.0 / M, device="cuda")
    new = lambda *s, dtype=dtype: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    out = {"y": new(M, V), "inner": new(M, I), "pre": new(M, 2 * I), "d_x": new(M, H), "d_up": new(2 * I, H),
           "lse": new(M, dtype=torch.float32), "logprob": new(M, dtype=torch.float32), "d_hidden": new(M, H),
           "d_head": new(V, H), "q": new(M, H, dtype=torch.int8), "s": new(M, dtype=torch.float32)}

    def run():
        xg.scaled_rows(x, out=(out["q"], out["s"]))
        xg.gemm_scaled(x, w, ws, out=out["y"])
        xg.gated(x, up, out=out["inner"], pre=out["pre"])
        xg.gated_grad(x, up, out["pre"], d, out=(out["d_x"], out["d_up"]))
        xg.head_logprobs(x, head, targets, out={"lse": out["lse"], "logprob": out["logprob"]})
        xg.head_logprobs_grad(x, head, targets, out["lse"], weight, out=(out["d_hidden"], out["d_head"]))
        return out
    return run, (x, up, head, w, ws, d, weight, targets)


SIZES = [(1, 256, 72, 1000), (7, 129, 65, 1003), (90, 200, 130, 2050), (333, 72, 520, 4099)]


def same(a, b):
    for name in a:
        assert torch.equal(a[name], b[name]), name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", SIZES)
def test_the_same_bits_each_time(size, dtype):
    run, _ = calls(*size, dtype)
    first = {k: v.clone() for k, v in run().items()}
    for _ in range(3):
        same(run(), first)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", SIZES)
def test_recorded(size, dtype):
    """Replayed with new inputs, with the program's own calls between the replays."""
    stream = torch.cuda.Stream()
    run, inputs = calls(*size, dtype)
    other, _ = calls(70, 300, 90, 3001, dtype, 5)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
    torch.cuda.synchronize()
    for k in range(4):
        inputs[0].mul_(0.5 + 0.5 * k)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: v.clone() for n, v in run().items()}
        for v in run().values():
            v.fill_(3)
        other()
        graph.replay()
        torch.cuda.synchronize()
        same(run(), got)
        graph.replay()
        other()
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_on_two_streams():
    """Calls on two streams at once, each with a handle and a workspace of its own."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    runs = [calls(300, 200, 130, 5001, torch.bfloat16, k)[0] for k in range(2)]
    expect = [{n: v.clone() for n, v in run().items()} for run in runs]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, run in zip(streams, runs):
            with torch.cuda.stream(s):
                run()
    torch.cuda.synchronize()
    for run, e in zip(runs, expect):
        with torch.cuda.stream(streams[0]):
            got = run()
        torch.cuda.synchronize()
        same(got, e)


@pytest.mark.gpu
def test_on_a_stream_that_is_not_current():
    run, (x, up, head, w, ws, d, weight, targets) = calls(40, 200, 130, 500, torch.bfloat16)
    expect = run()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    lse = xg.head_logprobs(x, head, targets, stream=stream)
    pre = torch.empty_like(expect["pre"])
    got = {"y": xg.gemm_scaled(x, w, ws, out=torch.empty_like(expect["y"]), stream=stream),
           "inner": xg.gated(x, up, pre=pre, stream=stream), "lse": lse["lse"], "logprob": lse["logprob"],
           "q": None, "s": None}
    got["q"], got["s"] = xg.scaled_rows(x, stream=stream)
    got["d_x"], got["d_up"] = xg.gated_grad(x, up, pre, d, stream=stream)
    got["d_hidden"], got["d_head"] = xg.head_logprobs_grad(x, head, targets, lse["lse"], weight, stream=stream)
    stream.synchronize()
    same(got, {n: expect[n] for n in got})


@pytest.mark.gpu
def test_a_capped_workspace_is_an_error():
    """Nothing is enqueued, and the outputs stay as they were."""
    h = xg.xgemm_create()
    try:
        assert xg.xgemm_set_workspace_limit(h, 8192) == xg.XGEMM_OK
        M, H, I, V = 200, 72, 40, 3000
        t = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        x, up, pre, d, head = t(M, H), t(2 * I, H), t(M, 2 * I), t(M, I), t(V, H)
        dx, du, dw = t(M, H) + 7, t(2 * I, H) + 7, t(V, H) + 7
        lse = torch.full((M,), 7.0, device="cuda")
        p = lambda a: a.data_ptr()  # noqa: E731
        bad = xg.XGEMM_ERR_ALLOC
        assert xg.xgemm_gated_grad(h, M, H, I, p(x), H, p(up), H, p(pre), 2 * I, p(d), I, p(dx), H, p(du), H, 0, 0, 1, None) == bad
        assert xg.xgemm_head_run(h, M, V, H, p(x), H, p(head), H, None, None, p(lse), 0, None) == bad
        assert xg.xgemm_head_grad(h, M, V, H, p(x), H, p(head), H, None, p(lse), None, p(lse), p(dx), H, p(dw), H, 0, 1,
                                  None) == bad
        torch.cuda.synchronize()
        assert all(bool((a == 7).all()) for a in (dx, du, dw, lse))
        assert "limit" in xg.xgemm_last_error(h)
    finally:
        assert xg.xgemm_destroy(h) == xg.XGEMM_OK
