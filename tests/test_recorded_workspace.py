"""Calls recorded into a graph keep a workspace that no other call frees or uses."""
import pytest
import torch

from paper_2609_16389_amd import xgemm as xg

pytestmark = pytest.mark.gpu


def layer(T, H, I, seed, E=8):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def new(*shape, scale=1.0):
        return torch.randn(shape, device="cuda", generator=gen).mul_(scale)

    return (new(T, H).bfloat16(), new(T, E), new(E, 2 * I, H, scale=H ** -0.5).bfloat16(),
            new(E, H, I, scale=I ** -0.5).bfloat16())


def record(stream, call):
    """A graph of `call`, made once before on the stream, and its outputs."""
    with torch.cuda.stream(stream):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    return graph


def overwrite_free_memory():
    """Give back what the allocator holds and write over memory that is free."""
    torch.cuda.empty_cache()
    junk = [torch.full((n,), 0x5a5a5a5a, dtype=torch.int32, device="cuda") for n in [1 << 16] * 64 + [1 << 20] * 16]
    torch.cuda.synchronize()
    return junk


def calls():
    """(name, inputs that change, call into out, the same call with what it needs more workspace for)."""
    small, large = layer(4, 256, 128, 1), layer(64, 2048, 512, 2)
    out = torch.empty((4, 256), dtype=torch.bfloat16, device="cuda")
    yield "experts", small[0], out, lambda o: xg.experts(*small, 2, out=o), lambda: xg.experts(*large, 2)
    row, rows = torch.randn(1, 70001, device="cuda"), torch.randn(64, 200000, device="cuda")
    lp = {"lse": torch.empty(1, device="cuda"), "top_logprob": torch.empty(1, 5, device="cuda"),
          "top_id": torch.empty(1, 5, dtype=torch.int64, device="cuda")}
    yield "logprobs", row, lp, lambda o: xg.logprobs(row, top=5, out=o), lambda: xg.logprobs(rows, top=32)
    a, b = torch.randn(64, 8192, device="cuda").bfloat16(), torch.randn(8192, 64, device="cuda").bfloat16()
    c, d = torch.randn(512, 16384, device="cuda").bfloat16(), torch.randn(16384, 512, device="cuda").bfloat16()
    yield ("gemm", a, torch.empty((64, 64), device="cuda"), lambda o: xg.gemm(a, b, out=o),
           lambda: (xg.gemm(c, d), xg.gemm(c[:511, :16383], d[:16383, :511])))


def copies(out):
    return {k: v.clone() for k, v in out.items()} if isinstance(out, dict) else {"out": out.clone()}


def fresh(out):
    return {k: torch.empty_like(v) for k, v in out.items()} if isinstance(out, dict) else torch.empty_like(out)


@pytest.mark.parametrize("which", [0, 1, 2], ids=["experts", "logprobs", "gemm"])
def test_replayed_after_the_workspace_has_grown(which):
    _, x, out, call, larger = list(calls())[which]
    stream = torch.cuda.Stream()
    graph = record(stream, lambda: call(out))
    with torch.cuda.stream(stream):
        for _ in range(2):
            larger()
    junk = overwrite_free_memory()
    for seed in range(3):
        x.copy_(torch.randn(x.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        expected = fresh(out)
        call(expected)
        got, want = copies(out), copies(expected)
        assert all(torch.equal(got[k], want[k]) for k in want), which
    assert all(bool((j == 0x5a5a5a5a).all()) for j in junk)   # (nothing was written where it was freed)


@pytest.mark.parametrize("which", [0, 1, 2], ids=["experts", "logprobs", "gemm"])
def test_replays_beside_calls_on_the_recording_stream(which):
    """Replays on one stream and direct calls on the stream that recorded, in no
    order between them."""
    _, x, out, call, larger = list(calls())[which]
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    graph = record(stream, lambda: call(out))
    expected = fresh(out)
    call(expected)
    torch.cuda.synchronize()
    want, got = copies(expected), []
    for _ in range(20):
        direct = fresh(out)
        with torch.cuda.stream(stream):
            call(direct)
        with torch.cuda.stream(other):
            graph.replay()
            got.append(copies(out))
        got.append(direct if isinstance(direct, dict) else {"out": direct})
    torch.cuda.synchronize()
    assert all(torch.equal(g[k], want[k]) for g in got for k in want), which


def test_a_second_recording_may_need_more():
    """The first graph keeps the buffer that it recorded."""
    first, second = layer(2, 128, 64, 3), layer(40, 1024, 256, 4)
    out1, out2 = torch.empty_like(first[0]), torch.empty_like(second[0])
    stream = torch.cuda.Stream()
    g1 = record(stream, lambda: xg.experts(*first, 2, out=out1))
    g2 = record(stream, lambda: xg.experts(*second, 2, out=out2))
    junk = overwrite_free_memory()
    for _ in range(3):
        for g, args, out in ((g1, first, out1), (g2, second, out2)):
            args[0].copy_(torch.randn(args[0].shape, device="cuda"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, xg.experts(*args, 2))
    assert all(bool((j == 0x5a5a5a5a).all()) for j in junk)
