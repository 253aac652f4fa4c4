"""The products whose ends are fused, called from several threads at once, each on a
stream (and so a handle and a workspace) of its own."""
import threading

import pytest
import torch

from test_fused_calls import calls, same


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_threads_with_streams_of_their_own(dtype):
    sizes = [(1, 256, 72, 1000), (90, 200, 130, 2050), (333, 72, 520, 4099), (300, 201, 131, 5001)]
    runs = [calls(*size, dtype, k)[0] for k, size in enumerate(sizes)]
    expect = [{n: v.clone() for n, v in run().items()} for run in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    assert len({s.cuda_stream for s in streams}) == len(streams)
    start, errors = threading.Barrier(len(runs)), []

    def work(k):
        try:
            start.wait(30)
            with torch.cuda.stream(streams[k]):
                for _ in range(20):
                    for v in runs[k]().values():
                        pass
                streams[k].synchronize()
        except BaseException as e:   # noqa: B902 (shown by the test's own thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(runs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not errors, errors
    assert not any(t.is_alive() for t in threads)
    for k, run in enumerate(runs):
        with torch.cuda.stream(streams[k]):
            got = run()
        streams[k].synchronize()
        same(got, expect[k])
