"""Calls on a stream of their own: memory is handed out in the order of the
streams that use it, and tensors may be let go as soon as a call returns."""

import pytest

from serving_helpers import Setup

pytestmark = pytest.mark.gpu
SLEEP = 20_000_000          # cycles: some 10 ms of a stream's time


def _calls(rrq):
    """(name, call(stream) -> tensors) of every call that allocates, each on
    inputs whose results are large enough for a block of their own."""
    import torch
    s = Setup(rrq, [(300, 300), (700, 900)], 2, 128, 64, "int8", seed=1).fill().to_gpu()
    Q = torch.randn((1000, 8, 128), device="cuda")
    logits = torch.randn((20000, 600), device="cuda")
    return s, [("read", lambda **kw: rrq.cache_read(s.cache, s.batch, torch.float32, **kw)),
               ("attention", lambda **kw: (rrq.cache_attention(s.cache, s.batch, Q, **kw),)),
               ("scoring", lambda **kw: rrq.token_logprobs(logits, None, 32, **kw)[1:])]


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_outputs_wait_for_nothing_they_overwrite(gpu, which, raw):
    """A block just freed on the current stream, with work that reads it still
    to come, is not written by a call on another stream."""
    import torch
    s, calls = _calls(gpu)
    call = calls[which][1]
    want = call()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    freed = [torch.full_like(t, 7) for t in want]
    at = {t.data_ptr() for t in freed}
    torch.cuda._sleep(SLEEP)
    read = [t.clone() for t in freed]
    del freed
    got = call(stream=side.cuda_stream if raw else side)
    assert not at & {t.data_ptr() for t in got}
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    assert all((t == 7).all() for t in read)


@pytest.mark.parametrize("which", [0, 1, 2])
def test_outputs_are_kept_for_the_caller(gpu, which):
    """Work on the caller's stream reads a result that has been let go; the call's
    stream does not get its memory back before."""
    import torch
    s, calls = _calls(gpu)
    call = calls[which][1]
    want = call()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(SLEEP)
    read = [t.clone() for t in got]
    shapes = [(t.shape, t.dtype) for t in got]
    del got
    with torch.cuda.stream(side):
        other = [torch.full(shape, 9, dtype=dtype, device="cuda") for shape, dtype in shapes]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(read, want)) and len(other) == len(read)


def test_inputs_may_be_let_go(gpu):
    """Queries, a batch and a cache's source are freed while the call's stream
    has not come to them; new tensors of the caller's do not take their place."""
    import torch
    s = Setup(gpu, [(500, 900), (500, 500)], 2, 128, 64, "int8", seed=2).fill().to_gpu()
    Q = torch.randn((1000, 8, 128), device="cuda")
    K = torch.randn((1000, 2, 128), device="cuda")
    parts = [t.clone() for t in (s.batch.page_table, s.batch.lengths, s.batch.offsets)]

    def run(stream):
        q, k, b = Q.clone(), K.clone(), gpu.CacheBatch(*(t.clone() for t in parts), 1000)
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(SLEEP)
        gpu.cache_write(s.cache, b, k, k, stream=stream)
        out = gpu.cache_attention(s.cache, b, q, stream=stream)
        sizes = [(t.shape, t.dtype) for t in (q, k, *b.tensors)]
        del q, k, b
        new = [torch.full(shape, 3, dtype=dtype, device="cuda") for shape, dtype in sizes]
        torch.cuda.synchronize()
        return out, new

    want, _ = run(None)
    got, _ = run(torch.cuda.Stream())
    assert torch.equal(got, want)


def test_the_default_stream_by_its_handle(gpu):
    """0 names the default stream, from inside another one too."""
    import torch
    s, calls = _calls(gpu)
    for name, call in calls:
        want = call()
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream()):
            got = call(stream=0)
            torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name


def test_an_error_leaves_the_current_stream(gpu):
    import torch
    s, _ = _calls(gpu)
    before = torch.cuda.current_stream()
    side = torch.cuda.Stream()
    with pytest.raises(ValueError):
        gpu.cache_attention(s.cache, s.batch, torch.zeros((3, 8, 128), device="cuda"), stream=side)
    with pytest.raises(gpu.RRQError):
        gpu.token_logprobs(torch.zeros((2, 40), device="cuda"), n_top=33, stream=side)
    assert torch.cuda.current_stream() == before


def test_a_captured_call_that_names_its_stream(gpu):
    """Inputs from the default stream, captured on a stream given by name;
    replayed on new inputs, with eager calls between."""
    import torch
    s, _ = _calls(gpu)
    Q = torch.randn((1000, 8, 128), device="cuda")
    logits = torch.randn((1000, 20000), device="cuda")
    side = torch.cuda.Stream()

    def step(**kw):
        return (gpu.cache_attention(s.cache, s.batch, Q, **kw),
                *gpu.cache_read(s.cache, s.batch, **kw),
                *gpu.token_logprobs(logits, None, 3, **kw)[1:])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step(stream=side)
    for seed in range(4):
        Q.normal_()
        logits.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed
