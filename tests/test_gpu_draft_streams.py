"""The drafting calls on a stream of their own: memory is handed out in the order of the
streams that use it, and tensors may be let go as soon as a call returns."""

import pytest

from serving_helpers import Setup

pytestmark = pytest.mark.gpu
SLEEP = 20_000_000          # cycles: some 10 ms of a stream's time
NAMES = ["norm", "append", "tree", "verify"]


def _call(rrq, name):
    """(inputs, call(inputs, stream=...) -> tensors), results large enough for blocks of
    their own; the call leaves its inputs as they are, as far as its results go."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    if name == "norm":
        x = dict(residual=normal(900, 700), y=normal(900, 700), weight=normal(700),
                 bias=normal(700), gate=normal(900, 700), post_weight=normal(700))
        return x, lambda x, **kw: rrq.block_norm(**x, post="rms", **kw)
    if name == "verify":
        B, n, V = 8000, 3, 50
        x = dict(logits=normal(B * n, V), tokens=torch.randint(0, V, (B * n,), device="cuda"),
                 offsets=torch.arange(0, B * n + 1, n, dtype=torch.int32, device="cuda"),
                 uniforms=torch.rand(B * n, device="cuda"), draft=normal(B, n - 1, V))
        return x, lambda x, **kw: rrq.verify_drafts(max_accept=n - 1, **x, **kw)
    s = Setup(rrq, [(300, 300), (700, 900)], 2, 128, 64, "int8", seed=1).fill().to_gpu()
    x = dict(Q=normal(1000, 8, 128))
    if name == "tree":
        x["seen"] = torch.full((1000, 11), -1, dtype=torch.int64, device="cuda")
        x["positions"] = torch.arange(1000, dtype=torch.int32, device="cuda")
        return x, lambda x, **kw: (rrq.tree_attention(s.cache, s.batch, window=400, **x, **kw),)
    x.update(K=normal(1000, 2, 128), V=normal(1000, 2, 128),
             positions=torch.arange(1000, dtype=torch.int32, device="cuda"))
    rotary = rrq.Rotary(rrq.rotary_frequencies(128))
    return x, lambda x, **kw: (rrq.cache_append(s.cache, s.batch, rotary, **x, **kw),)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_outputs_wait_for_nothing_they_overwrite(gpu, name, raw):
    """A block just freed on the current stream, with work that reads it still to come, is
    not written by a call on another stream."""
    import torch
    x, call = _call(gpu, name)
    want = call(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    freed = [torch.full_like(t, 7) for t in want]
    at = {t.data_ptr() for t in freed}
    torch.cuda._sleep(SLEEP)
    read = [t.clone() for t in freed]
    del freed
    got = call(x, stream=side.cuda_stream if raw else side)
    assert not at & {t.data_ptr() for t in got}
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    assert all((t == 7).all() for t in read)


@pytest.mark.parametrize("name", NAMES)
def test_outputs_are_kept_for_the_caller(gpu, name):
    """Work on the caller's stream reads a result that has been let go; the call's stream
    does not get its memory back before."""
    import torch
    x, call = _call(gpu, name)
    want = call(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(x, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(SLEEP)
    read = [t.clone() for t in got]
    shapes = [(t.shape, t.dtype) for t in got]
    del got
    with torch.cuda.stream(side):
        other = [torch.full(shape, 9, dtype=dtype, device="cuda") for shape, dtype in shapes]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(read, want)) and len(other) == len(read)


@pytest.mark.parametrize("name", NAMES)
def test_inputs_may_be_let_go(gpu, name):
    """Inputs are freed while the call's stream has not come to them; new tensors of the
    caller's do not take their place."""
    import torch
    x, call = _call(gpu, name)
    want = call(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    copies = {k: t.clone() for k, t in x.items()}
    with torch.cuda.stream(side):
        torch.cuda._sleep(SLEEP)
    side_wait = torch.cuda.current_stream().record_event()
    side.wait_event(side_wait)
    shapes = [(t.shape, t.dtype) for t in copies.values()]
    got = call(copies, stream=side)
    copies.clear()
    other = [torch.zeros(shape, dtype=dtype, device="cuda") for shape, dtype in shapes]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(other) == len(shapes)


def test_two_streams_at_once(gpu):
    """Calls of their own workspaces on two streams, again and again."""
    import torch
    pairs = [_call(gpu, name) for name in ("tree", "verify")]
    want = [call(x) for x, call in pairs]
    sides = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for (x, call), side in zip(pairs, sides):
            got.append(call(x, stream=side))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 2]))
