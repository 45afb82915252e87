"""Which GPU and stream a serving call works on, with the runtime replaced: two
GPUs, tensors on the one that is not current. No GPU needed."""

from contextlib import contextmanager
from types import SimpleNamespace

import pytest
import torch

from paper_2608_04048_amd import placement, serving


class OnSecond(torch.Tensor):
    """A tensor that says it is on cuda:1."""

    def get_device(self):
        return 1


def _on_second(*shape):
    return torch.zeros(shape).as_subclass(OnSecond)


@pytest.fixture
def world(monkeypatch):
    """cuda:0 current, each GPU on its stream 10 + index; what the library was
    asked to do, and the streams that tensors were kept for."""
    w = SimpleNamespace(device=0, streams={0: 10, 1: 11}, launched=[], kept=[])

    def stream_object(index, handle):
        return SimpleNamespace(device_index=index, device=f"cuda:{index}", cuda_stream=handle)

    @contextmanager
    def stream_context(stream):
        before = w.device, dict(w.streams)
        w.device = stream.device_index
        w.streams[w.device] = stream.cuda_stream
        try:
            yield
        finally:
            w.device, w.streams = before

    def enqueue(name):
        def call(*args):
            w.launched.append((name, w.device, args[-1]))
            return 0
        return call

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: w.device, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda index=None: stream_object(index, w.streams[index]))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda index=None: stream_object(index, 0))
    monkeypatch.setattr(torch.cuda, "stream", stream_context)
    monkeypatch.setattr(torch.cuda, "ExternalStream",
                        lambda handle, device: stream_object(device, handle))
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda t, s: w.kept.append((id(t), s.cuda_stream)), raising=False)
    monkeypatch.setattr(serving, "_stream", lambda s: w.streams[w.device])
    monkeypatch.setattr(serving, "rrq_token_logprobs_workspace", lambda *sizes: 0)
    monkeypatch.setattr(serving, "_lib", SimpleNamespace(**{
        n: enqueue(n) for n in ("rrq_cache_write", "rrq_cache_read", "rrq_cache_attention",
                                "rrq_token_logprobs")}))
    cpu = torch.device("cpu")
    w.cache = SimpleNamespace(index=1, device=cpu, n_kv_heads=2, head_dim=64, page_size=16,
                              ref=None, tensors=(_on_second(1),))
    w.batch = SimpleNamespace(index=1, device=cpu, n_tokens=3, ref=None, tensors=(_on_second(1),),
                              workspace_bytes={(2, 64, 16, 4): 0})
    w.K, w.Q, w.logits = _on_second(3, 2, 64), _on_second(3, 4, 64), _on_second(3, 50)
    w.calls = (
        ("rrq_cache_write", lambda **kw: serving.cache_write(w.cache, w.batch, w.K, w.K, **kw)),
        ("rrq_cache_read", lambda **kw: serving.cache_read(w.cache, w.batch, **kw)),
        ("rrq_cache_attention", lambda **kw: serving.cache_attention(w.cache, w.batch, w.Q, **kw)),
        ("rrq_token_logprobs", lambda **kw: serving.token_logprobs(w.logits, None, 5, **kw)))
    return w


def test_the_gpu_of_the_tensors(world):
    for name, call in world.calls:
        call()
        assert world.launched.pop() == (name, 1, 11) and not world.launched
        assert world.device == 0 and world.streams == {0: 10, 1: 11}


def test_the_current_gpu_takes_no_detour(world, monkeypatch):
    world.device = 1
    monkeypatch.setattr(serving, "on_stream", None)
    for name, call in world.calls:
        call()
        assert world.launched.pop() == (name, 1, 11)
    assert not world.kept


@pytest.mark.parametrize("device", [0, 1])
def test_a_given_stream(world, device):
    world.device = device
    for name, call in world.calls:
        world.kept.clear()
        result = call(stream=77)
        assert world.launched.pop() == (name, 1, 77) and world.device == device
        # inputs for the call's stream, results for the caller's on that GPU
        assert (id(world.cache.tensors[0]), 77) in world.kept or name == "rrq_token_logprobs"
        results = result if isinstance(result, tuple) else (result,)
        for t in results:
            assert t is None or (id(t), 11) in world.kept
        call(stream=0)
        assert world.launched.pop() == (name, 1, 0)


def test_a_stream_of_another_gpu(world, monkeypatch):
    monkeypatch.setattr(torch.cuda, "Stream", SimpleNamespace)
    other = SimpleNamespace(device_index=0, device="cuda:0", cuda_stream=5)
    for _, call in world.calls:
        with pytest.raises(ValueError, match="cuda:1"):
            call(stream=other)
    assert not world.launched


def test_a_refused_call_keeps_nothing(world):
    world.Q = _on_second(3, 4, 32)
    with pytest.raises(ValueError):
        world.calls[2][1](stream=77)
    assert not world.launched and not world.kept and world.streams == {0: 10, 1: 11}
    assert placement.elsewhere(1, None) and not placement.elsewhere(0, None)
