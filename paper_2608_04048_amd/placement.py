"""Where a tensor-level call works: on the GPU of its tensors, and there on the
stream it is given.

A kernel launched while another GPU is the current one would run on that GPU.

Memory that torch allocates belongs to the stream that was current then: it may
still be read by work queued on that stream (a tensor freed a moment ago), so a
kernel on another stream must not write it at once. A call for another stream
therefore runs with that stream as the current one, outputs and workspaces
included.
"""

from __future__ import annotations

import torch


def _stream_on(index: int, stream):
    """The torch stream that a stream object or a raw handle names; the current
    one of that GPU for None."""
    if stream is None:
        return torch.cuda.current_stream(index)
    if not isinstance(stream, torch.cuda.Stream):
        handle = stream if isinstance(stream, int) else stream.cuda_stream
        if handle == 0:         # (an ExternalStream of 0 would be a stream of torch's pool)
            return torch.cuda.default_stream(index)
        return torch.cuda.ExternalStream(handle, device=index)
    if stream.device_index != index:
        raise ValueError(f"stream must be on cuda:{index}, got {stream.device}")
    return stream


def elsewhere(index: int, stream) -> bool:
    """Whether a call on cuda:index has to leave the caller's GPU or stream."""
    return stream is not None or torch._C._cuda_getDevice() != index


class on_stream:
    """Context in which cuda:index is the current GPU and `stream` its current
    stream.

    `used` are the tensors of the call (others are passed over): once it is
    enqueued, none of them is handed out again before `stream` has passed it. What
    the call returns goes through ``returned``, so that the caller's own stream
    may use it on.
    """

    def __init__(self, index: int, stream, *used):
        self.stream = _stream_on(index, stream)
        self.used = used
        self.caller = torch.cuda.current_stream(index)
        self.context = torch.cuda.stream(self.stream)

    def __enter__(self):
        self.context.__enter__()
        return self

    def __exit__(self, error, value, trace):
        self.context.__exit__(error, value, trace)
        if error is None:
            for t in self.used:
                if isinstance(t, torch.Tensor):
                    t.record_stream(self.stream)

    def returned(self, result):
        for t in result if isinstance(result, tuple) else (result,):
            if t is not None:
                t.record_stream(self.caller)
        return result
