"""What a decoder served from RRQ packages runs beside the linear layers: an
8-bit paged key/value cache, attention over it, and token scoring.

Binding of include/rrq_serve.h in librrq.so. ``rrq_cache_write``,
``rrq_cache_read``, ``rrq_cache_attention`` and ``rrq_token_logprobs`` marshal
arguments one to one; ``cache_write``, ``cache_read``, ``cache_attention`` and
``token_logprobs`` take torch tensors, check them and allocate the outputs.
Every computation runs in the HIP kernels.

    cache = KVCache.empty(n_pages, n_kv_heads=8, head_dim=128)
    batch = CacheBatch(page_table, lengths, offsets, n_tokens)
    cache_write(cache, batch, K, V)          # this step's tokens
    out = cache_attention(cache, batch, Q)   # bfloat16, rrq_linear's X
    logprob, entropy, ids, top = token_logprobs(logits, targets, n_top=5)

A ``KVCache`` and a ``CacheBatch`` keep the tensors they were made of and a C
descriptor of them; a program makes them once and updates the tensors in place
(``lengths`` on the device from step to step).

Forward only: no call records a graph for gradients, and results of inputs that
require one are detached.

``stream`` (a torch stream or a raw handle; by default torch's current stream) is
where a call allocates and works, on the GPU of its tensors whichever is current.
The caller orders it after the work that made the inputs, and orders the use of
the outputs after it; the tensors themselves may be let go at once.
"""

from __future__ import annotations

import ctypes
import math

import torch

from . import (RRQ_BF16, RRQ_F32, RRQ_OK, RRQError, _check_device_tensor, _ptr, _stream,
               load_library)
from .placement import elsewhere, on_stream

RRQ_CODE_INT8 = 0
RRQ_CODE_FP8 = 1
CODE_TYPES = {"int8": RRQ_CODE_INT8, "fp8": RRQ_CODE_FP8}
RRQ_MAX_TOP = 32
PAGE_SIZES = (16, 32, 64, 128)
HEAD_DIMS = (64, 128, 256)


class RrqCache(ctypes.Structure):
    """struct rrq_cache of rrq_serve.h."""
    _fields_ = [("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("code_type", ctypes.c_int32)]


class RrqBatch(ctypes.Structure):
    """struct rrq_batch of rrq_serve.h."""
    _fields_ = [("page_table", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                ("offsets", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
                ("max_pages", ctypes.c_int64), ("n_seqs", ctypes.c_int64),
                ("n_tokens", ctypes.c_int64)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        P, I64, I32, F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float
        SZ = ctypes.c_size_t
        for name, args in (
                ("rrq_cache_write", [P, P, P, P, I32, I64, I64, I64, I64, P]),
                ("rrq_cache_read", [P, P, P, P, I32, P]),
                ("rrq_cache_attention", [P, P, P, I32, I64, I64, I32, F, I32, I64, P, I32, P, SZ,
                                         P]),
                ("rrq_cache_attention_workspace", [P, P, I32, P]),
                ("rrq_token_logprobs", [P, I32, I64, I64, I64, P, I32, P, P, P, P, P, SZ, P]),
                ("rrq_token_logprobs_workspace", [I64, I64, I32, P])):
            f = getattr(lib, name)
            f.argtypes, f.restype = args, ctypes.c_int
        _lib = lib
    return _lib


def _checked(status: int, where: str) -> None:
    if status != RRQ_OK:
        raise RRQError(status, where)


# ---------------------------------------------------------------------------
# C ABI, one to one (cache: RrqCache, batch: RrqBatch)
# ---------------------------------------------------------------------------

def rrq_cache_write(cache, batch, K, V, dtype: int, k_token_stride: int, k_head_stride: int,
                    v_token_stride: int, v_head_stride: int, stream=None) -> None:
    """Enqueue the quantised write of a batch's keys and values (see rrq_serve.h)."""
    _checked(_library().rrq_cache_write(ctypes.byref(cache), ctypes.byref(batch), _ptr(K), _ptr(V),
                                        dtype, k_token_stride, k_head_stride, v_token_stride,
                                        v_head_stride, _stream(stream)), "rrq_cache_write")


def rrq_cache_read(cache, batch, K_out, V_out, out_dtype: int, stream=None) -> None:
    """Enqueue the read of a batch's keys and values (see rrq_serve.h)."""
    _checked(_library().rrq_cache_read(ctypes.byref(cache), ctypes.byref(batch), _ptr(K_out),
                                       _ptr(V_out), out_dtype, _stream(stream)), "rrq_cache_read")


def rrq_cache_attention(cache, batch, Q, q_dtype: int, q_token_stride: int, q_head_stride: int,
                        n_heads: int, scale: float, causal: int, window: int, out,
                        out_dtype: int, workspace, workspace_bytes: int, stream=None) -> None:
    """Enqueue attention of a batch's tokens over the cache (see rrq_serve.h)."""
    _checked(_library().rrq_cache_attention(ctypes.byref(cache), ctypes.byref(batch), _ptr(Q),
                                            q_dtype, q_token_stride, q_head_stride, n_heads,
                                            scale, causal, window, _ptr(out), out_dtype,
                                            _ptr(workspace), workspace_bytes, _stream(stream)),
             "rrq_cache_attention")


def rrq_cache_attention_workspace(cache, batch, n_heads: int) -> int:
    """Bytes of workspace rrq_cache_attention needs."""
    n = ctypes.c_size_t(0)
    _checked(_library().rrq_cache_attention_workspace(ctypes.byref(cache), ctypes.byref(batch),
                                                      n_heads, ctypes.byref(n)),
             "rrq_cache_attention_workspace")
    return n.value


def rrq_token_logprobs(logits, dtype: int, n_rows: int, vocab: int, row_stride: int, targets,
                       n_top: int, logprobs, entropy, top_ids, top_logprobs, workspace,
                       workspace_bytes: int, stream=None) -> None:
    """Enqueue token scoring (see rrq_serve.h)."""
    _checked(_library().rrq_token_logprobs(_ptr(logits), dtype, n_rows, vocab, row_stride,
                                           _ptr(targets), n_top, _ptr(logprobs), _ptr(entropy),
                                           _ptr(top_ids), _ptr(top_logprobs), _ptr(workspace),
                                           workspace_bytes, _stream(stream)),
             "rrq_token_logprobs")


def rrq_token_logprobs_workspace(n_rows: int, vocab: int, n_top: int) -> int:
    """Bytes of workspace rrq_token_logprobs needs."""
    n = ctypes.c_size_t(0)
    _checked(_library().rrq_token_logprobs_workspace(n_rows, vocab, n_top, ctypes.byref(n)),
             "rrq_token_logprobs_workspace")
    return n.value


# ---------------------------------------------------------------------------
# Tensor-level helpers
# ---------------------------------------------------------------------------

class KVCache:
    """One layer's 8-bit cache: k_codes uint8 [n_pages, n_kv_heads, page_size,
    head_dim], v_codes uint8 [n_pages, n_kv_heads, head_dim, page_size],
    k_scales and v_scales float32 [n_pages, n_kv_heads] (finite, 0 or more), all
    contiguous on one GPU. code_type: "int8" or "fp8" (e4m3)."""

    def __init__(self, k_codes, v_codes, k_scales, v_scales, code_type: str = "int8"):
        if code_type not in CODE_TYPES:
            raise ValueError(f"code_type must be one of {sorted(CODE_TYPES)}, got {code_type!r}")
        for t, name, dtype in ((k_codes, "k_codes", torch.uint8), (v_codes, "v_codes", torch.uint8),
                               (k_scales, "k_scales", torch.float32),
                               (v_scales, "v_scales", torch.float32)):
            _check_device_tensor(t, name, dtype)
        if k_codes.dim() != 4:
            raise ValueError("k_codes must be [n_pages, n_kv_heads, page_size, head_dim]")
        pages, heads, page, dim = k_codes.shape
        if tuple(v_codes.shape) != (pages, heads, dim, page):
            raise ValueError(f"v_codes must be {(pages, heads, dim, page)}, got "
                             f"{tuple(v_codes.shape)}")
        for t, name in ((k_scales, "k_scales"), (v_scales, "v_scales")):
            if tuple(t.shape) != (pages, heads):
                raise ValueError(f"{name} must be {(pages, heads)}, got {tuple(t.shape)}")
        if len({t.device for t in (k_codes, v_codes, k_scales, v_scales)}) != 1:
            raise ValueError("the cache's tensors must be on one device")
        self.k_codes, self.v_codes = k_codes, v_codes
        self.k_scales, self.v_scales = k_scales, v_scales
        self.code_type = code_type
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = pages, heads, page, dim
        self.device = k_codes.device
        self.index = k_codes.get_device()
        self.tensors = (k_codes, v_codes, k_scales, v_scales)
        self.desc = RrqCache(_ptr(k_codes), _ptr(v_codes), _ptr(k_scales), _ptr(v_scales), pages,
                             heads, dim, page, CODE_TYPES[code_type])
        self.ref = ctypes.byref(self.desc)

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, page_size: int = 64,
              code_type: str = "int8", device="cuda") -> "KVCache":
        """A cache of uninitialised pages (a page needs no initial value)."""
        return cls(torch.empty((n_pages, n_kv_heads, page_size, head_dim), dtype=torch.uint8,
                               device=device),
                   torch.empty((n_pages, n_kv_heads, head_dim, page_size), dtype=torch.uint8,
                               device=device),
                   torch.empty((n_pages, n_kv_heads), dtype=torch.float32, device=device),
                   torch.empty((n_pages, n_kv_heads), dtype=torch.float32, device=device),
                   code_type)


class CacheBatch:
    """Which tokens of which sequences a call works on (struct rrq_batch):
    page_table int32 [n_seqs, max_pages] (rows may be strided), lengths int32
    [n_seqs], offsets int32 [n_seqs + 1], all on the GPU; n_tokens rows in the
    call's dense tensors (offsets[n_seqs])."""

    def __init__(self, page_table, lengths, offsets, n_tokens: int):
        for t, name in ((page_table, "page_table"), (lengths, "lengths"), (offsets, "offsets")):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name} must be a torch.Tensor")
            if not t.is_cuda:
                raise ValueError(f"{name} must be on a GPU device, got {t.device}")
            if t.dtype != torch.int32:
                raise TypeError(f"{name} must have dtype torch.int32, got {t.dtype}")
            if t.dim() > 0 and t.shape[-1] > 1 and t.stride(-1) != 1:
                raise ValueError(f"{name} must be contiguous in its last dimension")
        if page_table.dim() != 2:
            raise ValueError("page_table must be [n_seqs, max_pages]")
        n_seqs, max_pages = page_table.shape
        if tuple(lengths.shape) != (n_seqs,) or tuple(offsets.shape) != (n_seqs + 1,):
            raise ValueError(f"lengths must be [{n_seqs}] and offsets [{n_seqs + 1}], got "
                             f"{tuple(lengths.shape)} and {tuple(offsets.shape)}")
        if len({t.device for t in (page_table, lengths, offsets)}) != 1:
            raise ValueError("the batch's tensors must be on one device")
        # the stride of a single row means nothing
        stride = page_table.stride(0) if n_seqs > 1 else max_pages
        self.page_table, self.lengths, self.offsets = page_table, lengths, offsets
        self.n_seqs, self.max_pages, self.n_tokens = n_seqs, max_pages, int(n_tokens)
        self.device = page_table.device
        self.index = page_table.get_device()
        self.tensors = (page_table, lengths, offsets)
        self.workspace_bytes = {}       # by the cache's sizes and the head count
        self.desc = RrqBatch(_ptr(page_table), _ptr(lengths), _ptr(offsets), stride, max_pages,
                             n_seqs, self.n_tokens)
        self.ref = ctypes.byref(self.desc)


_DTYPES = {torch.float32: RRQ_F32, torch.bfloat16: RRQ_BF16}


def _dtype_code(dtype, name: str) -> int:
    code = _DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"{name} must be torch.float32 or torch.bfloat16, got {dtype}")
    return code


def _row_strides(t, name: str, rows: int, heads, dim: int, index: int):
    """Checks that t is [rows, heads, dim] on the GPU of that index with
    contiguous last dimension. Returns its token and head stride; one that is
    never used (one token, one head) may be anything, so it counts as 0."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.get_device() != index:
        raise ValueError(f"{name} must be on cuda:{index}, got {t.device}")
    shape = t.shape
    if len(shape) != 3 or shape[0] != rows or shape[2] != dim or (heads and shape[1] != heads):
        raise ValueError(f"{name} must be [{rows}, {heads or 'heads'}, {dim}], got {tuple(shape)}")
    token, head, one = t.stride()
    if one != 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")
    return token if rows > 1 else 0, head if shape[1] > 1 else 0


def _check_out(out, name, shape, dtype, index):
    _check_device_tensor(out, name, dtype)
    if out.get_device() != index or tuple(out.shape) != tuple(shape):
        raise ValueError(f"{name} must be {tuple(shape)} on cuda:{index}, got {tuple(out.shape)} "
                         f"on {out.device}")


def _device_index(cache, batch) -> int:
    if cache.index != batch.index:
        raise ValueError(f"cache and batch must be on one device, got cuda:{cache.index} and "
                         f"cuda:{batch.index}")
    return cache.index


def cache_write(cache: KVCache, batch: CacheBatch, K, V, stream=None) -> None:
    """Quantise keys and values [n_tokens, n_kv_heads, head_dim] (float32 or
    bfloat16, any token and head strides of whole 16 bytes) into the batch's
    pages."""
    index = _device_index(cache, batch)
    if elsewhere(index, stream):
        with on_stream(index, stream, *cache.tensors, *batch.tensors, K, V):
            return cache_write(cache, batch, K, V)
    rows, heads, dim = batch.n_tokens, cache.n_kv_heads, cache.head_dim
    kt, kh = _row_strides(K, "K", rows, heads, dim, index)
    vt, vh = _row_strides(V, "V", rows, heads, dim, index)
    if K.dtype != V.dtype:
        raise TypeError(f"K and V must have one dtype, got {K.dtype} and {V.dtype}")
    st = (_lib or _library()).rrq_cache_write(cache.ref, batch.ref, K.data_ptr(), V.data_ptr(),
                                              _dtype_code(K.dtype, "K"), kt, kh, vt, vh,
                                              _stream(None))
    if st != RRQ_OK:
        raise RRQError(st, "rrq_cache_write")


def cache_read(cache: KVCache, batch: CacheBatch, dtype=None, stream=None, out=None):
    """(K, V) [n_tokens, n_kv_heads, head_dim] of the batch's tokens, dequantised
    to float32 or bfloat16 (the default). ``out`` may pass the pair."""
    index = _device_index(cache, batch)
    if elsewhere(index, stream):
        used = (*cache.tensors, *batch.tensors, *(() if out is None else out))
        with on_stream(index, stream, *used) as there:
            return there.returned(cache_read(cache, batch, dtype, out=out))
    shape = (batch.n_tokens, cache.n_kv_heads, cache.head_dim)
    if out is None:
        dtype = torch.bfloat16 if dtype is None else dtype
        code = _dtype_code(dtype, "dtype")
        K = torch.empty(shape, dtype=dtype, device=cache.device)
        V = torch.empty_like(K)         # (quicker)
    else:
        K, V = out
        dtype = K.dtype if dtype is None else dtype
        code = _dtype_code(dtype, "dtype")
        _check_out(K, "out[0]", shape, dtype, index)
        _check_out(V, "out[1]", shape, dtype, index)
    st = (_lib or _library()).rrq_cache_read(cache.ref, batch.ref, K.data_ptr(), V.data_ptr(),
                                             code, _stream(None))
    if st != RRQ_OK:
        raise RRQError(st, "rrq_cache_read")
    return K, V


def _workspace(n_bytes: int, device):
    return torch.empty(n_bytes, dtype=torch.uint8, device=device) if n_bytes else None


def _workspace_args(w, index: int):
    """Address and bytes of a caller's workspace."""
    if w is None:
        return None, 0
    if (not isinstance(w, torch.Tensor) or w.dtype != torch.uint8 or w.get_device() != index or
            not w.is_contiguous()):
        raise ValueError(f"workspace must be a contiguous uint8 tensor on cuda:{index}")
    return w.data_ptr(), w.numel()


def _attention_bytes(cache, batch, n_heads: int) -> int:
    # (a function of these sizes alone)
    key = (cache.n_kv_heads, cache.head_dim, cache.page_size, n_heads)
    n = batch.workspace_bytes.get(key)
    if n is None:
        n = rrq_cache_attention_workspace(cache.desc, batch.desc, n_heads)
        batch.workspace_bytes[key] = n
    return n


def attention_workspace(cache: KVCache, batch: CacheBatch, n_heads: int):
    """A workspace for cache_attention on this cache, batch and head count
    (uint8 tensor, or None if none is needed; allocated, like any tensor, for the
    current stream). Calls that may run at the same time need their own."""
    return _workspace(_attention_bytes(cache, batch, n_heads), cache.device)


def cache_attention(cache: KVCache, batch: CacheBatch, Q, scale=None, causal: bool = True,
                    window: int = 0, out_dtype=None, workspace=None, stream=None, out=None):
    """Attention of queries [n_tokens, n_heads, head_dim] (float32 or bfloat16)
    over the batch's sequences: [n_tokens, n_heads, head_dim] in bfloat16 (the
    default) or float32. scale defaults to head_dim ** -0.5; window 0 is none. A
    float32 result is computed with operands of 22 bits, a bfloat16 one of 11
    (see rrq_serve.h)."""
    index = _device_index(cache, batch)
    if elsewhere(index, stream):
        with on_stream(index, stream, *cache.tensors, *batch.tensors, Q, workspace, out) as there:
            return there.returned(cache_attention(cache, batch, Q, scale, causal, window,
                                                  out_dtype, workspace, out=out))
    dim = cache.head_dim
    qt, qh = _row_strides(Q, "Q", batch.n_tokens, None, dim, index)
    shape = Q.shape
    n_heads = shape[1]
    if out is None:
        out_dtype = torch.bfloat16 if out_dtype is None else out_dtype
        out_code = _dtype_code(out_dtype, "out_dtype")
        out = torch.empty(shape, dtype=out_dtype, device=cache.device)
    else:
        out_dtype = out.dtype if out_dtype is None else out_dtype
        out_code = _dtype_code(out_dtype, "out")
        _check_out(out, "out", shape, out_dtype, index)
    if workspace is None:
        workspace = _workspace(_attention_bytes(cache, batch, n_heads), cache.device)
    w, w_bytes = _workspace_args(workspace, index)
    st = (_lib or _library()).rrq_cache_attention(
        cache.ref, batch.ref, Q.data_ptr(), _dtype_code(Q.dtype, "Q"), qt, qh, n_heads,
        1.0 / math.sqrt(dim) if scale is None else scale, 1 if causal else 0, window,
        out.data_ptr(), out_code, w, w_bytes, _stream(None))
    if st != RRQ_OK:
        raise RRQError(st, "rrq_cache_attention")
    return out


def logprobs_workspace(logits, n_top: int = 0):
    """A workspace for token_logprobs on logits of this shape (uint8 tensor, or
    None if none is needed). Calls that may run at the same time need their own."""
    return _workspace(rrq_token_logprobs_workspace(logits.shape[0], logits.shape[1], n_top),
                      logits.device)


def token_logprobs(logits, targets=None, n_top: int = 0, workspace=None, stream=None):
    """(logprobs, entropy, top_ids, top_logprobs) of logits [rows, vocab]
    (float32 or bfloat16, rows may be strided): the log probability of each
    row's target (int64 [rows]; one outside the vocabulary gives 0), the
    entropy, and the n_top likeliest tokens. logprobs is None without targets,
    top_ids and top_logprobs are None for n_top = 0."""
    if not isinstance(logits, torch.Tensor):
        raise TypeError("logits must be a torch.Tensor")
    index = logits.get_device()
    if index < 0:
        raise ValueError(f"logits must be on a GPU device, got {logits.device}")
    if elsewhere(index, stream):
        with on_stream(index, stream, logits, targets, workspace) as there:
            return there.returned(token_logprobs(logits, targets, n_top, workspace))
    code = _dtype_code(logits.dtype, "logits")
    if logits.dim() != 2:
        raise ValueError(f"logits must be [rows, vocab], got {tuple(logits.shape)}")
    rows, vocab = logits.shape
    row_stride, one = logits.stride()
    if vocab > 1 and one != 1:
        raise ValueError("logits must be contiguous in its last dimension")
    device = logits.device
    logprobs = top_ids = top_logprobs = target_ptr = logprob_ptr = id_ptr = top_ptr = None
    if targets is not None:
        if (not isinstance(targets, torch.Tensor) or targets.dtype != torch.int64 or
                targets.get_device() != index or tuple(targets.shape) != (rows,) or
                not targets.is_contiguous()):
            raise ValueError(f"targets must be a contiguous int64 tensor [{rows}] on {device}")
        logprobs = torch.empty(rows, dtype=torch.float32, device=device)
        target_ptr, logprob_ptr = targets.data_ptr(), logprobs.data_ptr()
    entropy = (torch.empty(rows, dtype=torch.float32, device=device) if logprobs is None else
               torch.empty_like(logprobs))
    if n_top > 0:
        top_ids = torch.empty((rows, n_top), dtype=torch.int64, device=device)
        top_logprobs = torch.empty((rows, n_top), dtype=torch.float32, device=device)
        id_ptr, top_ptr = top_ids.data_ptr(), top_logprobs.data_ptr()
    if workspace is None:
        workspace = _workspace(rrq_token_logprobs_workspace(rows, vocab, n_top), device)
    w, w_bytes = _workspace_args(workspace, index)
    st = (_lib or _library()).rrq_token_logprobs(
        logits.data_ptr(), code, rows, vocab, row_stride if rows > 1 else vocab, target_ptr, n_top,
        logprob_ptr, entropy.data_ptr(), id_ptr, top_ptr, w, w_bytes, _stream(None))
    if st != RRQ_OK:
        raise RRQError(st, "rrq_token_logprobs")
    return logprobs, entropy, top_ids, top_logprobs
