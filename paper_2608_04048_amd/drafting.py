"""What a decoder that drafts tokens with a short prefix of its packages and
checks them with a longer one runs beside the calls of ``serving``.

Binding of include/rrq_draft.h in librrq.so. The functions named like the C ABI
marshal arguments one to one; the others take torch tensors, check them and
allocate the outputs. Every computation runs in the HIP kernels.

    x, h = block_norm(h, y, weight)          # residual, and rrq_linear's next X
    rotary = Rotary(rotary_frequencies(128))
    Q = cache_append(cache, batch, rotary, Q, K, V, positions)
    out = tree_attention(cache, batch, Q, seen, positions)
    counts, following, paths = verify_drafts(logits, tokens, offsets, 5, uniforms, draft_logits)

Forward only, and ``stream`` as in ``serving``.
"""

from __future__ import annotations

import ctypes
import math

import torch

from . import RRQ_BF16, RRQ_F32, RRQ_OK, RRQError, _ptr, _stream, load_library
from .placement import elsewhere, on_stream
from .serving import (CacheBatch, KVCache, _attention_bytes, _check_out, _checked,
                      _device_index, _dtype_code, _row_strides, _workspace, _workspace_args)

RRQ_NORM_NONE = 0
RRQ_NORM_RMS = 1
RRQ_NORM_LAYER = 2
NORM_KINDS = {"rms": RRQ_NORM_RMS, "layer": RRQ_NORM_LAYER}
RRQ_ROTARY_HALF = 0
RRQ_ROTARY_INTERLEAVED = 1
ROTARY_LAYOUTS = {"half": RRQ_ROTARY_HALF, "interleaved": RRQ_ROTARY_INTERLEAVED}


class RrqNorm(ctypes.Structure):
    """struct rrq_norm of rrq_draft.h."""
    _fields_ = [("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("post_weight", ctypes.c_void_p), ("kind", ctypes.c_int32),
                ("post", ctypes.c_int32), ("eps", ctypes.c_float), ("scale", ctypes.c_float)]


class RrqRotary(ctypes.Structure):
    """struct rrq_rotary of rrq_draft.h."""
    _fields_ = [("frequencies", ctypes.c_void_p), ("amplitude", ctypes.c_double),
                ("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        P, I64, I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
        F, SZ = ctypes.c_float, ctypes.c_size_t
        for name, args in (
                ("rrq_block_norm", [P, P, I32, I64, P, I32, I64, P, I64, I64, I64, P, I32, P, P]),
                ("rrq_cache_append", [P, P, P, P, P, P, P, I32, I64, I64, I64, I64, I64, I64, I32,
                                      P, P]),
                ("rrq_tree_attention", [P, P, P, I32, I64, I64, I32, F, P, I64, P, I64, P, I32, P,
                                        SZ, P]),
                ("rrq_verify_drafts", [P, I32, I64, I64, I64, P, P, I64, P, P, P, I64, I64,
                                       ctypes.c_double, ctypes.c_double, I32, P, P, P, P, SZ, P]),
                ("rrq_verify_drafts_workspace", [I64, I64, I64, I64, P])):
            f = getattr(lib, name)
            f.argtypes, f.restype = args, ctypes.c_int
        _lib = lib
    return _lib


# ---------------------------------------------------------------------------
# C ABI, one to one (cache: RrqCache, batch: RrqBatch, norm: RrqNorm, rotary:
# RrqRotary)
# ---------------------------------------------------------------------------

def rrq_block_norm(norm, residual, residual_dtype: int, residual_stride: int, y, y_dtype: int,
                   y_stride: int, gate, gate_stride: int, n_rows: int, hidden: int, out,
                   out_dtype: int, h, stream=None) -> None:
    """Enqueue the norms between two blocks (see rrq_draft.h)."""
    _checked(_library().rrq_block_norm(ctypes.byref(norm), _ptr(residual), residual_dtype,
                                       residual_stride, _ptr(y), y_dtype, y_stride, _ptr(gate),
                                       gate_stride, n_rows, hidden, _ptr(out), out_dtype, _ptr(h),
                                       _stream(stream)), "rrq_block_norm")


def rrq_cache_append(cache, batch, rotary, positions, Q, K, V, dtype: int, q_token_stride: int,
                     q_head_stride: int, k_token_stride: int, k_head_stride: int,
                     v_token_stride: int, v_head_stride: int, n_heads: int, Q_out,
                     stream=None) -> None:
    """Enqueue the rotation of a batch's queries and keys and the quantised write of
    its keys and values (see rrq_draft.h)."""
    _checked(_library().rrq_cache_append(ctypes.byref(cache), ctypes.byref(batch),
                                         ctypes.byref(rotary), _ptr(positions), _ptr(Q), _ptr(K),
                                         _ptr(V), dtype, q_token_stride, q_head_stride,
                                         k_token_stride, k_head_stride, v_token_stride,
                                         v_head_stride, n_heads, _ptr(Q_out), _stream(stream)),
             "rrq_cache_append")


def rrq_tree_attention(cache, batch, Q, q_dtype: int, q_token_stride: int, q_head_stride: int,
                       n_heads: int, scale: float, seen, seen_words: int, positions, window: int,
                       out, out_dtype: int, workspace, workspace_bytes: int, stream=None) -> None:
    """Enqueue attention of drafted tokens over the cache (see rrq_draft.h)."""
    _checked(_library().rrq_tree_attention(ctypes.byref(cache), ctypes.byref(batch), _ptr(Q),
                                           q_dtype, q_token_stride, q_head_stride, n_heads, scale,
                                           _ptr(seen), seen_words, _ptr(positions), window,
                                           _ptr(out), out_dtype, _ptr(workspace), workspace_bytes,
                                           _stream(stream)), "rrq_tree_attention")


def rrq_verify_drafts(logits, dtype: int, n_rows: int, vocab: int, row_stride: int, tokens,
                      offsets, n_seqs: int, uniforms, parents, draft, draft_seq_stride: int,
                      draft_row_stride: int, temperature: float, draft_temperature: float,
                      max_accept: int, counts, following, paths, workspace, workspace_bytes: int,
                      stream=None) -> None:
    """Enqueue the verification of drafted tokens (see rrq_draft.h)."""
    _checked(_library().rrq_verify_drafts(_ptr(logits), dtype, n_rows, vocab, row_stride,
                                          _ptr(tokens), _ptr(offsets), n_seqs, _ptr(uniforms),
                                          _ptr(parents), _ptr(draft), draft_seq_stride,
                                          draft_row_stride, temperature, draft_temperature,
                                          max_accept, _ptr(counts), _ptr(following), _ptr(paths),
                                          _ptr(workspace), workspace_bytes, _stream(stream)),
             "rrq_verify_drafts")


def rrq_verify_drafts_workspace(n_rows: int, vocab: int, n_seqs: int, draft_rows: int) -> int:
    """Bytes of workspace rrq_verify_drafts needs."""
    n = ctypes.c_size_t(0)
    _checked(_library().rrq_verify_drafts_workspace(n_rows, vocab, n_seqs, draft_rows,
                                                    ctypes.byref(n)),
             "rrq_verify_drafts_workspace")
    return n.value


# ---------------------------------------------------------------------------
# Tensor-level helpers
# ---------------------------------------------------------------------------

def _matrix(t, name: str, rows: int, cols: int, index: int) -> int:
    """Checks that t is [rows, cols] on the GPU of that index, contiguous in its
    last dimension; its row stride."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.get_device() != index:
        raise ValueError(f"{name} must be on cuda:{index}, got {t.device}")
    if t.shape != (rows, cols):
        raise ValueError(f"{name} must be {(rows, cols)}, got {tuple(t.shape)}")
    stride, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")
    return stride


def _vector(t, name: str, cols: int, dtype, index: int):
    """Address of a contiguous vector; None for None."""
    if t is None:
        return None
    if (not isinstance(t, torch.Tensor) or t.dtype != dtype or t.get_device() != index or
            t.shape != (cols,) or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor [{cols}] on cuda:{index}")
    return t.data_ptr()


def block_norm(residual, y=None, weight=None, bias=None, kind: str = "rms", post=None,
               post_weight=None, gate=None, scale: float = 1.0, eps: float = 1e-6, out_dtype=None,
               stream=None, out=None):
    """(out, h) of h = residual + scale * gate * post(y) * post_weight and
    out = kind(h) * weight + bias, row by row.

    residual [rows, hidden] and the block's output y of that shape are float32 or
    bfloat16 each, their rows may be strided (columns of a wider tensor); without y
    the residual is normalised and returned as h. kind is "rms" or "layer", post
    one of them or None (no norm of y). weight, bias and post_weight are float32
    [hidden] or None. gate, of y's type, is [hidden] or [rows, hidden] (rows may be
    strided). h has the residual's type, out is bfloat16 (the default: rrq_linear's
    X) or float32. ``out`` may pass the pair; its second may be the residual
    itself, which is then updated in place."""
    if not isinstance(residual, torch.Tensor):
        raise TypeError("residual must be a torch.Tensor")
    index = residual.get_device()
    if index < 0:
        raise ValueError(f"residual must be on a GPU device, got {residual.device}")
    if elsewhere(index, stream):
        used = (residual, y, weight, bias, post_weight, gate, *(() if out is None else out))
        with on_stream(index, stream, *used) as there:
            return there.returned(block_norm(residual, y, weight, bias, kind, post, post_weight,
                                             gate, scale, eps, out_dtype, out=out))
    kind_code = NORM_KINDS.get(kind)
    post_code = RRQ_NORM_NONE if post is None else NORM_KINDS.get(post)
    if kind_code is None or post_code is None:
        raise ValueError(f"kind and post must be of {sorted(NORM_KINDS)} (post may be None), got "
                         f"{kind!r} and {post!r}")
    if residual.dim() != 2:
        raise ValueError(f"residual must be [rows, hidden], got {tuple(residual.shape)}")
    rows, cols = residual.shape
    r_code = _dtype_code(residual.dtype, "residual")
    r_stride = _matrix(residual, "residual", rows, cols, index)
    y_ptr = gate_ptr = h_ptr = None
    y_stride = gate_stride = 0
    y_code = r_code
    if y is None:
        if post is not None or post_weight is not None or gate is not None:
            raise ValueError("post, post_weight and gate need y")
    else:
        y_stride = _matrix(y, "y", rows, cols, index)
        y_code = _dtype_code(y.dtype, "y")
        y_ptr = y.data_ptr()
        if post is None and post_weight is not None:
            raise ValueError("post_weight needs post")
        if gate is not None:
            if isinstance(gate, torch.Tensor) and gate.dim() == 2:
                gate_stride = _matrix(gate, "gate", rows, cols, index)
                if gate.dtype != y.dtype:
                    raise TypeError(f"gate must have y's dtype {y.dtype}, got {gate.dtype}")
                gate_ptr = gate.data_ptr()
                if rows > 1 and gate_stride < cols:
                    raise ValueError("gate's rows must not overlap; one row for all is [hidden]")
            else:
                gate_ptr = _vector(gate, "gate", cols, y.dtype, index)
    if out is None:
        out_dtype = torch.bfloat16 if out_dtype is None else out_dtype
        out_code = _dtype_code(out_dtype, "out_dtype")
        h = torch.empty_like(residual, memory_format=torch.contiguous_format)
        x = torch.empty_like(h, dtype=out_dtype)
        h = h if y is not None else residual
    else:
        x, h = out
        for t, name in ((x, "out[0]"), (h, "out[1]")):
            _matrix(t, name, rows, cols, index)
            if not t.is_contiguous() and y is not None:
                raise ValueError(f"{name} must be contiguous")
        if not x.is_contiguous():
            raise ValueError("out[0] must be contiguous")
        out_code = _dtype_code(x.dtype, "out[0]")
        if out_dtype is not None and x.dtype != out_dtype:
            raise TypeError(f"out[0] must have dtype {out_dtype}, got {x.dtype}")
        if h.dtype != residual.dtype:
            raise TypeError(f"out[1] must have the residual's dtype, got {h.dtype}")
        if y is None and h is not residual:
            raise ValueError("without y, out[1] must be the residual itself")
    if y is not None:
        h_ptr = h.data_ptr()
    norm = RrqNorm(_vector(weight, "weight", cols, torch.float32, index),
                   _vector(bias, "bias", cols, torch.float32, index),
                   _vector(post_weight, "post_weight", cols, torch.float32, index),
                   kind_code, post_code, eps, scale)
    st = (_lib or _library()).rrq_block_norm(
        ctypes.byref(norm), residual.data_ptr(), r_code, r_stride, y_ptr, y_code, y_stride,
        gate_ptr, gate_stride, rows, cols, x.data_ptr(), out_code, h_ptr, _stream(None))
    if st != RRQ_OK:
        raise RRQError(st, "rrq_block_norm")
    return x, h


def rotary_frequencies(rot_dim: int, base: float = 10000.0, stretch: float = 1.0,
                       trained: int = 32768, slow: float = 1.0, fast: float = 32.0,
                       device="cuda"):
    """float64 [rot_dim / 2]: pair i turns by base ** (-2 i / rot_dim) a position.

    For a context `stretch` times the `trained` one, pairs that turn less than
    `slow` times in the trained context are slowed by the stretch, those that turn
    more than `fast` times stay, and between them the share that stays is linear in
    the turns."""
    f = base ** (-torch.arange(rot_dim // 2, dtype=torch.float64) * 2 / rot_dim)
    if stretch != 1.0:
        stay = ((trained * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        f = f * stay + f / stretch * (1 - stay)
    return f.to(device)


class Rotary:
    """Rotary positions: frequencies float64 [rot_dim / 2] on the GPU (radians a
    position), of which pair i is channels i and i + rot_dim / 2 (layout "half") or
    2 i and 2 i + 1 ("interleaved") of a head; further channels stay as they are.
    amplitude multiplies what is rotated."""

    def __init__(self, frequencies, layout: str = "half", amplitude: float = 1.0):
        if layout not in ROTARY_LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(ROTARY_LAYOUTS)}, got {layout!r}")
        if not isinstance(frequencies, torch.Tensor):
            raise TypeError("frequencies must be a torch.Tensor")
        if frequencies.dtype != torch.float64:
            raise TypeError(f"frequencies must have dtype torch.float64, got {frequencies.dtype}")
        if not frequencies.is_cuda:
            raise ValueError(f"frequencies must be on a GPU device, got {frequencies.device}")
        if frequencies.dim() != 1 or not frequencies.is_contiguous():
            raise ValueError("frequencies must be a contiguous vector")
        self.frequencies, self.layout, self.amplitude = frequencies, layout, float(amplitude)
        self.rot_dim = 2 * frequencies.shape[0]
        self.index = frequencies.get_device()
        self.desc = RrqRotary(_ptr(frequencies), self.amplitude, self.rot_dim,
                              ROTARY_LAYOUTS[layout])
        self.ref = ctypes.byref(self.desc)


def _check_positions(positions, rows: int, index: int):
    """Address of a batch's positions; None for None."""
    return _vector(positions, "positions", rows, torch.int32, index)


def cache_append(cache: KVCache, batch: CacheBatch, rotary: Rotary, Q, K, V, positions=None,
                 stream=None, out=None):
    """Rotate the batch's queries [n_tokens, n_heads, head_dim] and keys, and quantise
    keys and values [n_tokens, n_kv_heads, head_dim] into their pages: float32 or
    bfloat16, one type, any token and head strides of whole 16 bytes. positions
    (int32 [n_tokens]) defaults to the rows' places in their sequences. Returns the
    rotated queries; ``out`` may pass their tensor, Q itself as well."""
    index = _device_index(cache, batch)
    if elsewhere(index, stream):
        used = (*cache.tensors, *batch.tensors, rotary.frequencies, Q, K, V, positions, out)
        with on_stream(index, stream, *used) as there:
            return there.returned(cache_append(cache, batch, rotary, Q, K, V, positions, out=out))
    if rotary.index != index:
        raise ValueError(f"rotary must be on cuda:{index}, got cuda:{rotary.index}")
    rows, heads, dim = batch.n_tokens, cache.n_kv_heads, cache.head_dim
    qt, qh = _row_strides(Q, "Q", rows, None, dim, index)
    kt, kh = _row_strides(K, "K", rows, heads, dim, index)
    vt, vh = _row_strides(V, "V", rows, heads, dim, index)
    dtype = Q.dtype
    if K.dtype != dtype or V.dtype != dtype:
        raise TypeError(f"Q, K and V must have one dtype, got {dtype}, {K.dtype} and {V.dtype}")
    code = _dtype_code(dtype, "Q")
    at = _check_positions(positions, rows, index)
    if out is None:
        # (1.2 us; torch.empty with this shape and device 2.1)
        out = torch.empty_like(Q, memory_format=torch.contiguous_format)
    else:
        _check_out(out, "out", Q.shape, dtype, index)
    st = (_lib or _library()).rrq_cache_append(
        cache.ref, batch.ref, rotary.ref, at, Q.data_ptr(), K.data_ptr(), V.data_ptr(), code,
        qt, qh, kt, kh, vt, vh, Q.shape[1], out.data_ptr(), _stream(None))
    if st != RRQ_OK:
        raise RRQError(st, "rrq_cache_append")
    return out


def tree_attention(cache: KVCache, batch: CacheBatch, Q, seen, positions=None, scale=None,
                   window: int = 0, out_dtype=None, workspace=None, stream=None, out=None):
    """Attention of drafted tokens, as ``serving.cache_attention`` (with its
    workspace, ``attention_workspace``): a row sees the positions before its
    sequence's rows of this batch (of its window, counted from its position), and of
    those rows the ones whose bits are set in its row of ``seen`` (int64 [n_tokens,
    words], contiguous: bit j % 64 of word j // 64 is the sequence's row j). All rows of
    the batch have to be in the cache, also those that no bit names. positions (int32
    [n_tokens]) defaults to the rows' places in their sequences."""
    index = _device_index(cache, batch)
    if elsewhere(index, stream):
        used = (*cache.tensors, *batch.tensors, Q, seen, positions, workspace, out)
        with on_stream(index, stream, *used) as there:
            return there.returned(tree_attention(cache, batch, Q, seen, positions, scale, window,
                                                 out_dtype, workspace, out=out))
    dim, rows = cache.head_dim, batch.n_tokens
    qt, qh = _row_strides(Q, "Q", rows, None, dim, index)
    shape = Q.shape
    n_heads = shape[1]
    if (not isinstance(seen, torch.Tensor) or seen.dtype != torch.int64 or
            seen.get_device() != index or seen.dim() != 2 or seen.shape[0] != rows or
            not seen.is_contiguous()):
        raise ValueError(f"seen must be a contiguous int64 tensor [{rows}, words] on cuda:{index}")
    at = _check_positions(positions, rows, index)
    if out is None:
        out_dtype = torch.bfloat16 if out_dtype is None else out_dtype
        out_code = _dtype_code(out_dtype, "out_dtype")
        out = torch.empty_like(Q, dtype=out_dtype, memory_format=torch.contiguous_format)
    else:
        out_dtype = out.dtype if out_dtype is None else out_dtype
        out_code = _dtype_code(out_dtype, "out")
        _check_out(out, "out", shape, out_dtype, index)
    if workspace is None:
        workspace = _workspace(_attention_bytes(cache, batch, n_heads), cache.device)
    w, w_bytes = _workspace_args(workspace, index)
    st = (_lib or _library()).rrq_tree_attention(
        cache.ref, batch.ref, Q.data_ptr(), _dtype_code(Q.dtype, "Q"), qt, qh, n_heads,
        1.0 / math.sqrt(dim) if scale is None else scale, seen.data_ptr(), seen.shape[1], at,
        window, out.data_ptr(), out_code, w, w_bytes, _stream(None))
    if st != RRQ_OK:
        raise RRQError(st, "rrq_tree_attention")
    return out


def _verify_bytes(logits, n_seqs: int, draft) -> int:
    rows = 0 if draft is None else draft.shape[0] * draft.shape[1]
    return rrq_verify_drafts_workspace(logits.shape[0], logits.shape[1], n_seqs, rows)


def verify_workspace(logits, n_seqs: int, draft=None):
    """A workspace for verify_drafts on logits and draft distributions of these shapes
    (uint8 tensor, or None if none is needed). Calls that may run at the same time
    need their own."""
    return _workspace(_verify_bytes(logits, n_seqs, draft), logits.device)


def verify_drafts(logits, tokens, offsets, max_accept: int, uniforms, draft=None, parents=None,
                  temperature: float = 1.0, draft_temperature: float = 1.0, workspace=None,
                  stream=None):
    """(counts, following, paths): how many drafted tokens of each sequence the target
    accepts, the token that follows them, and the accepted rows.

    logits [rows, vocab] (float32 or bfloat16, rows may be strided): rows offsets[b] ..
    offsets[b + 1] - 1 (offsets int32 [n_seqs + 1]) are the target's after sequence b's
    last token (row 0) and after each drafted one. tokens (int64 [rows]) holds the
    drafted tokens in rows 1 on, uniforms (float32 [rows], in [0, 1)) a random number
    for each, and in row 0 the one that the following token is drawn with. parents
    (int32 [rows], row numbers within the sequence) makes the drafts a tree; without it
    they are a chain. draft [n_seqs, max_accept, vocab] (a chain's only, of the logits'
    type) gives the distributions the drafts were drawn from, logits as well; without it
    a rejected token's probability is taken out. A temperature of 0 is greedy.

    counts is int32 [n_seqs], following int64 [n_seqs], paths int32 [n_seqs, max_accept + 1]:
    row 0, the accepted rows in order, then -1. At most max_accept drafts of a sequence are
    accepted. following is -1 for a sequence without rows, or that ends at a row of -inf or
    one with a NaN or +inf; at a temperature of 0 those are numbers as others (a NaN less
    than any), a row of -inf gives token 0, and only one of nothing but NaN -1."""
    if not isinstance(logits, torch.Tensor):
        raise TypeError("logits must be a torch.Tensor")
    index = logits.get_device()
    if index < 0:
        raise ValueError(f"logits must be on a GPU device, got {logits.device}")
    if elsewhere(index, stream):
        used = (logits, tokens, offsets, uniforms, draft, parents, workspace)
        with on_stream(index, stream, *used) as there:
            return there.returned(verify_drafts(logits, tokens, offsets, max_accept, uniforms,
                                                draft, parents, temperature, draft_temperature,
                                                workspace))
    code = _dtype_code(logits.dtype, "logits")
    if logits.dim() != 2:
        raise ValueError(f"logits must be [rows, vocab], got {tuple(logits.shape)}")
    rows, vocab = logits.shape
    row_stride = _matrix(logits, "logits", rows, vocab, index)
    if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError(f"offsets must be a contiguous int32 tensor [n_seqs + 1] on cuda:{index}")
    n_seqs = offsets.shape[0] - 1
    token_ptr = _vector(tokens, "tokens", rows, torch.int64, index)
    offset_ptr = _vector(offsets, "offsets", n_seqs + 1, torch.int32, index)
    uniform_ptr = _vector(uniforms, "uniforms", rows, torch.float32, index)
    parent_ptr = _vector(parents, "parents", rows, torch.int32, index)
    if token_ptr is None or uniform_ptr is None:
        raise TypeError("tokens and uniforms must be torch.Tensors")
    if max_accept < 0:
        raise ValueError(f"max_accept must be 0 or more, got {max_accept}")
    draft_ptr, seq_stride, draft_stride = None, 0, 0
    if draft is not None:
        if parents is not None:
            raise ValueError("draft distributions need a chain: parents must be None")
        if not isinstance(draft, torch.Tensor):
            raise TypeError("draft must be a torch.Tensor")
        if draft.get_device() != index:
            raise ValueError(f"draft must be on cuda:{index}, got {draft.device}")
        if tuple(draft.shape) != (n_seqs, max_accept, vocab):
            raise ValueError(f"draft must be {(n_seqs, max_accept, vocab)}, got "
                             f"{tuple(draft.shape)}")
        if draft.dtype != logits.dtype:
            raise TypeError(f"draft must have the logits' dtype {logits.dtype}, got {draft.dtype}")
        seq_stride, draft_stride, one = draft.stride()
        if one != 1 and vocab > 1:
            raise ValueError("draft must be contiguous in its last dimension")
        if draft.numel() > 0:
            draft_ptr = draft.data_ptr()
    counts = torch.empty(n_seqs, dtype=torch.int32, device=logits.device)
    following = torch.empty_like(counts, dtype=torch.int64)     # (quicker)
    paths = torch.empty((n_seqs, max_accept + 1), dtype=torch.int32, device=logits.device)
    if workspace is None:
        workspace = _workspace(_verify_bytes(logits, n_seqs, draft), logits.device)
    w, w_bytes = _workspace_args(workspace, index)
    st = (_lib or _library()).rrq_verify_drafts(
        logits.data_ptr(), code, rows, vocab, row_stride, token_ptr, offset_ptr, n_seqs,
        uniform_ptr, parent_ptr, draft_ptr, seq_stride, draft_stride, temperature,
        draft_temperature, max_accept, counts.data_ptr(), following.data_ptr(), paths.data_ptr(),
        w, w_bytes, _stream(None))
    if st != RRQ_OK:
        raise RRQError(st, "rrq_verify_drafts")
    return counts, following, paths
