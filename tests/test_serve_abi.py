"""include/rrq_serve.h: exports, workspace sizes, and the refusal of every bad
argument before any device work. No GPU needed."""

import ctypes
import os
import re

import pytest

import paper_2608_04048_amd as rrq
from paper_2608_04048_amd import serving

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "rrq_serve.h")
FAKE = 0x10000          # aligned, never dereferenced: every case fails validation first


def test_library_exports_every_declared_function():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(rrq_\w+)\s*\(", text)))
    assert names == ["rrq_cache_attention", "rrq_cache_attention_workspace", "rrq_cache_read",
                     "rrq_cache_write", "rrq_token_logprobs", "rrq_token_logprobs_workspace"]
    lib = rrq.load_library()
    for name in names:
        assert hasattr(lib, name) and hasattr(rrq, name), name
    for name, value in re.findall(r"\b(RRQ_[A-Z0-9_]+)\s*=\s*(\d+)", text):
        assert getattr(rrq, name) == int(value), name
    assert f"#define RRQ_MAX_TOP {rrq.RRQ_MAX_TOP}" in text


def test_structures_match_the_header():
    assert ctypes.sizeof(rrq.RrqCache) == 4 * 8 + 8 + 4 * 4
    assert ctypes.sizeof(rrq.RrqBatch) == 3 * 8 + 4 * 8
    assert "smaller" in rrq.rrq_status_string(rrq.RRQ_ERR_WORKSPACE)


def _cache(**kw):
    d = dict(k_codes=FAKE, v_codes=FAKE, k_scales=FAKE, v_scales=FAKE, n_pages=10, n_kv_heads=2,
             head_dim=128, page_size=64, code_type=0)
    d.update(kw)
    return rrq.RrqCache(**d)


def _batch(**kw):
    d = dict(page_table=FAKE, lengths=FAKE, offsets=FAKE, table_stride=5, max_pages=5, n_seqs=2,
             n_tokens=3)
    d.update(kw)
    return rrq.RrqBatch(**d)


def _ref(x):
    return ctypes.byref(x) if x is not None else None


CACHE_CASES = [
    (dict(k_codes=None), rrq.RRQ_ERR_NULL), (dict(v_codes=None), rrq.RRQ_ERR_NULL),
    (dict(k_scales=None), rrq.RRQ_ERR_NULL), (dict(v_scales=None), rrq.RRQ_ERR_NULL),
    (dict(k_codes=FAKE + 8), rrq.RRQ_ERR_ALIGN), (dict(v_codes=FAKE + 1), rrq.RRQ_ERR_ALIGN),
    (dict(k_scales=FAKE + 2), rrq.RRQ_ERR_ALIGN), (dict(v_scales=FAKE + 1), rrq.RRQ_ERR_ALIGN),
    (dict(n_pages=0), rrq.RRQ_ERR_SHAPE), (dict(n_pages=1 << 60), rrq.RRQ_ERR_SHAPE),
    (dict(n_kv_heads=0), rrq.RRQ_ERR_SHAPE), (dict(n_kv_heads=1025), rrq.RRQ_ERR_SHAPE),
    (dict(head_dim=96), rrq.RRQ_ERR_SHAPE), (dict(head_dim=0), rrq.RRQ_ERR_SHAPE),
    (dict(page_size=8), rrq.RRQ_ERR_SHAPE), (dict(page_size=48), rrq.RRQ_ERR_SHAPE),
    (dict(page_size=256), rrq.RRQ_ERR_SHAPE),
    (dict(code_type=2), rrq.RRQ_ERR_FORMAT), (dict(code_type=-1), rrq.RRQ_ERR_FORMAT),
]
BATCH_CASES = [
    (dict(page_table=None), rrq.RRQ_ERR_NULL), (dict(lengths=None), rrq.RRQ_ERR_NULL),
    (dict(offsets=None), rrq.RRQ_ERR_NULL), (dict(page_table=FAKE + 2), rrq.RRQ_ERR_ALIGN),
    (dict(lengths=FAKE + 1), rrq.RRQ_ERR_ALIGN), (dict(offsets=FAKE + 2), rrq.RRQ_ERR_ALIGN),
    (dict(max_pages=0), rrq.RRQ_ERR_SHAPE), (dict(table_stride=4), rrq.RRQ_ERR_SHAPE),
    (dict(n_seqs=-1), rrq.RRQ_ERR_SHAPE), (dict(n_seqs=(1 << 20) + 1), rrq.RRQ_ERR_SHAPE),
    (dict(n_tokens=-1), rrq.RRQ_ERR_SHAPE), (dict(n_tokens=(1 << 26) + 1), rrq.RRQ_ERR_SHAPE),
]


def _write(cache=_cache(), batch=_batch(), K=FAKE, V=FAKE, dtype=0, kt=1024, kh=128, vt=1024,
           vh=128):
    return serving._library().rrq_cache_write(_ref(cache), _ref(batch), K, V, dtype, kt, kh, vt,
                                              vh, None)


def _read(cache=_cache(), batch=_batch(), K=FAKE, V=FAKE, dtype=0):
    return serving._library().rrq_cache_read(_ref(cache), _ref(batch), K, V, dtype, None)


def _attend(cache=_cache(), batch=_batch(), Q=FAKE, dtype=0, qt=1024, qh=128, heads=4, scale=0.1,
            causal=1, window=0, out=FAKE, out_dtype=1, w=FAKE, wb=1 << 40):
    return serving._library().rrq_cache_attention(_ref(cache), _ref(batch), Q, dtype, qt, qh,
                                                  heads, scale, causal, window, out, out_dtype, w,
                                                  wb, None)


@pytest.mark.parametrize("call", [_write, _read, _attend])
@pytest.mark.parametrize("kw,status", CACHE_CASES)
def test_cache_descriptor_refusals(call, kw, status):
    assert call(cache=_cache(**kw)) == status


@pytest.mark.parametrize("call", [_write, _read, _attend])
@pytest.mark.parametrize("kw,status", BATCH_CASES)
def test_batch_descriptor_refusals(call, kw, status):
    assert call(batch=_batch(**kw)) == status


@pytest.mark.parametrize("call", [_write, _read, _attend])
def test_missing_descriptors(call):
    assert call(cache=None) == rrq.RRQ_ERR_NULL
    assert call(batch=None) == rrq.RRQ_ERR_NULL
    # nothing to do: nothing else is looked at
    empty = _batch(n_seqs=0, page_table=None, lengths=None, offsets=None, max_pages=0)
    assert call(batch=empty) == rrq.RRQ_OK
    assert call(batch=_batch(n_tokens=0)) == rrq.RRQ_OK


@pytest.mark.parametrize("kw,status", [
    (dict(K=None), rrq.RRQ_ERR_NULL), (dict(V=None), rrq.RRQ_ERR_NULL),
    (dict(K=FAKE + 4), rrq.RRQ_ERR_ALIGN), (dict(V=FAKE + 8), rrq.RRQ_ERR_ALIGN),
    (dict(dtype=2), rrq.RRQ_ERR_DTYPE), (dict(kt=1026), rrq.RRQ_ERR_ALIGN),
    (dict(kh=2), rrq.RRQ_ERR_ALIGN), (dict(vt=1026), rrq.RRQ_ERR_ALIGN),
    (dict(dtype=1, vh=132), rrq.RRQ_ERR_ALIGN), (dict(kt=-128), rrq.RRQ_ERR_SHAPE),
    (dict(vh=1 << 40), rrq.RRQ_ERR_SHAPE),
])
def test_write_refusals(kw, status):
    assert _write(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(K=None), rrq.RRQ_ERR_NULL), (dict(V=None), rrq.RRQ_ERR_NULL),
    (dict(K=FAKE + 4), rrq.RRQ_ERR_ALIGN), (dict(V=FAKE + 8), rrq.RRQ_ERR_ALIGN),
    (dict(dtype=-1), rrq.RRQ_ERR_DTYPE),
])
def test_read_refusals(kw, status):
    assert _read(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(Q=None), rrq.RRQ_ERR_NULL), (dict(out=None), rrq.RRQ_ERR_NULL),
    (dict(Q=FAKE + 4), rrq.RRQ_ERR_ALIGN), (dict(out=FAKE + 8), rrq.RRQ_ERR_ALIGN),
    (dict(dtype=2), rrq.RRQ_ERR_DTYPE), (dict(out_dtype=7), rrq.RRQ_ERR_DTYPE),
    (dict(qt=1026), rrq.RRQ_ERR_ALIGN), (dict(dtype=1, qh=132), rrq.RRQ_ERR_ALIGN),
    (dict(qt=-128), rrq.RRQ_ERR_SHAPE), (dict(heads=3), rrq.RRQ_ERR_SHAPE),
    (dict(heads=0), rrq.RRQ_ERR_SHAPE), (dict(heads=1 << 17), rrq.RRQ_ERR_SHAPE),
    (dict(scale=float("inf")), rrq.RRQ_ERR_SHAPE), (dict(scale=float("nan")), rrq.RRQ_ERR_SHAPE),
    (dict(causal=2), rrq.RRQ_ERR_SHAPE), (dict(window=-1), rrq.RRQ_ERR_SHAPE),
    (dict(heads=1 << 16, batch=_batch(n_tokens=1 << 20)), rrq.RRQ_ERR_SHAPE),
])
def test_attention_refusals(kw, status):
    assert _attend(**kw) == status


def test_attention_workspace():
    long = _batch(n_seqs=1, n_tokens=1, max_pages=1000, table_stride=1000)
    need = rrq.rrq_cache_attention_workspace(_cache(), long, 4)
    assert need > 0 and need % 4 == 0
    assert _attend(batch=long, wb=need - 1) == rrq.RRQ_ERR_WORKSPACE
    assert _attend(batch=long, w=None) == rrq.RRQ_ERR_NULL
    assert _attend(batch=long, w=FAKE + 8) == rrq.RRQ_ERR_ALIGN
    assert rrq.rrq_cache_attention_workspace(_cache(), _batch(n_tokens=0), 4) == 0
    # the buffers are not looked at
    no = dict(k_codes=None, v_codes=None, k_scales=None, v_scales=None)
    assert rrq.rrq_cache_attention_workspace(_cache(**no), long, 4) == need
    for kw, heads in ((dict(head_dim=100), 4), ({}, 3)):
        with pytest.raises(rrq.RRQError) as ei:
            rrq.rrq_cache_attention_workspace(_cache(**kw), long, heads)
        assert ei.value.status == rrq.RRQ_ERR_SHAPE
    assert serving._library().rrq_cache_attention_workspace(
        ctypes.byref(_cache()), ctypes.byref(long), 4, None) == rrq.RRQ_ERR_NULL


def _logprobs(x=FAKE, dtype=0, rows=2, vocab=1000, stride=1000, targets=FAKE, n_top=3,
              logprobs=FAKE, entropy=FAKE, ids=FAKE, top=FAKE, w=FAKE, wb=1 << 40):
    return serving._library().rrq_token_logprobs(x, dtype, rows, vocab, stride, targets, n_top,
                                                 logprobs, entropy, ids, top, w, wb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), rrq.RRQ_ERR_NULL), (dict(logprobs=None), rrq.RRQ_ERR_NULL),
    (dict(ids=None), rrq.RRQ_ERR_NULL), (dict(top=None), rrq.RRQ_ERR_NULL),
    (dict(x=FAKE + 2), rrq.RRQ_ERR_ALIGN), (dict(x=FAKE + 1, dtype=1), rrq.RRQ_ERR_ALIGN),
    (dict(targets=FAKE + 4), rrq.RRQ_ERR_ALIGN), (dict(logprobs=FAKE + 2), rrq.RRQ_ERR_ALIGN),
    (dict(entropy=FAKE + 2), rrq.RRQ_ERR_ALIGN), (dict(ids=FAKE + 4), rrq.RRQ_ERR_ALIGN),
    (dict(top=FAKE + 1), rrq.RRQ_ERR_ALIGN), (dict(dtype=2), rrq.RRQ_ERR_DTYPE),
    (dict(rows=-1), rrq.RRQ_ERR_SHAPE), (dict(rows=(1 << 23) + 1), rrq.RRQ_ERR_SHAPE),
    (dict(vocab=0), rrq.RRQ_ERR_SHAPE), (dict(vocab=(1 << 30) + 1), rrq.RRQ_ERR_SHAPE),
    (dict(stride=999), rrq.RRQ_ERR_SHAPE), (dict(n_top=-1), rrq.RRQ_ERR_SHAPE),
    (dict(n_top=33), rrq.RRQ_ERR_SHAPE), (dict(vocab=2, n_top=3), rrq.RRQ_ERR_SHAPE),
    (dict(vocab=1 << 20, stride=1 << 20, w=None), rrq.RRQ_ERR_NULL),
    (dict(vocab=1 << 20, stride=1 << 20, w=FAKE + 4), rrq.RRQ_ERR_ALIGN),
    (dict(vocab=1 << 20, stride=1 << 20, wb=16), rrq.RRQ_ERR_WORKSPACE),
    (dict(rows=0, x=None), rrq.RRQ_OK),
])
def test_logprobs_refusals(kw, status):
    assert _logprobs(**kw) == status


def test_logprobs_workspace():
    assert rrq.rrq_token_logprobs_workspace(0, 1000, 3) == 0
    assert rrq.rrq_token_logprobs_workspace(1, 1 << 20, 32) > 0
    for args in ((1, 0, 0), (-1, 5, 0), (1, 5, 6), (1, 50, 33)):
        with pytest.raises(rrq.RRQError) as ei:
            rrq.rrq_token_logprobs_workspace(*args)
        assert ei.value.status == rrq.RRQ_ERR_SHAPE
    assert serving._library().rrq_token_logprobs_workspace(1, 5, 1, None) == rrq.RRQ_ERR_NULL


def test_tensor_helpers_refuse_host_tensors():
    import torch
    with pytest.raises(ValueError, match="GPU"):
        rrq.token_logprobs(torch.zeros((2, 5)))
    with pytest.raises(TypeError):
        rrq.token_logprobs([[1.0]])
    with pytest.raises(ValueError, match="GPU"):
        rrq.KVCache(torch.zeros((1, 1, 16, 64), dtype=torch.uint8),
                    torch.zeros((1, 1, 64, 16), dtype=torch.uint8), torch.zeros((1, 1)),
                    torch.zeros((1, 1)))
    with pytest.raises(ValueError, match="code_type"):
        rrq.KVCache(None, None, None, None, "int4")
    with pytest.raises(ValueError, match="GPU"):
        i = torch.zeros((1, 1), dtype=torch.int32)
        rrq.CacheBatch(i, i[0], torch.zeros(2, dtype=torch.int32), 1)
