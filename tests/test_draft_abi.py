"""include/rrq_draft.h: exports, workspace sizes, and the refusal of every bad
argument before any device work. No GPU needed."""

import ctypes
import os
import re

import numpy as np
import pytest

import paper_2608_04048_amd as rrq
from paper_2608_04048_amd import drafting
from test_serve_abi import BATCH_CASES, CACHE_CASES, _batch, _cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "rrq_draft.h")
FAKE = 0x10000          # aligned, never dereferenced: every case fails validation first


def test_library_exports_every_declared_function():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(rrq_\w+)\s*\(", text)))
    lib = rrq.load_library()
    for name in names:
        assert hasattr(lib, name) and hasattr(rrq, name), name
    for name, value in re.findall(r"\b(RRQ_[A-Z0-9_]+)\s*=\s*(\d+)", text):
        assert getattr(rrq, name) == int(value), name


def test_structures_match_the_header():
    assert ctypes.sizeof(rrq.RrqNorm) == 3 * 8 + 4 * 4
    assert ctypes.sizeof(rrq.RrqRotary) == 2 * 8 + 2 * 4


def _ref(x):
    return ctypes.byref(x) if x is not None else None


def _norm_struct(**kw):
    d = dict(weight=FAKE, bias=FAKE, post_weight=FAKE, kind=1, post=0, eps=1e-6, scale=1.0)
    d.update(kw)
    return rrq.RrqNorm(**d)


def _norm(norm=_norm_struct(), r=FAKE, rt=0, rs=64, y=FAKE, yt=0, ys=64, gate=FAKE, gs=64, rows=2,
          hidden=64, out=FAKE, ot=1, h=FAKE):
    return drafting._library().rrq_block_norm(_ref(norm), r, rt, rs, y, yt, ys, gate, gs, rows,
                                              hidden, out, ot, h, None)


@pytest.mark.parametrize("kw,status", [
    (dict(norm=None), rrq.RRQ_ERR_NULL), (dict(r=None), rrq.RRQ_ERR_NULL),
    (dict(out=None), rrq.RRQ_ERR_NULL), (dict(h=None), rrq.RRQ_ERR_NULL),
    (dict(norm=_norm_struct(kind=0)), rrq.RRQ_ERR_FORMAT),
    (dict(norm=_norm_struct(kind=3)), rrq.RRQ_ERR_FORMAT),
    (dict(norm=_norm_struct(post=-1)), rrq.RRQ_ERR_FORMAT),
    (dict(norm=_norm_struct(post=3)), rrq.RRQ_ERR_FORMAT),
    (dict(norm=_norm_struct(eps=-1e-6)), rrq.RRQ_ERR_SHAPE),
    (dict(norm=_norm_struct(eps=float("nan"))), rrq.RRQ_ERR_SHAPE),
    (dict(norm=_norm_struct(scale=float("inf"))), rrq.RRQ_ERR_SHAPE),
    (dict(norm=_norm_struct(weight=FAKE + 2)), rrq.RRQ_ERR_ALIGN),
    (dict(norm=_norm_struct(bias=FAKE + 1)), rrq.RRQ_ERR_ALIGN),
    (dict(norm=_norm_struct(post_weight=FAKE + 2)), rrq.RRQ_ERR_ALIGN),
    (dict(y=None), rrq.RRQ_ERR_SHAPE), (dict(y=None, gate=None, norm=_norm_struct(post=1)),
                                        rrq.RRQ_ERR_SHAPE),
    (dict(rows=-1), rrq.RRQ_ERR_SHAPE), (dict(rows=(1 << 26) + 1), rrq.RRQ_ERR_SHAPE),
    (dict(hidden=0), rrq.RRQ_ERR_SHAPE), (dict(hidden=65537), rrq.RRQ_ERR_SHAPE),
    (dict(rs=63), rrq.RRQ_ERR_SHAPE), (dict(ys=0), rrq.RRQ_ERR_SHAPE),
    (dict(gs=63), rrq.RRQ_ERR_SHAPE), (dict(rs=1 << 40), rrq.RRQ_ERR_SHAPE),
    (dict(rt=2), rrq.RRQ_ERR_DTYPE), (dict(yt=-1), rrq.RRQ_ERR_DTYPE),
    (dict(ot=2), rrq.RRQ_ERR_DTYPE), (dict(r=FAKE + 2), rrq.RRQ_ERR_ALIGN),
    (dict(rt=1, r=FAKE + 1), rrq.RRQ_ERR_ALIGN), (dict(h=FAKE + 2), rrq.RRQ_ERR_ALIGN),
    (dict(y=FAKE + 2), rrq.RRQ_ERR_ALIGN), (dict(gate=FAKE + 1, yt=1), rrq.RRQ_ERR_ALIGN),
    (dict(out=FAKE + 1), rrq.RRQ_ERR_ALIGN), (dict(rows=0, r=None, out=None), rrq.RRQ_OK),
])
def test_norm_refusals(kw, status):
    assert _norm(**kw) == status


def _rotary(**kw):
    d = dict(frequencies=FAKE, amplitude=1.0, rot_dim=128, layout=0)
    d.update(kw)
    return rrq.RrqRotary(**d)


def _append(cache=_cache(), batch=_batch(), rotary=_rotary(), positions=FAKE, Q=FAKE, K=FAKE,
            V=FAKE, dtype=0, qt=2048, qh=128, kt=2048, kh=128, vt=2048, vh=128, heads=4, out=FAKE):
    return drafting._library().rrq_cache_append(_ref(cache), _ref(batch), _ref(rotary), positions,
                                                Q, K, V, dtype, qt, qh, kt, kh, vt, vh, heads,
                                                out, None)


@pytest.mark.parametrize("kw,status", CACHE_CASES)
def test_cache_descriptor_refusals(kw, status):
    assert _append(cache=_cache(**kw)) == status


@pytest.mark.parametrize("kw,status", BATCH_CASES)
def test_batch_descriptor_refusals(kw, status):
    assert _append(batch=_batch(**kw)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(cache=None), rrq.RRQ_ERR_NULL), (dict(batch=None), rrq.RRQ_ERR_NULL),
    (dict(rotary=None), rrq.RRQ_ERR_NULL),
    (dict(rotary=_rotary(frequencies=None)), rrq.RRQ_ERR_NULL),
    (dict(rotary=_rotary(frequencies=FAKE + 4)), rrq.RRQ_ERR_ALIGN),
    (dict(rotary=_rotary(rot_dim=0)), rrq.RRQ_ERR_SHAPE),
    (dict(rotary=_rotary(rot_dim=-8)), rrq.RRQ_ERR_SHAPE),
    (dict(rotary=_rotary(rot_dim=12)), rrq.RRQ_ERR_SHAPE),
    (dict(rotary=_rotary(rot_dim=136)), rrq.RRQ_ERR_SHAPE),
    (dict(rotary=_rotary(layout=2)), rrq.RRQ_ERR_FORMAT),
    (dict(rotary=_rotary(layout=-1)), rrq.RRQ_ERR_FORMAT),
    (dict(rotary=_rotary(amplitude=float("inf"))), rrq.RRQ_ERR_SHAPE),
    (dict(positions=FAKE + 2), rrq.RRQ_ERR_ALIGN), (dict(dtype=2), rrq.RRQ_ERR_DTYPE),
    (dict(Q=None), rrq.RRQ_ERR_NULL), (dict(K=None), rrq.RRQ_ERR_NULL),
    (dict(V=None), rrq.RRQ_ERR_NULL), (dict(out=None), rrq.RRQ_ERR_NULL),
    (dict(Q=FAKE + 4), rrq.RRQ_ERR_ALIGN), (dict(K=FAKE + 8), rrq.RRQ_ERR_ALIGN),
    (dict(V=FAKE + 2), rrq.RRQ_ERR_ALIGN), (dict(out=FAKE + 8), rrq.RRQ_ERR_ALIGN),
    (dict(qt=2050), rrq.RRQ_ERR_ALIGN), (dict(dtype=1, kh=132), rrq.RRQ_ERR_ALIGN),
    (dict(vt=-128), rrq.RRQ_ERR_SHAPE), (dict(heads=0), rrq.RRQ_ERR_SHAPE),
    (dict(heads=(1 << 16) + 1), rrq.RRQ_ERR_SHAPE),
    (dict(batch=_batch(n_tokens=0), Q=None, K=None, V=None, out=None), rrq.RRQ_OK),
    (dict(batch=_batch(n_seqs=0, page_table=None, max_pages=0), Q=None), rrq.RRQ_OK),
])
def test_append_refusals(kw, status):
    assert _append(**kw) == status


def test_rotary_frequencies():
    """Unstretched powers, slow pairs slowed, fast ones kept."""
    import torch
    f = rrq.rotary_frequencies(128, device="cpu")
    assert f.dtype == torch.float64 and np.allclose(f.numpy(), 10000.0 ** (-np.arange(64) / 64), rtol=1e-14)
    g = rrq.rotary_frequencies(128, stretch=4.0, device="cpu")
    turns = 32768 * f / (2 * np.pi)
    assert torch.equal(g[turns >= 32], f[turns >= 32])
    assert torch.equal(g[turns <= 1], f[turns <= 1] / 4)
    between = (turns > 1) & (turns < 32)
    assert between.any() and (g[between] < f[between]).all()
    assert (g[between] > f[between] / 4).all()


def _tree(cache=_cache(), batch=_batch(), Q=FAKE, dtype=0, qt=1024, qh=128, heads=4, scale=0.1,
          seen=FAKE, words=1, positions=FAKE, window=0, out=FAKE, out_dtype=1, w=FAKE, wb=1 << 40):
    return drafting._library().rrq_tree_attention(_ref(cache), _ref(batch), Q, dtype, qt, qh,
                                                  heads, scale, seen, words, positions, window,
                                                  out, out_dtype, w, wb, None)


@pytest.mark.parametrize("kw,status", CACHE_CASES)
def test_tree_cache_refusals(kw, status):
    assert _tree(cache=_cache(**kw)) == status


@pytest.mark.parametrize("kw,status", BATCH_CASES)
def test_tree_batch_refusals(kw, status):
    assert _tree(batch=_batch(**kw)) == status


LONG = _batch(n_seqs=1, n_tokens=1, max_pages=1000, table_stride=1000)


@pytest.mark.parametrize("kw,status", [
    (dict(cache=None), rrq.RRQ_ERR_NULL), (dict(batch=None), rrq.RRQ_ERR_NULL),
    (dict(Q=None), rrq.RRQ_ERR_NULL), (dict(out=None), rrq.RRQ_ERR_NULL),
    (dict(seen=None), rrq.RRQ_ERR_NULL), (dict(seen=FAKE + 4), rrq.RRQ_ERR_ALIGN),
    (dict(words=0), rrq.RRQ_ERR_SHAPE), (dict(words=(1 << 20) + 1), rrq.RRQ_ERR_SHAPE),
    (dict(positions=FAKE + 2), rrq.RRQ_ERR_ALIGN),
    (dict(Q=FAKE + 4), rrq.RRQ_ERR_ALIGN), (dict(out=FAKE + 8), rrq.RRQ_ERR_ALIGN),
    (dict(dtype=2), rrq.RRQ_ERR_DTYPE), (dict(out_dtype=7), rrq.RRQ_ERR_DTYPE),
    (dict(qt=1026), rrq.RRQ_ERR_ALIGN), (dict(qt=-128), rrq.RRQ_ERR_SHAPE),
    (dict(heads=3), rrq.RRQ_ERR_SHAPE), (dict(heads=0), rrq.RRQ_ERR_SHAPE),
    (dict(scale=float("inf")), rrq.RRQ_ERR_SHAPE), (dict(window=-1), rrq.RRQ_ERR_SHAPE),
    (dict(batch=LONG, w=None), rrq.RRQ_ERR_NULL), (dict(batch=LONG, wb=16), rrq.RRQ_ERR_WORKSPACE),
    (dict(batch=LONG, w=FAKE + 8), rrq.RRQ_ERR_ALIGN),
    (dict(batch=_batch(n_tokens=0), Q=None, seen=None, out=None), rrq.RRQ_OK),
])
def test_tree_refusals(kw, status):
    assert _tree(**kw) == status


def _verify(x=FAKE, dtype=0, rows=6, vocab=1000, stride=1000, tokens=FAKE, offsets=FAKE, seqs=2,
            uniforms=FAKE, parents=None, draft=FAKE, ds=3000, dr=1000, t=1.0, dt=1.0, accept=3,
            counts=FAKE, following=FAKE, paths=FAKE, w=FAKE, wb=1 << 40):
    return drafting._library().rrq_verify_drafts(x, dtype, rows, vocab, stride, tokens, offsets,
                                                 seqs, uniforms, parents, draft, ds, dr, t, dt,
                                                 accept, counts, following, paths, w, wb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), rrq.RRQ_ERR_NULL), (dict(tokens=None), rrq.RRQ_ERR_NULL),
    (dict(offsets=None), rrq.RRQ_ERR_NULL), (dict(uniforms=None), rrq.RRQ_ERR_NULL),
    (dict(counts=None), rrq.RRQ_ERR_NULL), (dict(following=None), rrq.RRQ_ERR_NULL),
    (dict(paths=None), rrq.RRQ_ERR_NULL), (dict(w=None), rrq.RRQ_ERR_NULL),
    (dict(x=FAKE + 2), rrq.RRQ_ERR_ALIGN), (dict(x=FAKE + 1, dtype=1), rrq.RRQ_ERR_ALIGN),
    (dict(draft=FAKE + 2), rrq.RRQ_ERR_ALIGN), (dict(tokens=FAKE + 4), rrq.RRQ_ERR_ALIGN),
    (dict(offsets=FAKE + 2), rrq.RRQ_ERR_ALIGN), (dict(uniforms=FAKE + 1), rrq.RRQ_ERR_ALIGN),
    (dict(parents=FAKE + 2, draft=None), rrq.RRQ_ERR_ALIGN),
    (dict(counts=FAKE + 2), rrq.RRQ_ERR_ALIGN), (dict(following=FAKE + 4), rrq.RRQ_ERR_ALIGN),
    (dict(paths=FAKE + 2), rrq.RRQ_ERR_ALIGN), (dict(w=FAKE + 8), rrq.RRQ_ERR_ALIGN),
    (dict(dtype=2), rrq.RRQ_ERR_DTYPE), (dict(rows=-1), rrq.RRQ_ERR_SHAPE),
    (dict(rows=(1 << 23) + 1, vocab=10), rrq.RRQ_ERR_SHAPE), (dict(vocab=0), rrq.RRQ_ERR_SHAPE),
    (dict(vocab=(1 << 30) + 1), rrq.RRQ_ERR_SHAPE), (dict(stride=999), rrq.RRQ_ERR_SHAPE),
    (dict(rows=1 << 22, vocab=1 << 17, stride=1 << 17), rrq.RRQ_ERR_SHAPE),
    (dict(seqs=-1), rrq.RRQ_ERR_SHAPE), (dict(seqs=(1 << 20) + 1), rrq.RRQ_ERR_SHAPE),
    (dict(accept=-1), rrq.RRQ_ERR_SHAPE), (dict(accept=(1 << 20) + 1), rrq.RRQ_ERR_SHAPE),
    (dict(seqs=1 << 20, accept=1 << 20), rrq.RRQ_ERR_SHAPE),
    (dict(parents=FAKE), rrq.RRQ_ERR_SHAPE), (dict(t=-1.0), rrq.RRQ_ERR_SHAPE),
    (dict(t=float("nan")), rrq.RRQ_ERR_SHAPE), (dict(t=float("inf")), rrq.RRQ_ERR_SHAPE),
    (dict(t=1e-30), rrq.RRQ_ERR_SHAPE), (dict(dt=0.0), rrq.RRQ_ERR_SHAPE),
    (dict(ds=-1), rrq.RRQ_ERR_SHAPE), (dict(dr=-1), rrq.RRQ_ERR_SHAPE),
    (dict(wb=16), rrq.RRQ_ERR_WORKSPACE), (dict(seqs=0, x=None, offsets=None), rrq.RRQ_OK),
])
def test_verify_refusals(kw, status):
    assert _verify(**kw) == status


def test_verify_workspace():
    need = rrq.rrq_verify_drafts_workspace(6, 1000, 2, 6)
    assert need > rrq.rrq_verify_drafts_workspace(6, 1000, 2, 0) > 0
    assert _verify(wb=need - 1) == rrq.RRQ_ERR_WORKSPACE
    assert rrq.rrq_verify_drafts_workspace(6, 1000, 0, 0) == 0
    for args in ((-1, 5, 1, 0), (1, 0, 1, 0), (1, 5, -1, 0), (1, 5, 1, -1), (1 << 22, 1 << 17, 1, 0)):
        with pytest.raises(rrq.RRQError) as ei:
            rrq.rrq_verify_drafts_workspace(*args)
        assert ei.value.status == rrq.RRQ_ERR_SHAPE
    assert drafting._library().rrq_verify_drafts_workspace(1, 5, 1, 0, None) == rrq.RRQ_ERR_NULL
