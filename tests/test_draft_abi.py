"""include/rrq_draft.h: exports, workspace sizes, and the refusal of every bad
argument before any device work. No GPU needed."""

import ctypes
import os
import re

import pytest

import paper_2608_04048_amd as rrq
from paper_2608_04048_amd import drafting

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "rrq_draft.h")
FAKE = 0x10000          # aligned, never dereferenced: every case fails validation first


def test_library_exports_every_declared_function():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(rrq_\w+)\s*\(", text)))
    assert "rrq_block_norm" in names
    lib = rrq.load_library()
    for name in names:
        assert hasattr(lib, name) and hasattr(rrq, name), name
    for name, value in re.findall(r"\b(RRQ_[A-Z0-9_]+)\s*=\s*(\d+)", text):
        assert getattr(rrq, name) == int(value), name


def test_structures_match_the_header():
    assert ctypes.sizeof(rrq.RrqNorm) == 3 * 8 + 4 * 4


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
