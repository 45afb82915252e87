"""Inputs shared by the tests of the cache and of attention."""

import numpy as np

from oracle import serving as ora


def bf16(x):
    """float32 values rounded to bfloat16 (ties to even), as float32."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000
    return b.astype(np.uint32).view(np.float32)


class Setup:
    """A cache, its page table and a batch, on the host (the oracle's) and on
    the GPU. Pages are dealt in random order; unused bytes and scales hold
    what a kernel must not use: 0xFF codes (no number in e4m3) and NaN."""

    def __init__(self, rrq, seqs, heads, dim, page, code, seed=0, spare_pages=2):
        import torch
        self.rrq, self.code = rrq, code
        self.rng = np.random.default_rng(seed)
        self.new = [n for n, _ in seqs]
        self.lengths = [length for _, length in seqs]
        self.offsets = [0]
        for n in self.new:
            self.offsets.append(self.offsets[-1] + n)
        pages = [-(-length // page) for length in self.lengths]
        n_pages = sum(pages) + spare_pages
        order = self.rng.permutation(n_pages)
        self.table = np.full((len(seqs), max(max(pages), 1)), -7, np.int32)
        at = 0
        for b, n in enumerate(pages):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.spare = order[at:]
        shape = (n_pages, heads, page, dim)
        self.host = ora.Cache(np.full(shape, 0xFF, np.uint8),
                              np.full((n_pages, heads, dim, page), 0xFF, np.uint8),
                              np.full((n_pages, heads), np.nan, np.float32),
                              np.full((n_pages, heads), np.nan, np.float32), code)
        self.torch = torch

    def fill(self, upto=None):
        """Codes and scales of every sequence's first upto[b] tokens (default:
        all of them), drawn directly."""
        upto = self.lengths if upto is None else upto
        P = self.host.page
        for b, length in enumerate(upto):
            for j in range(-(-length // P)):
                page, n = self.table[b, j], min(P, length - j * P)
                for name in ("k", "v"):
                    for h in range(self.host.k.shape[1]):
                        block = self.host.block(name, page, h)
                        y = self.rng.normal(size=(n, block.shape[1])) * (
                            40 if self.code == "int8" else 120)
                        block[:n] = ora.encode(y, self.code)
                        self.host.scales(name)[page, h] = np.float32(
                            self.rng.uniform(0.5, 1.5) * (0.02 if self.code == "int8" else 0.007))
        return self

    def to_gpu(self, n_tokens=None):
        t = self.torch
        h = self.host
        self.k, self.v = t.from_numpy(h.k.copy()).cuda(), t.from_numpy(h.v.copy()).cuda()
        self.ks, self.vs = t.from_numpy(h.ks.copy()).cuda(), t.from_numpy(h.vs.copy()).cuda()
        self.cache = self.rrq.KVCache(self.k, self.v, self.ks, self.vs, self.code)
        self.batch = self.rrq.CacheBatch(
            t.from_numpy(self.table).cuda(),
            t.tensor(self.lengths, dtype=t.int32, device="cuda"),
            t.tensor(self.offsets, dtype=t.int32, device="cuda"),
            self.offsets[-1] if n_tokens is None else n_tokens)
        return self


def assert_same_blocks(got, want, what):
    """Byte or bit equality, naming the first places that differ."""
    got, want = np.asarray(got), np.asarray(want)
    if got.dtype == np.float32:
        got, want = got.view(np.uint32), want.view(np.uint32)
    bad = np.argwhere(got != want)
    assert bad.size == 0, f"{what}: {len(bad)} differ, first {bad[:4].tolist()}"
