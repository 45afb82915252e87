"""Plain CPU definitions of the calls of include/rrq_serve.h: the 8-bit cache,
attention over it and token scoring. Written from the header's formulas in
numpy, one sequence, page and head at a time; binary32 where the definition
rounds, 64 bits elsewhere.
"""

import numpy as np

C_MAX = {"int8": 127.0, "fp8": 448.0}
F32 = np.float32


def fp8_values():
    """The value of each e4m3 byte: sign, 4 exponent bits (bias 7), 3 mantissa
    bits; the all-ones pattern is no number."""
    out = np.zeros(256)
    for b in range(256):
        sign, e, m = b >> 7, (b >> 3) & 15, b & 7
        if e == 15 and m == 7:
            v = np.nan
        elif e == 0:
            v = m * 2.0 ** -9
        else:
            v = (1 + m / 8) * 2.0 ** (e - 7)
        out[b] = -v if sign else v
    return out


_FP8 = fp8_values()
_FP8_POSITIVE = _FP8[:127]           # ascending, 0 .. 448


def decode(codes, code):
    """Values of uint8 codes, in 64 bits."""
    codes = np.asarray(codes, np.uint8)
    return codes.view(np.int8).astype(np.float64) if code == "int8" else _FP8[codes]


def encode(y, code):
    """uint8 codes nearest to y, ties to even."""
    y = np.asarray(y, np.float64)
    if code == "int8":
        return np.clip(np.rint(y), -127, 127).astype(np.int8).view(np.uint8)
    a = np.minimum(np.abs(y), 448.0)
    hi = np.clip(np.searchsorted(_FP8_POSITIVE, a), 1, 126)     # first value >= a
    lo = hi - 1
    to_hi, to_lo = _FP8_POSITIVE[hi] - a, a - _FP8_POSITIVE[lo]
    # neighbouring codes are neighbouring bytes: even mantissa, even byte
    pick = np.where((to_hi < to_lo) | ((to_hi == to_lo) & (hi % 2 == 0)), hi, lo)
    return (pick + 128 * np.signbit(y)).astype(np.uint8)


def _f32(x):
    return np.asarray(x, np.float64).astype(F32).astype(np.float64)


class Cache:
    """A cache in host memory: k [pages, heads, page, dim], v [pages, heads,
    dim, page] uint8, ks and vs float32 [pages, heads]."""

    def __init__(self, k, v, ks, vs, code):
        self.k, self.v, self.ks, self.vs, self.code = k, v, ks, vs, code
        self.page = k.shape[2]

    def block(self, name, page, head):
        """The block's codes as [tokens, dim] (a view)."""
        return self.k[page, head] if name == "k" else self.v[page, head].T

    def scales(self, name):
        return self.ks if name == "k" else self.vs


def write(cache, table, lengths, offsets, K, V):
    """Quantise rows K, V [tokens, heads, dim] in place."""
    P, code = cache.page, cache.code
    inv_max = _f32(F32(1) / F32(C_MAX[code]))
    for b, length in enumerate(lengths):
        n = offsets[b + 1] - offsets[b]
        start = length - n
        for j in range(max(start, 0) // P, -(-length // P)) if n > 0 and length > 0 else ():
            lo, hi = max(0, max(start, 0) - j * P), min(P, length - j * P)
            row = offsets[b] + j * P + lo - start
            for name, X in (("k", K), ("v", V)):
                for h in range(X.shape[1]):
                    x = X[row:row + hi - lo, h].astype(np.float64)
                    scales = cache.scales(name)
                    page = table[b][j]
                    old = float(scales[page, h]) if lo else 0.0
                    s = max(old, float(_f32(np.abs(x).max() * inv_max)))
                    if s < 2.0 ** -126:
                        s = 0.0
                    inv = float(_f32(1.0 / s)) if s > 0 else 0.0
                    block = cache.block(name, page, h)
                    if lo and s > old > 0:
                        kept = decode(block[:lo], code)
                        block[:lo] = encode(_f32(kept * float(_f32(old * inv))), code)
                    block[lo:hi] = encode(_f32(x * inv), code)
                    scales[page, h] = s


def dense(cache, table_row, name, head, length):
    """Positions 0 .. length - 1 of a sequence's head, [length, dim], 64 bits."""
    P = cache.page
    dim = cache.k.shape[3]
    out = np.zeros((length, dim))
    for j in range(-(-length // P)):
        page = table_row[j]
        n = min(P, length - j * P)
        codes = cache.block(name, page, head)[:n]
        out[j * P:j * P + n] = (decode(codes, cache.code) *
                                float(cache.scales(name)[page, head]))
    return out


def attention(cache, table, lengths, offsets, Q, scale, causal=True, window=0):
    """(out, weight) [tokens, heads, dim] in 64 bits: the attention, and the
    mean of |v| under its weights. Also returns the largest sum of |q||k| of a
    row, [tokens, heads] (for error bounds)."""
    T, Hq, D = Q.shape
    ratio = Hq // cache.k.shape[1]
    out, mean_abs = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    reach = np.zeros((T, Hq))
    for b, length in enumerate(lengths):
        n = offsets[b + 1] - offsets[b]
        if n <= 0:
            continue
        for h in range(Hq):
            k = dense(cache, table[b], "k", h // ratio, length)
            v = dense(cache, table[b], "v", h // ratio, length)
            for i in range(n):
                pos = length - n + i
                hi = min(length, pos + 1) if causal else length
                lo = max(0, pos + 1 - window) if window else 0
                row = offsets[b] + i
                if hi <= lo:
                    continue
                q = Q[row, h].astype(np.float64)
                s = scale * (k[lo:hi] @ q)
                p = np.exp(s - s.max())
                p /= p.sum()
                out[row, h] = p @ v[lo:hi]
                mean_abs[row, h] = p @ np.abs(v[lo:hi])
                reach[row, h] = (np.abs(k[lo:hi]) @ np.abs(q)).max()
    return out, mean_abs, reach


def token_logprobs(x, targets, n_top):
    """(logprobs, entropy, ids, top) of logits x [rows, vocab], 64 bits; rows
    without NaN or +inf."""
    x = np.asarray(x, np.float64)
    rows, vocab = x.shape
    m = x.max(1, keepdims=True)
    safe = np.where(np.isneginf(m), 0.0, m)
    e = np.exp(x - safe)
    total = e.sum(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        # differences first: next to 1e38 a sum of 64 bits would lose the log
        lp = (x - safe) - np.where(total > 0, np.log(total), 0.0)
        p = np.where(total > 0, e / total, 0.0)
        entropy = -np.where(p > 0, p * lp, 0.0).sum(1)
    inside = (targets >= 0) & (targets < vocab)
    got = lp[np.arange(rows), np.where(inside, targets, 0)]
    logprobs = np.where(inside, got, 0.0)
    ids = np.argsort(-x, axis=1, kind="stable")[:, :n_top]
    return logprobs, entropy, ids, np.take_along_axis(lp, ids, 1)
