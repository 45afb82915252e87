"""Verification where a segment of a row holds several blocks of 8192 logits: many rows, or
long vocabularies; and drawing from more than 512 blocks of 4096."""

import numpy as np
import pytest

from test_gpu_verify import check, make, upload

pytestmark = pytest.mark.gpu

BLOCK = 8192
# (sequences of two rows, vocabulary): with the draft's rows too, a segment has two blocks
SHAPES = [(300, 70001), (2100, 9001)]

# Of a row's sum, relative to the weight that it is off by: a logit passes its thread's
# reference by less than 6 powers of two (else the reference moves up), so that the
# difference to it and the product with log2(e) / T, each off by half a step, put
# 2 x 6 ln 2 = 8.4 units of 2^-24 on its weight; the exponential instruction is good to a
# last place (2 units), and 7 additions in binary32 to a unit each: 17.4.
SUM = 18 * 2.0 ** -24


def _rounded(x, dtype):
    x = x.astype(np.float32)
    if dtype == "bf16":
        b = x.view(np.uint32).astype(np.uint64)
        x = ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return x


def _logits(rng, rows, vocab, dtype):
    """Rows of normal logits: as they are, with a logit of a segment's second block far
    above the others (20, or 45: past 2^60 of the weights so far), with a first block of
    -inf, and with peaks in both blocks."""
    x = rng.standard_normal((rows, vocab), dtype=np.float32) * np.float32(2.5)
    first = 2 * BLOCK * rng.integers(0, max(1, vocab // (2 * BLOCK)), rows)
    for r in range(rows):
        at = first[r] + BLOCK + int(rng.integers(0, min(BLOCK, vocab - BLOCK - first[r])))
        early = first[r] + int(rng.integers(0, BLOCK))
        kind = r // 2 % 6
        if kind == 1:
            x[r, at] = 20
        elif kind == 2:
            x[r, at] = 45 + x[r, at]
        elif kind == 3:
            x[r, first[r]:first[r] + BLOCK] = -np.inf
        elif kind == 4:
            x[r, at], x[r, early] = 41.3, 41.1
        elif kind == 5:
            x[r, :BLOCK] = -np.inf
            x[r, first[r] + BLOCK:] -= 30
            x[r, at] = 3
    return _rounded(x, dtype)


def _case(seqs, vocab, dtype, draft, seed):
    rng = np.random.default_rng(seed)
    rows = 2 * seqs
    logits = _logits(rng, rows, vocab, dtype)
    q = _logits(rng, seqs, vocab, dtype)[:, None] if draft else None
    tokens = rng.integers(0, vocab, rows)
    tokens[1::2] = np.where(np.arange(seqs) % 3 > 0, logits[::2].argmax(1), tokens[1::2])
    return dict(logits=logits, tokens=tokens, offsets=np.arange(0, rows + 1, 2), max_accept=1,
                uniforms=rng.random(rows).astype(np.float32), draft=q, parents=None), dtype, 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["chain", "draft"])
@pytest.mark.parametrize("seqs,vocab", SHAPES)
def test_several_blocks_a_segment(gpu, seqs, vocab, kind, dtype):
    # (two sums behind a decision)
    counts, _, _ = check(gpu, _case(seqs, vocab, dtype, kind == "draft", seed=51), near=2 * SUM)
    assert 0.1 < counts.float().mean() < 0.95


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,vocab", SHAPES)
def test_greedy_over_several_blocks(gpu, seqs, vocab, dtype):
    a, dtype, pad = _case(seqs, vocab, dtype, False, seed=52)
    # equal largest logits in different blocks, both orders of finding them
    for b in range(0, seqs, 4):
        a["logits"][2 * b, [8999, 17, 8193]] = 60.0
        a["logits"][2 * b + 2, [9000, 8195]] = 60.0
    a["tokens"][1::8] = 17
    a["tokens"][3::8] = 8195
    counts, following, _ = check(gpu, (a, dtype, pad), 0.0)
    assert (counts[0::4] == 1).all() and (counts[1::4] == 1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sums_of_far_logits(gpu, dtype):
    """A token of a segment's first block, and a likelier one of its second, 40 above what
    the threads there saw first: accepted for the last number of binary32 that the sum's
    bound puts below the border, rejected for the first past it."""
    import torch
    seqs, vocab = 300, 70001
    rng = np.random.default_rng(53)
    a, _, pad = _case(seqs, vocab, dtype, False, seed=54)
    a["logits"][:] = _rounded(rng.standard_normal(a["logits"].shape, dtype=np.float32) * 2, dtype)
    low, high = np.zeros(seqs, np.float32), np.zeros(seqs, np.float32)
    for b in range(seqs):
        first = 2 * BLOCK * int(rng.integers(0, 4))
        early, late = first + rng.integers(0, BLOCK), first + BLOCK + rng.integers(0, BLOCK)
        tops = 39 + rng.random()
        x = a["logits"][2 * b]
        x[early], x[late] = _rounded(np.array([tops, tops + 0.9 + rng.random()]), dtype)
        a["tokens"][2 * b + 1] = early
        p = np.exp(x.astype(np.float64) - float(x[late]))
        p = p[early] / p.sum()
        lo, hi = np.float32(p * (1 - SUM)), np.float32(p * (1 + SUM))
        low[b] = lo if lo <= p * (1 - SUM) else np.nextafter(lo, np.float32(0))
        high[b] = hi if hi >= p * (1 + SUM) else np.nextafter(hi, np.float32(1))
    args = upload((a, dtype, pad))
    for u, accepted in ((low, 1), (high, 0)):
        args["uniforms"][1::2] = torch.from_numpy(u).cuda()
        counts, _, _ = gpu.verify_drafts(**args)
        wrong = (counts != accepted).nonzero().flatten().tolist()
        assert not wrong, f"{len(wrong)} of {seqs} rows, first {wrong[:5]}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["chain", "draft"])
def test_vocabularies_past_512_blocks(gpu, kind, dtype):
    """More blocks than the drawing workgroup has threads: tokens on both sides of the
    512th, the last ones, and one that a draft leaves nothing else but."""
    vocab = (1 << 21) + 4097
    a, _, pad = make([2] * 4, 8, dtype, draft=kind == "draft", seed=55)
    rng = np.random.default_rng(56)
    x = rng.standard_normal((8, vocab), dtype=np.float32)
    x[0, :1 << 21] -= 20
    x[2, 1 << 21:] = -np.inf
    x[4, vocab - 1] = 30
    a["logits"] = _rounded(x, dtype)
    if kind == "draft":
        q = rng.standard_normal((4, 1, vocab), dtype=np.float32)
        q[2, 0, vocab - 1] = 5
        a["draft"] = _rounded(q, dtype)
    a["tokens"][1::2] = [5, 6, 7, 8]
    a["uniforms"][::2] = [0.3, 0.9, 0.5, 0.2]
    a["uniforms"][1::2] = 0.9999
    _, following, _ = check(gpu, (a, dtype, pad))
    assert following[0].item() >= 1 << 21 and following[1].item() < 1 << 21
    assert following[2].item() == vocab - 1


def test_greedy_past_512_blocks(gpu):
    vocab = (1 << 21) + 4097
    a, dtype, pad = make([2] * 3, 8, seed=57)
    a["logits"] = np.random.default_rng(58).standard_normal((6, vocab), dtype=np.float32)
    a["logits"][0, [vocab - 1, 1 << 21, 3]] = [9.0, 9.5, 9.25]
    a["logits"][2, [vocab - 1, 100]] = 9.0
    a["logits"][4, vocab - 1] = 9.0
    a["tokens"][1::2] = [1 << 21, vocab - 1, vocab - 1]
    counts, following, _ = check(gpu, (a, dtype, pad), 0.0)
    assert counts.tolist() == [1, 0, 1] and following[1].item() == 100
