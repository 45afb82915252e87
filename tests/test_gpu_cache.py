"""The 8-bit cache on the GPU against the oracle's definition: codes and
scales bit for bit after a write (and nothing outside the written slots
touched), values of a read bit for bit."""

import numpy as np
import pytest

from oracle import serving as ora
from serving_helpers import Setup, assert_same_blocks, bf16

pytestmark = pytest.mark.gpu

CODES = ["int8", "fp8"]
# (new tokens, length with them) of each sequence
RAGGED = [(1, 1), (5, 21), (0, 9), (40, 40), (3, 130), (17, 33)]


def _rows(rng, n, heads, dim):
    x = rng.normal(size=(n, heads, dim)).astype(np.float32)
    return x * np.float32(2.0) ** rng.integers(-3, 4, size=(n, heads, 1)).astype(np.float32)


def _upload(torch, x, dtype):
    """x on the GPU as columns of a wider row (strided) in dtype."""
    n, heads, dim = x.shape
    wide = torch.full((max(n, 1), heads + 3, dim), float("nan"), device="cuda", dtype=dtype)
    wide[:n, 2:2 + heads] = torch.from_numpy(x).cuda().to(dtype)
    return wide[:n, 2:2 + heads]


def _check(s, K, V, dtype):
    torch = s.torch
    before_k, before_v = s.host.k.copy(), s.host.v.copy()
    s.to_gpu()
    s.rrq.cache_write(s.cache, s.batch, _upload(torch, K, dtype), _upload(torch, V, dtype))
    torch.cuda.synchronize()
    ora.write(s.host, s.table, s.lengths, s.offsets, K, V)
    assert_same_blocks(s.ks.cpu().numpy(), s.host.ks, "key scales")
    assert_same_blocks(s.vs.cpu().numpy(), s.host.vs, "value scales")
    assert_same_blocks(s.k.cpu().numpy(), s.host.k, "key codes")
    assert_same_blocks(s.v.cpu().numpy(), s.host.v, "value codes")
    return before_k, before_v


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,dim,page", [(1, 64, 16), (3, 128, 32), (2, 256, 64), (2, 64, 128),
                                            (1, 256, 16), (2, 128, 128)])
def test_write_equals_the_definition(gpu, code, dtype, heads, dim, page):
    import torch
    s = Setup(gpu, RAGGED, heads, dim, page, code, seed=dim + page).fill(
        [length - n for n, length in RAGGED])
    n = s.offsets[-1]
    K, V = _rows(s.rng, n, heads, dim), _rows(s.rng, n, heads, dim)
    if dtype == "bf16":
        K, V = bf16(K), bf16(V)
    _check(s, K, V, torch.float32 if dtype == "f32" else torch.bfloat16)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_scale_that_grows_past_the_range_of_its_ratio(gpu, code, dtype):
    """The stored scale over the new one is below every binary32: the kept
    codes become zeros."""
    import torch
    seqs = [(1, 12), (4, 16), (2, 31)]
    s = Setup(gpu, seqs, 2, 64, 16, code, seed=4).fill([length - n for n, length in seqs])
    s.host.ks *= np.float32(1e-30)
    s.host.vs *= np.float32(1e-30)
    K = bf16(_rows(s.rng, s.offsets[-1], 2, 64) * np.float32(1e33))
    V = bf16(_rows(s.rng, s.offsets[-1], 2, 64) * np.float32(1e34))
    _check(s, K, V, torch.float32 if dtype == "f32" else torch.bfloat16)
    page = s.host.block("k", s.table[0, 0], 0)
    assert (page[:11] & 0x7F == 0).all()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("gain", [1e-3, 1.0, 37.0, 1e4])
def test_a_growing_scale_moves_the_codes_already_there(gpu, code, gain):
    import torch
    seqs = [(1, 12), (4, 16), (1, 17), (2, 31)]
    s = Setup(gpu, seqs, 2, 128, 16, code, seed=3).fill([length - n for n, length in seqs])
    K = _rows(s.rng, s.offsets[-1], 2, 128) * np.float32(gain)
    V = _rows(s.rng, s.offsets[-1], 2, 128) * np.float32(gain)
    _check(s, K, V, torch.float32)


@pytest.mark.parametrize("code", CODES)
def test_zero_tiny_and_huge_values(gpu, code):
    import torch
    seqs = [(2, 2), (2, 7), (3, 3), (2, 9), (1, 6)]
    s = Setup(gpu, seqs, 1, 64, 16, code, seed=4).fill([0, 5, 0, 7, 5])
    K = np.zeros((s.offsets[-1], 1, 64), np.float32)
    K[2, 0, 5] = -0.0
    K[4, 0, 0] = 1e-41                   # a subnormal alone: the block is all zero
    K[5, 0, 1] = -3e-38                  # 3e-38 / 127 is subnormal
    K[6, 0, 2] = 1e-36
    K[7, 0, 3] = 3e38
    K[8, 0, 3] = -2.5e38
    K[9, 0, :] = np.linspace(-3, 3, 64)
    V = K[:, :, ::-1].copy()
    _check(s, K, V, torch.float32)


@pytest.mark.parametrize("code", CODES)
def test_a_write_repeated_leaves_the_same_codes(gpu, code):
    import torch
    seqs = [(3, 20), (16, 40), (1, 1)]
    s = Setup(gpu, seqs, 2, 128, 16, code, seed=5).fill([17, 24, 0])
    K = torch.from_numpy(_rows(s.rng, 20, 2, 128)).cuda()
    V = torch.from_numpy(_rows(s.rng, 20, 2, 128)).cuda()
    s.to_gpu()
    s.rrq.cache_write(s.cache, s.batch, K, V)
    first = [t.clone() for t in (s.k, s.v)], [t.cpu().numpy() for t in (s.ks, s.vs)]
    s.rrq.cache_write(s.cache, s.batch, K, V)
    assert torch.equal(s.k, first[0][0]) and torch.equal(s.v, first[0][1])
    assert_same_blocks(s.ks.cpu().numpy(), first[1][0], "key scales")
    assert_same_blocks(s.vs.cpu().numpy(), first[1][1], "value scales")


@pytest.mark.parametrize("code", CODES)
def test_token_by_token(gpu, code):
    """A page filled one token a call, as decoding does."""
    import torch
    s = Setup(gpu, [(1, 20), (1, 35)], 2, 64, 16, code, seed=6)
    rows = [_rows(s.rng, 20, 2, 64), _rows(s.rng, 35, 2, 64)]
    s.to_gpu()
    for step in range(1, 36):
        now = [b for b in range(2) if step <= s.lengths[b]]
        K = np.stack([rows[b][step - 1] for b in now])
        batch = s.rrq.CacheBatch(
            torch.from_numpy(s.table[now]).cuda(),
            torch.full((len(now),), step, dtype=torch.int32, device="cuda"),
            torch.arange(len(now) + 1, dtype=torch.int32, device="cuda"), len(now))
        x = torch.from_numpy(K).cuda()
        s.rrq.cache_write(s.cache, batch, x, -x)
        ora.write(s.host, s.table[now], [step] * len(now), list(range(len(now) + 1)), K, -K)
    assert_same_blocks(s.ks.cpu().numpy(), s.host.ks, "key scales")
    assert_same_blocks(s.k.cpu().numpy(), s.host.k, "key codes")
    assert_same_blocks(s.v.cpu().numpy(), s.host.v, "value codes")


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,dim,page", [(1, 64, 16), (3, 128, 32), (2, 256, 64), (2, 64, 128)])
def test_read_equals_the_definition(gpu, code, dtype, heads, dim, page):
    import torch
    s = Setup(gpu, RAGGED, heads, dim, page, code, seed=7).fill().to_gpu()
    K, V = s.rrq.cache_read(s.cache, s.batch,
                            torch.float32 if dtype == "f32" else torch.bfloat16)
    for name, got in (("k", K), ("v", V)):
        got = got.float().cpu().numpy()
        for b, (n, length) in enumerate(RAGGED):
            for h in range(heads):
                want = ora.dense(s.host, s.table[b], name, h, length)[length - n:]
                want = want.astype(np.float32)
                want = bf16(want) if dtype == "bf16" else want
                assert_same_blocks(got[s.offsets[b]:s.offsets[b + 1], h] + 0.0, want + 0.0,
                                   f"{name} of sequence {b}, head {h}")


@pytest.mark.parametrize("at", [3, 100])
def test_read_writes_only_the_batch_rows(gpu, at):
    import torch
    s = Setup(gpu, [(4, 20), (2, 5)], 1, 64, 16, "int8", seed=8).fill()
    s.offsets = [at, at + 4, at + 6]
    s.to_gpu(n_tokens=at + 9)
    K = torch.full((at + 9, 1, 64), 77.0, device="cuda")
    V = torch.full((at + 9, 1, 64), 77.0, device="cuda")
    s.rrq.cache_read(s.cache, s.batch, out=(K, V))
    inside = torch.zeros(at + 9, dtype=torch.bool)
    inside[at:at + 6] = True
    for t in (K, V):
        t = t.cpu()
        assert (t[~inside] == 77).all() and (t[inside].abs() < 10).all()


def test_pages_out_of_range_are_left_alone(gpu):
    """Page numbers past the cache and positions past the table are neither
    written nor read."""
    import torch
    s = Setup(gpu, [(40, 40), (10, 10)], 1, 64, 16, "int8", seed=9).fill()
    s.table[0, 1] = s.host.k.shape[0] + 5
    s.table[1, 0] = -1
    s.to_gpu()
    x = torch.ones((50, 1, 64), device="cuda")
    s.rrq.cache_write(s.cache, s.batch, x, x)
    K, _ = s.rrq.cache_read(s.cache, s.batch, torch.float32)
    K = K.cpu()
    # 127 fl(1/127) and its reciprocal product: 1 to a rounding
    assert torch.allclose(K[:16], torch.ones(()), atol=1e-6) and (K[16:32] == 0).all()
    assert torch.allclose(K[32:40], torch.ones(()), atol=1e-6) and (K[40:] == 0).all()
    # a length past the table: only the table's positions exist
    s.batch.lengths[0] = 50
    n_before = s.k.clone()
    s.rrq.cache_write(s.cache, s.batch, 2 * x, 2 * x)
    kept = [p for p in range(s.k.shape[0]) if p not in (s.table[0, 0], s.table[0, 2])]
    assert torch.equal(s.k[kept], n_before[kept])


def test_another_stream(gpu):
    import torch
    s = Setup(gpu, RAGGED, 2, 128, 32, "int8", seed=10).fill().to_gpu()
    want = s.rrq.cache_read(s.cache, s.batch)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = s.rrq.cache_read(s.cache, s.batch, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_long_cache_offsets_pass_32_bits(gpu):
    """Pages whose code offsets lie past 2^32 bytes."""
    import torch
    n_pages = (1 << 32) // (8 * 128 * 128) + 40
    cache = gpu.KVCache.empty(n_pages, 8, 128, 128, "int8")
    pages = [n_pages - 1, 3, n_pages - 7]
    batch = gpu.CacheBatch(torch.tensor([pages], dtype=torch.int32, device="cuda"),
                           torch.tensor([300], dtype=torch.int32, device="cuda"),
                           torch.tensor([0, 300], dtype=torch.int32, device="cuda"), 300)
    x = torch.randn((300, 8, 128), device="cuda")
    gpu.cache_write(cache, batch, x, x.flip(0))
    K, V = gpu.cache_read(cache, batch, torch.float32)
    # half a step of the block's scale, and the rounding of the scaled value
    step = x.abs().max() / 127
    assert (K - x).abs().max() <= 0.51 * step and (V - x.flip(0)).abs().max() <= 0.51 * step
    q = torch.randn((300, 16, 128), device="cuda")
    far = gpu.cache_attention(cache, batch, q, out_dtype=torch.float32)
    near_cache = gpu.KVCache.empty(3, 8, 128, 128, "int8")
    near = gpu.CacheBatch(torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda"),
                          batch.lengths, batch.offsets, 300)
    gpu.cache_write(near_cache, near, x, x.flip(0))
    want = gpu.cache_attention(near_cache, near, q, out_dtype=torch.float32)
    assert torch.equal(far, want)


def test_empty_calls(gpu):
    import torch
    s = Setup(gpu, [(0, 9), (0, 0)], 1, 64, 16, "int8", seed=11).fill().to_gpu()
    x = torch.empty((0, 1, 64), device="cuda")
    before = s.k.clone()
    s.rrq.cache_write(s.cache, s.batch, x, x)
    K, V = s.rrq.cache_read(s.cache, s.batch)
    assert K.shape == V.shape == (0, 1, 64) and torch.equal(before, s.k)
