"""Attention with a bfloat16 result, the default: its kernels take operands of
one part where a binary32 result's take two, so both have the edges of rows,
ranges, masks and scales tested. Bounds are test_gpu_attention's."""

import numpy as np
import pytest

from oracle import serving as ora
from serving_helpers import Setup, bf16
from test_gpu_attention import DECODE, _run

pytestmark = pytest.mark.gpu
OUT = dict(out="bf16", gain=1.5)


@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("heads,kv,dim,page", [(4, 4, 64, 16), (5, 1, 128, 64), (4, 2, 256, 128),
                                               (16, 1, 64, 128), (3, 1, 256, 16), (36, 1, 128, 16)])
def test_single_tokens(gpu, code, heads, kv, dim, page):
    s = Setup(gpu, DECODE, kv, dim, page, code, seed=heads + dim).fill()
    _run(s, heads, q="f32", **OUT)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("seqs", [[(5, 300), (2, 2), (7, 64), (1, 129)],
                                  [(70, 70), (33, 180), (1, 5), (0, 0), (129, 400)]])
@pytest.mark.parametrize("kv", [1, 8])
def test_several_tokens(gpu, dim, seqs, kv):
    """Few row tiles and, with 8 kv heads, many."""
    s = Setup(gpu, seqs, kv, dim, 32, "fp8", seed=dim + kv).fill()
    _run(s, 2 * kv, **OUT)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [1, 17, 32, 33, 65, 100])
@pytest.mark.parametrize("window", [0, 1, 65, 1500])
def test_ranges_and_windows(gpu, dim, rows, window):
    s = Setup(gpu, [(rows, 6000), (rows, rows), (rows, 700)], 1, dim, 64, "int8",
              seed=dim + rows).fill()
    _run(s, 2, window=window, **OUT)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 31, 65])
@pytest.mark.parametrize("code", ["int8", "fp8"])
def test_many_rows_in_ranges_and_windows(gpu, dim, window, code):
    s = Setup(gpu, [(40, 2600), (70, 70), (0, 30), (33, 900), (90, 1500)], 8, dim, 16, code,
              seed=dim).fill()
    _run(s, 16, window=window, **OUT)


@pytest.mark.parametrize("kv,seqs", [(2, [(3, 100), (1, 7)]), (2, [(50, 200), (20, 3), (2, 0)]),
                                     (8, [(80, 200), (60, 3), (40, 0), (90, 130)])])
@pytest.mark.parametrize("window", [0, 5])
@pytest.mark.parametrize("dim", [64, 256])
def test_without_causality(gpu, kv, seqs, window, dim):
    s = Setup(gpu, seqs, kv, dim, 16, "int8", seed=dim).fill()
    _run(s, 2 * kv, causal=False, window=window, **OUT)


@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("kv,seqs,seen", [(1, [(2, 0), (8, 3), (1, 40)], 7),
                                          (8, [(100, 0), (200, 3), (60, 60)], 297)])
def test_rows_that_see_nothing_are_zeros(gpu, code, kv, seqs, seen):
    s = Setup(gpu, seqs, kv, 64, 16, code, seed=42).fill()
    got, _ = _run(s, 3 * kv, **OUT)
    assert (got[:seen] == 0).all() and (np.abs(got[seen:]).max(axis=(1, 2)) > 0).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("ratio,seqs", [(3, [(43, 200), (64, 300), (43, 43)]),
                                        (40, [(1, 300), (2, 70), (4, 130)])])
def test_groups_that_straddle_tiles(gpu, dim, ratio, seqs):
    s = Setup(gpu, seqs, 8, dim, 32, "int8", seed=dim + ratio).fill()
    _run(s, ratio * 8, **OUT)


@pytest.mark.parametrize("kv,rows", [(1, 1), (1, 24), (8, 100)])
@pytest.mark.parametrize("power", [-12, -45, -100])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_most_of_the_weight_on_small_values(gpu, kv, rows, power, dim):
    s = Setup(gpu, [(rows, 300), (rows, 120), (rows, 1500)], kv, dim, 16, "int8", seed=dim).fill()
    for b, kept in enumerate(((7,), (0, 7), (40, 60))):
        for j, page in enumerate(s.table[b]):
            if page >= 0 and j not in kept:
                s.host.vs[page] *= np.float32(2.0 ** power)
    _run(s, 2 * kv, out="bf16")


@pytest.mark.parametrize("kv,rows", [(1, 6), (8, 100)])
@pytest.mark.parametrize("powers", [(0, 30), (0, -40, 3, -20), (-50, 30, -10, 60), (None, 0),
                                    (None, -30, None, 5)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_keep_their_precision_beside_larger_values(gpu, kv, rows, powers, dim):
    """As test_gpu_attention_forms', with the result's 8 bits."""
    s = Setup(gpu, [(rows, rows + 60), (rows, rows), (rows, 900)], kv, dim, 16, "int8",
              seed=dim + rows).fill()
    for table in s.table:
        for j, page in enumerate(table):
            if page >= 0:
                power = powers[j * len(powers) // 9 % len(powers)]
                s.host.vs[page] *= np.float32(0 if power is None else 2.0 ** power)
                if power is None:
                    s.host.v[page] = 0
    D, T = dim, s.offsets[-1]
    Q = bf16(s.rng.normal(size=(T, kv, D)).astype(np.float32))
    s.to_gpu()
    got = s.rrq.cache_attention(s.cache, s.batch, s.torch.from_numpy(Q).cuda().bfloat16())
    got = got.float().cpu().numpy()
    want, mean_abs, reach = ora.attention(s.host, s.table, s.lengths, s.offsets, Q, D ** -0.5,
                                          True, 0)
    d = D ** -0.5 * reach * ((D + 8) * 2.0 ** -24 + 2.0 ** -22)
    rel = np.expm1(2 * d) + 1.01 * 2.0 ** -11 + (max(s.lengths) + 64) * 2.0 ** -23
    off = (rel[..., None] * mean_abs +
           max(s.lengths) * 2.0 ** -30 * mean_abs.max(-1, keepdims=True))
    bound = off + 1.01 * 2.0 ** -8 * (np.abs(want) + off) + 1e-37
    far = np.abs(got - want) > bound
    assert not far.any(), (np.argwhere(far)[:4], (np.abs(got - want) / bound).max())


@pytest.mark.parametrize("kv,seqs", [(1, [(3, 150), (1, 9)]), (8, [(100, 150), (130, 190)])])
@pytest.mark.parametrize("gain", [1e-30, 1e8, 0.0])
def test_query_ranges(gpu, kv, seqs, gain):
    s = Setup(gpu, seqs, kv, 128, 32, "fp8", seed=47).fill()
    _run(s, kv, q="f32", out="bf16", gain=gain, scale=0.09 / gain if gain else 0.09)


@pytest.mark.parametrize("kv,seqs", [(1, [(3, 900), (1, 4000)]), (8, [(100, 900), (130, 400)])])
@pytest.mark.parametrize("scale", [0.0, 3.0, -0.2])
def test_peaked_and_flat_rows(gpu, kv, seqs, scale):
    s = Setup(gpu, seqs, kv, 128, 64, "int8", seed=46).fill()
    _run(s, kv, out="bf16", scale=scale)


@pytest.mark.parametrize("kv,rows", [(1, 1), (1, 40), (8, 100)])
def test_pages_before_the_window_are_not_used(gpu, kv, rows):
    s = Setup(gpu, [(rows, 700), (rows, 600)], kv, 128, 16, "fp8", seed=31).fill()
    kept = s.table.copy()
    s.table[0, :(700 - rows - 99) // 16] = -1
    s.table[1, :(600 - rows - 99) // 16] = s.spare[0]
    D, T = 128, s.offsets[-1]
    Q = bf16(s.rng.normal(size=(T, 2 * kv, D)).astype(np.float32))
    s.to_gpu()
    got = s.rrq.cache_attention(s.cache, s.batch, s.torch.from_numpy(Q).cuda().bfloat16(),
                                window=100)
    s.table = kept
    s.batch.page_table.copy_(s.torch.from_numpy(kept))
    want = s.rrq.cache_attention(s.cache, s.batch, s.torch.from_numpy(Q).cuda().bfloat16(),
                                 window=100)
    assert s.torch.isfinite(got).all() and s.torch.equal(got, want)
