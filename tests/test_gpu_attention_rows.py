"""Attention's many-row form (prompt chunks of several sequences and kv heads)
at its edges, within test_gpu_attention's bound. Calls of few row tiles take
the other form, so these have 8 kv heads or more rows."""

import numpy as np
import pytest

from oracle import serving as ora
from serving_helpers import Setup, bf16
from test_gpu_attention import _bound, _run

pytestmark = pytest.mark.gpu
KV = 8
RAGGED = [(70, 70), (33, 180), (1, 5), (0, 0), (129, 400)]


@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 32), (256, 64), (128, 128), (64, 128),
                                      (256, 16)])
def test_ragged_chunks(gpu, code, dim, page):
    s = Setup(gpu, RAGGED, KV, dim, page, code, seed=dim + page).fill()
    _run(s, 2 * KV, gain=1.5)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("q", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_types(gpu, q, out, dim):
    s = Setup(gpu, [(60, 70), (150, 300), (31, 31)], KV, dim, 16, "int8", seed=dim).fill()
    _run(s, KV, q=q, out=out, gain=2.0)


@pytest.mark.parametrize("window", [1, 2, 31, 63, 64, 65, 200, 100000])
@pytest.mark.parametrize("dim", [64, 256])
def test_windows(gpu, window, dim):
    s = Setup(gpu, [(90, 300), (3, 65), (166, 166)], KV, dim, 16, "fp8", seed=window + dim).fill()
    _run(s, 2 * KV, window=window, gain=1.5)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 5])
def test_without_causality(gpu, dim, window):
    s = Setup(gpu, [(80, 200), (60, 3), (40, 0), (90, 130)], KV, dim, 16, "int8",
              seed=dim).fill()
    _run(s, KV, causal=False, window=window)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_that_see_nothing_are_zeros(gpu, dim):
    s = Setup(gpu, [(100, 0), (200, 3), (60, 40)], KV, dim, 16, "fp8", seed=dim).fill()
    got, _ = _run(s, KV)
    seen = [297 <= i < 300 or i >= 300 + 20 for i in range(360)]
    assert (got[~np.array(seen)] == 0).all()
    assert (np.abs(got[np.array(seen)]).max(axis=(1, 2)) > 0).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("ratio,seqs", [(3, [(43, 200), (64, 300), (43, 43)]),
                                        (5, [(26, 100), (13, 40), (52, 300)]),
                                        (40, [(1, 300), (2, 70), (4, 130)])])
def test_groups_that_straddle_tiles(gpu, dim, ratio, seqs):
    s = Setup(gpu, seqs, KV, dim, 32, "int8", seed=dim + ratio).fill()
    _run(s, ratio * KV, gain=1.5)


@pytest.mark.parametrize("power", [-12, -25, -45, -100])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_most_of_the_weight_on_small_values(gpu, dim, power):
    s = Setup(gpu, [(100, 300), (100, 120), (100, 1500)], KV, dim, 16, "int8", seed=dim).fill()
    for b, kept in enumerate(((7,), (0, 7), (40, 60))):
        for j, page in enumerate(s.table[b]):
            if page >= 0 and j not in kept:
                s.host.vs[page] *= np.float32(2.0 ** power)
    _run(s, KV)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("powers", [(0, 30), (0, -40, 3, -20), (0, 65, 10), (-50, 30, -10, 60),
                                    (-70, 0, 10), (None, 0), (None, -30, None, 5)])
def test_rows_keep_their_precision_beside_larger_values(gpu, dim, powers):
    """As test_gpu_attention_forms', whose bound this is."""
    s = Setup(gpu, [(100, 160), (100, 100), (100, 900)], KV, dim, 16, "int8", seed=dim).fill()
    for table in s.table:
        for j, page in enumerate(table):
            if page >= 0:
                power = powers[j * len(powers) // 9 % len(powers)]
                s.host.vs[page] *= np.float32(0 if power is None else 2.0 ** power)
                if power is None:
                    s.host.v[page] = 0
    D, T = dim, s.offsets[-1]
    Q = bf16(s.rng.normal(size=(T, KV, D)).astype(np.float32))
    s.to_gpu()
    got = s.rrq.cache_attention(s.cache, s.batch, s.torch.from_numpy(Q).cuda().bfloat16(),
                                out_dtype=s.torch.float32).cpu().numpy()
    want, mean_abs, reach = ora.attention(s.host, s.table, s.lengths, s.offsets, Q, D ** -0.5,
                                          True, 0)
    d = D ** -0.5 * reach * ((D + 8) * 2.0 ** -24 + 2.0 ** -22)
    rel = np.expm1(2 * d) + 1.01 * 2.0 ** -11 + (max(s.lengths) + 64) * 2.0 ** -23
    bound = rel[..., None] * mean_abs * (1 + 2.0 ** -23) + 2.0 ** -23 * np.abs(want) + 1e-37
    far = np.abs(got - want) > bound + max(s.lengths) * 2.0 ** -30 * mean_abs.max(-1, keepdims=True)
    assert not far.any(), (np.argwhere(far)[:4], (np.abs(got - want) / bound).max())


def test_absent_pages_and_pages_before_the_window(gpu):
    """Keys of an absent page do not count; pages that only lie before the
    window are not used, wherever their entries point."""
    s = Setup(gpu, [(100, 600), (80, 300), (60, 150)], KV, 64, 16, "fp8", seed=3).fill()
    kept = s.table.copy()
    s.table[0, :(500 - 99) // 16] = -1
    s.table[1, :(220 - 99) // 16] = s.spare[0]
    s.table[2, 0] = 10 ** 6
    D, T = 64, s.offsets[-1]
    Q = bf16(s.rng.normal(size=(T, KV, D)).astype(np.float32))
    s.to_gpu()
    got = s.rrq.cache_attention(s.cache, s.batch, s.torch.from_numpy(Q).cuda().bfloat16(),
                                window=100, out_dtype=s.torch.float32).cpu().numpy()
    want, mean_abs, reach = ora.attention(s.host, kept, s.lengths, s.offsets, Q, D ** -0.5, True,
                                          100)
    # sequence 2, whose first page is absent: rows from position 116 on do not
    # see it (window 100), the ones before see 16 keys less
    ok = np.abs(got - want) <= _bound(s, Q, want, mean_abs, reach, D ** -0.5, False, False)
    assert ok[:180].all() and ok[180 + 116 - 90:].all()
    for i in range(180, 180 + 116 - 90):
        pos, h = 90 + i - 180, i % KV
        k = ora.dense(s.host, kept[2], "k", h, 150)[16:pos + 1]
        v = ora.dense(s.host, kept[2], "v", h, 150)[16:pos + 1]
        low = max(0, pos - 99 - 16)
        sc = k[low:] @ Q[i, h].astype(np.float64) / 8
        p = np.exp(sc - sc.max())
        p /= p.sum()
        # as test_gpu_attention's for absent pages
        assert np.abs(got[i, h] - p @ v[low:]).max() <= 2e-3 * (p @ np.abs(v[low:])).max()


def test_a_query_that_is_not_a_number_stays_in_its_row(gpu):
    import torch
    s = Setup(gpu, [(140, 200), (90, 90)], KV, 64, 16, "int8", seed=49).fill().to_gpu()
    Q = torch.randn((230, 2 * KV, 64), device="cuda")
    want = s.rrq.cache_attention(s.cache, s.batch, Q)
    Q[7, 2, 5] = float("nan")
    Q[200, 0, 1] = float("inf")
    got = s.rrq.cache_attention(s.cache, s.batch, Q)
    hit = torch.zeros((230, 2 * KV), dtype=torch.bool, device="cuda")
    hit[7, 2] = hit[200, 0] = True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit])


@pytest.mark.parametrize("gain", [1e-30, 1e-8, 1e8, 0.0])
def test_query_ranges(gpu, gain):
    s = Setup(gpu, [(100, 150), (130, 190)], KV, 128, 32, "fp8", seed=47).fill()
    _run(s, KV, q="f32", gain=gain, scale=0.09 / gain if gain else 0.09)


@pytest.mark.parametrize("scale", [0.0, 3.0, -0.2])
def test_peaked_and_flat_rows(gpu, scale):
    s = Setup(gpu, [(100, 900), (130, 400)], KV, 128, 64, "int8", seed=46).fill()
    _run(s, KV, scale=scale)


def test_rows_outside_the_offsets_are_left(gpu):
    import torch
    s = Setup(gpu, [(190, 300), (100, 200)], KV, 64, 16, "int8", seed=50).fill()
    s.offsets = [5, 195, 295]
    s.to_gpu(n_tokens=310)
    Q = torch.randn((310, KV, 64), device="cuda")
    out = torch.full((310, KV, 64), 55.0, device="cuda")
    s.rrq.cache_attention(s.cache, s.batch, Q, out=out)
    assert (out[:5] == 55).all() and (out[295:] == 55).all() and (out[5:295] != 55).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_several_ranges(gpu, dim):
    s = Setup(gpu, [(40, 2600), (70, 70), (0, 30), (33, 900), (90, 1500)], KV, dim, 64, "int8",
              seed=dim).fill()
    _run(s, 2 * KV, gain=1.5)
    assert s.rrq.attention_workspace(s.cache, s.batch, 2 * KV) is not None


def test_offsets_past_32_bits_and_captured(gpu):
    import torch
    s = Setup(gpu, [(200, 700), (200, 2000)], KV, 128, 128, "int8", seed=9).fill().to_gpu()
    Q = torch.randn((400, 2 * KV, 128), device="cuda")
    want = s.rrq.cache_attention(s.cache, s.batch, Q)
    used = s.host.k.shape[0]
    far = 36000
    big = s.rrq.KVCache.empty(far + used, KV, 128, 128, "int8")
    big.k_codes[far:], big.v_codes[far:] = s.k, s.v
    big.k_scales[far:], big.v_scales[far:] = s.ks, s.vs
    batch = s.rrq.CacheBatch(s.batch.page_table + far, s.batch.lengths, s.batch.offsets, 400)
    assert torch.equal(s.rrq.cache_attention(big, batch, Q), want)
    w = s.rrq.attention_workspace(big, batch, 2 * KV)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.rrq.cache_attention(big, batch, Q, workspace=w, out=out)
    for length in (2000, 1234, 300):
        batch.lengths[1] = length
        Q.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, s.rrq.cache_attention(big, batch, Q))
