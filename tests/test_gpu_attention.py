"""Attention over the 8-bit cache against the oracle in 64 bits.

Bound, from the header's arithmetic (u = 2^-11, one rounding to 11 bits):
a score is off by at most
    d = |scale| R (u [binary32 queries only] + (D + 8) 2^-24)
with R the largest sum |q||k| of the row (rounding of the query, of the binary32
sum, and of the few factors), and by |s| 2^-22 <= |scale| R 2^-22 from the
exponential's argument; weights change by e^(2d) - 1 at most, are rounded by
u, and both sums over n keys add n + 64 roundings of 2^-24. So
    |out - exact| <= (e^(2d) - 1 + 1.01 u + (n + 64) 2^-23) A + r |out|
with A the mean of |v| under the weights and r = 1.01 2^-8 (8 bits) for bfloat16
output (2^-23 for binary32), and 2^-30 of the largest |v| for weights below
the smallest normal of the rounded form.
"""

import numpy as np
import pytest

from oracle import serving as ora
from serving_helpers import Setup, bf16

pytestmark = pytest.mark.gpu
U16 = 2.0 ** -11


def _bound(s, Q, want, mean_abs, reach, scale, q_f32, out_bf16):
    D = Q.shape[2]
    d = abs(scale) * reach * ((U16 if q_f32 else 0) + (D + 8) * 2.0 ** -24 + 2.0 ** -22)
    rel = np.expm1(2 * d) + 1.01 * U16 + (max(s.lengths) + 64) * 2.0 ** -23
    r = 1.01 * 2.0 ** -8 if out_bf16 else 2.0 ** -23
    return (rel[..., None] * mean_abs + r * (np.abs(want) + rel[..., None] * mean_abs) +
            2.0 ** -30 * np.nanmax(mean_abs, initial=0.0) + 1e-37)


def _run(s, heads, scale=None, causal=True, window=0, q="bf16", out="f32", gain=1.0, **kw):
    torch = s.torch
    D = s.host.k.shape[3]
    T = s.offsets[-1]
    Q = (s.rng.normal(size=(T, heads, D)) * gain).astype(np.float32)
    if q == "bf16":
        Q = bf16(Q)
    s.to_gpu()
    dt = torch.bfloat16 if q == "bf16" else torch.float32
    wide = torch.full((max(T, 1), heads + 2, D), float("nan"), device="cuda", dtype=dt)
    wide[:T, 1:1 + heads] = torch.from_numpy(Q).cuda().to(dt)
    got = s.rrq.cache_attention(s.cache, s.batch, wide[:T, 1:1 + heads], scale, causal, window,
                                torch.float32 if out == "f32" else torch.bfloat16, **kw)
    got = got.float().cpu().numpy()
    scale = D ** -0.5 if scale is None else scale
    want, mean_abs, reach = ora.attention(s.host, s.table, s.lengths, s.offsets, Q, scale, causal,
                                          window)
    bound = _bound(s, Q, want, mean_abs, reach, scale, q == "f32", out == "bf16")
    assert np.isfinite(got).all(), np.argwhere(~np.isfinite(got))[:4]
    bad = np.abs(got - want) > bound
    assert not bad.any(), (np.argwhere(bad)[:4], (np.abs(got - want) / bound).max())
    return got, want


DECODE = [(1, 1), (1, 16), (1, 17), (1, 200), (1, 1030), (1, 64), (0, 5)]


@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("heads,kv,dim,page", [(4, 4, 64, 16), (8, 2, 128, 32), (5, 1, 128, 64),
                                               (4, 2, 256, 128), (16, 1, 64, 128), (3, 1, 256, 16),
                                               (36, 1, 128, 16)])
def test_single_tokens(gpu, code, heads, kv, dim, page):
    s = Setup(gpu, DECODE, kv, dim, page, code, seed=heads + dim).fill()
    _run(s, heads, q="f32", gain=1.5)


@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("q", ["f32", "bf16"])
def test_types(gpu, code, out, q):
    s = Setup(gpu, [(3, 70), (1, 300), (20, 20)], 2, 128, 16, code, seed=21).fill()
    _run(s, 6, q=q, out=out, gain=2.0)


@pytest.mark.parametrize("heads,kv,dim,page", [(4, 1, 64, 16), (6, 2, 128, 32), (2, 2, 256, 64),
                                               (5, 1, 128, 128)])
@pytest.mark.parametrize("seqs", [[(5, 300), (2, 2), (7, 64), (1, 129)],
                                  [(70, 70), (33, 180), (1, 5), (0, 0), (129, 400)],
                                  [(260, 515)]])
def test_several_tokens(gpu, heads, kv, dim, page, seqs):
    s = Setup(gpu, seqs, kv, dim, page, "int8", seed=dim + len(seqs)).fill()
    _run(s, heads, gain=1.5)


@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 200, 100000])
@pytest.mark.parametrize("seqs", [[(1, 700), (1, 64), (1, 1)], [(90, 300), (3, 65), (66, 66)]])
def test_windows(gpu, window, seqs):
    s = Setup(gpu, seqs, 1, 128, 16, "fp8", seed=window).fill()
    _run(s, 4, window=window, gain=1.5)


def test_pages_before_the_window_are_not_used(gpu):
    """A sliding-window cache may have freed them: their entries point
    nowhere, or at pages that hold anything."""
    s = Setup(gpu, [(1, 700), (40, 600)], 1, 128, 16, "fp8", seed=31).fill()
    kept = s.table.copy()
    s.table[0, :(699 - 99) // 16] = -1
    s.table[1, :(560 - 99) // 16] = s.spare[0]
    got_table = s.table
    D, T = 128, s.offsets[-1]
    Q = bf16(s.rng.normal(size=(T, 2, D)).astype(np.float32))
    s.to_gpu()
    got = s.rrq.cache_attention(s.cache, s.batch,
                                s.torch.from_numpy(Q).cuda().to(s.torch.bfloat16),
                                window=100, out_dtype=s.torch.float32).cpu().numpy()
    want, mean_abs, reach = ora.attention(s.host, kept, s.lengths, s.offsets, Q, D ** -0.5, True,
                                          100)
    bound = _bound(s, Q, want, mean_abs, reach, D ** -0.5, False, False)
    assert (got_table != kept).any() and (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("seqs", [[(3, 100), (1, 7)], [(50, 200), (20, 3), (2, 0)]])
@pytest.mark.parametrize("window", [0, 5])
def test_without_causality(gpu, seqs, window):
    s = Setup(gpu, seqs, 2, 64, 16, "int8", seed=41).fill()
    _run(s, 4, causal=False, window=window)


@pytest.mark.parametrize("code", ["int8", "fp8"])
def test_rows_that_see_nothing_are_zeros(gpu, code):
    # sequence 0 is empty; of sequence 1 the first 5 of 8 rows lie before its start
    s = Setup(gpu, [(2, 0), (8, 3), (1, 40)], 1, 64, 16, code, seed=42).fill()
    got, _ = _run(s, 3)
    assert (got[:7] == 0).all() and (np.abs(got[7:]).max(axis=(1, 2)) > 0).all()


def test_unequal_scales_of_one_tile(gpu):
    """Pages of one 64-key tile whose value scales differ by 2^40, and blocks
    that are all zero."""
    s = Setup(gpu, [(1, 64), (1, 300), (17, 200)], 1, 64, 16, "int8", seed=43).fill()
    for b, j, f in ((0, 1, 2.0 ** -40), (1, 0, 2.0 ** 30), (1, 7, 0.0), (2, 3, 2.0 ** 20)):
        page = s.table[b, j]
        s.host.vs[page] *= np.float32(f)
        if f == 0:
            s.host.v[page] = 0
    s.host.ks[s.table[1, 4]] = 0
    s.host.k[s.table[1, 4]] = 0
    _run(s, 2)


def test_peaked_and_flat_rows(gpu):
    s = Setup(gpu, [(1, 3000), (4, 900)], 1, 128, 64, "int8", seed=44).fill()
    _run(s, 4, scale=0.0)
    s = Setup(gpu, [(1, 3000), (4, 900)], 1, 128, 64, "int8", seed=45).fill()
    _run(s, 4, scale=3.0)
    s = Setup(gpu, [(1, 3000), (4, 900)], 1, 128, 64, "int8", seed=46).fill()
    _run(s, 4, scale=-0.2)


@pytest.mark.parametrize("gain", [1e-30, 1e-8, 1e8])
def test_query_ranges(gpu, gain):
    s = Setup(gpu, [(2, 150), (30, 90)], 1, 128, 32, "fp8", seed=47).fill()
    _run(s, 3, q="f32", gain=gain, scale=0.09 / gain)


@pytest.mark.parametrize("heads", [(3, 1), (8, 8)])
def test_queries_at_the_end_of_their_range(gpu, heads):
    # up to 2e37, past 2^16 times 2^107
    n, kv = heads
    s = Setup(gpu, [(100, 150), (130, 190)], kv, 128, 32, "fp8", seed=50).fill()
    _run(s, n, q="f32", gain=5e36, scale=0.09 / 5e36)


def test_zero_queries(gpu):
    s = Setup(gpu, [(2, 150)], 1, 128, 32, "int8", seed=48).fill()
    _run(s, 3, gain=0.0)


def test_a_query_that_is_not_a_number_stays_in_its_row(gpu):
    import torch
    s = Setup(gpu, [(40, 100), (1, 90)], 1, 64, 16, "int8", seed=49).fill().to_gpu()
    Q = torch.randn((41, 4, 64), device="cuda")
    want = s.rrq.cache_attention(s.cache, s.batch, Q)
    Q[7, 2, 5] = float("nan")
    Q[40, 0, 1] = float("inf")
    got = s.rrq.cache_attention(s.cache, s.batch, Q)
    hit = torch.zeros((41, 4), dtype=torch.bool, device="cuda")
    hit[7, 2] = hit[40, 0] = True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit])


def test_rows_outside_the_offsets_are_left(gpu):
    import torch
    for seqs, offsets, n in (([(4, 2000), (1, 50)], [2, 6, 7], 11), ([(90, 200)], [5, 95], 100)):
        s = Setup(gpu, seqs, 1, 64, 16, "int8", seed=50).fill()
        s.offsets = offsets
        s.to_gpu(n_tokens=n)
        Q = torch.randn((n, 4, 64), device="cuda")
        out = torch.full((n, 4, 64), 55.0, device="cuda")
        s.rrq.cache_attention(s.cache, s.batch, Q, out=out)
        inside = torch.zeros(n, dtype=torch.bool, device="cuda")
        inside[offsets[0]:offsets[-1]] = True
        assert (out[~inside] == 55).all() and (out[inside] != 55).all()


def test_many_sequences(gpu):
    """More sequences than one step of the sequence search compares."""
    rng = np.random.default_rng(51)
    seqs = [(int(rng.integers(0, 3)), int(rng.integers(2, 40))) for _ in range(300)]
    s = Setup(gpu, seqs, 1, 64, 16, "int8", seed=52).fill()
    _run(s, 2)


def test_pages_out_of_range_are_left_out(gpu):
    """Keys of an absent page do not count, as if masked."""
    s = Setup(gpu, [(1, 200), (60, 150)], 1, 64, 16, "int8", seed=53).fill()
    want_host = ora.Cache(*(x.copy() for x in (s.host.k, s.host.v, s.host.ks, s.host.vs)), "int8")
    kept = s.table.copy()
    s.table[0, 3] = 10 ** 6
    s.table[1, 2] = -5
    T = s.offsets[-1]
    Q = bf16(s.rng.normal(size=(T, 2, 64)).astype(np.float32))
    s.to_gpu()
    got = s.rrq.cache_attention(s.cache, s.batch,
                                s.torch.from_numpy(Q).cuda().to(s.torch.bfloat16),
                                out_dtype=s.torch.float32).cpu().numpy()
    for b, gone in ((0, 3), (1, 2)):
        n, length = s.new[b], s.lengths[b]
        k = ora.dense(want_host, kept[b], "k", 0, length)
        v = ora.dense(want_host, kept[b], "v", 0, length)
        for i in range(n):
            seen = np.arange(length) <= length - n + i
            seen[16 * gone:16 * gone + 16] = False
            for h in range(2):
                q = Q[s.offsets[b] + i, h].astype(np.float64)
                sc = k[seen] @ q / 8
                p = np.exp(sc - sc.max())
                p /= p.sum()
                # as _bound, for these sizes: d < 3e-4 of |scale| R < 30
                assert np.abs(got[s.offsets[b] + i, h] - p @ v[seen]).max() <= 2e-3 * (
                    p @ np.abs(v[seen])).max()


def test_a_kept_workspace_and_another_stream(gpu):
    import torch
    s = Setup(gpu, [(1, 5000), (2, 900)], 2, 128, 64, "int8", seed=54).fill().to_gpu()
    Q = torch.randn((3, 8, 128), device="cuda")
    want = s.rrq.cache_attention(s.cache, s.batch, Q)
    w = s.rrq.attention_workspace(s.cache, s.batch, 8)
    if w is not None:
        w.fill_(0xFF)
    assert torch.equal(s.rrq.cache_attention(s.cache, s.batch, Q, workspace=w), want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = s.rrq.cache_attention(s.cache, s.batch, Q, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    if w is not None:
        with pytest.raises(s.rrq.RRQError) as ei:
            s.rrq.cache_attention(s.cache, s.batch, Q, workspace=w[:w.numel() - 1])
        assert ei.value.status == s.rrq.RRQ_ERR_WORKSPACE


def test_results_are_deterministic(gpu):
    import torch
    s = Setup(gpu, [(1, 9000), (3, 4000), (100, 700)], 2, 128, 64, "fp8", seed=55).fill().to_gpu()
    Q = torch.randn((104, 8, 128), device="cuda")
    want = s.rrq.cache_attention(s.cache, s.batch, Q)
    for _ in range(5):
        assert torch.equal(s.rrq.cache_attention(s.cache, s.batch, Q), want)


def test_a_captured_step_follows_the_lengths(gpu):
    """Write and attention captured once; replayed as the sequences grow."""
    import torch
    s = Setup(gpu, [(1, 40), (1, 900)], 2, 128, 16, "int8", seed=56).fill()
    grown = 30
    table = np.full((2, s.table.shape[1] + 3), -7, np.int32)
    table[:, :s.table.shape[1]] = s.table
    pages = s.host.k.shape[0]
    for b, j in ((0, 3), (0, 4), (1, 57), (1, 58)):
        if table[b, j] < 0:
            table[b, j] = pages
            pages += 1
    for name in ("k", "v", "ks", "vs"):
        a = getattr(s.host, name)
        more = np.full((pages - a.shape[0],) + a.shape[1:], 0 if a.dtype == np.uint8 else 1, a.dtype)
        setattr(s.host, name, np.concatenate([a, more]))
    s.table = table
    s.to_gpu()
    K = torch.empty((2, 2, 128), device="cuda")
    Q = torch.empty((2, 8, 128), device="cuda")
    out = torch.empty((2, 8, 128), device="cuda", dtype=torch.bfloat16)
    w = s.rrq.attention_workspace(s.cache, s.batch, 8)

    def step():
        s.rrq.cache_write(s.cache, s.batch, K, K)
        s.rrq.cache_attention(s.cache, s.batch, Q, workspace=w, out=out)

    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    K.normal_(generator=g)
    Q.normal_(generator=g)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(grown):
        s.batch.lengths += 1
        K.normal_(generator=g)
        Q.normal_(generator=g)
        graph.replay()
        got = out.clone()
        torch.cuda.synchronize()
        step()              # the same tokens again: the same codes
        assert torch.equal(got, out), i
