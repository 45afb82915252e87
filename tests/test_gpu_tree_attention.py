"""Attention of drafted tokens over the 8-bit cache against the definition in 64
bits, within the bounds of test_gpu_attention.py (and, for binary32 results, whose
operands have 22 bits, those of test_gpu_attention_binary32.py)."""

import numpy as np
import pytest

from oracle import drafting as ora
from serving_helpers import Setup, bf16
from test_gpu_attention import _bound

pytestmark = pytest.mark.gpu


def paths(rng, n, chain=False):
    """For each row of a tree of n rows the set of rows from the root to it."""
    out = []
    for j in range(n):
        parent = j - 1 if chain else int(rng.integers(max(0, j // 3 - 1), max(1, j)))
        out.append((out[parent] if j else set()) | {j})
    return out


def words_of(sets, words):
    bits = np.zeros((len(sets), words), np.uint64)
    for i, s in enumerate(sets):
        for j in s:
            if j < 64 * words:
                bits[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return bits.view(np.int64)


def depths(sets, s):
    """Positions of rows by their depth."""
    return [length - n + len(sets[s.offsets[b] + i]) - 1
            for b, (n, length) in enumerate(zip(s.new, s.lengths)) for i in range(n)]


def run(s, heads, sets, window=0, positions=None, words=None, q="bf16", out="f32", gain=1.5,
        scale=None, check=True, **kw):
    torch = s.torch
    D, T = s.host.k.shape[3], s.offsets[-1]
    words = words or max(1, -(-max(s.new) // 64))
    Q = (s.rng.normal(size=(T, heads, D)) * gain).astype(np.float32)
    if q == "bf16":
        Q = bf16(Q)
    s.to_gpu()
    dt = torch.bfloat16 if q == "bf16" else torch.float32
    wide = torch.full((max(T, 1), heads + 2, D), float("nan"), device="cuda", dtype=dt)
    wide[:T, 1:1 + heads] = torch.from_numpy(Q).cuda().to(dt)
    seen = torch.from_numpy(words_of(sets, words)).cuda().view(T, words)
    at = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda")
    got = s.rrq.tree_attention(s.cache, s.batch, wide[:T, 1:1 + heads], seen, at, scale, window,
                               torch.float32 if out == "f32" else torch.bfloat16, **kw)
    result = got.float().cpu().numpy()
    scale = D ** -0.5 if scale is None else scale
    sets = [{j for j in x if j < 64 * words} for x in sets]
    want, mean_abs, reach = ora.tree_attention(s.host, s.table, s.lengths, s.offsets, Q, sets,
                                               positions, scale, window)
    assert np.isfinite(result).all(), np.argwhere(~np.isfinite(result))[:4]
    if check:
        bound = _bound(s, Q, want, mean_abs, reach, scale, q == "f32", out == "bf16")
        bad = np.abs(result - want) > bound
        assert not bad.any(), (np.argwhere(bad)[:4], (np.abs(result - want) / bound).max())
    return result, want


def trees(s, chain=False):
    return [x for n in s.new for x in paths(s.rng, n, chain)]


FEW = [(7, 300), (2, 2), (1, 64), (0, 9), (5, 129), (8, 8), (3, 66)]
MANY = [(70, 70), (33, 180), (65, 300), (0, 5), (129, 400), (64, 128), (1, 1)]


@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("heads,kv,dim,page", [(4, 4, 64, 16), (8, 2, 128, 32), (5, 1, 128, 64),
                                               (4, 2, 256, 128), (16, 1, 64, 128), (3, 1, 256, 16),
                                               (36, 1, 128, 16)])
@pytest.mark.parametrize("seqs", [FEW, MANY])
def test_trees(gpu, code, heads, kv, dim, page, seqs):
    s = Setup(gpu, seqs, kv, dim, page, code, seed=heads + dim).fill()
    run(s, heads, trees(s), q="f32")


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("q", ["f32", "bf16"])
@pytest.mark.parametrize("dim,code", [(64, "fp8"), (128, "int8"), (256, "int8")])
@pytest.mark.parametrize("seqs", [FEW, MANY])
def test_types(gpu, out, q, dim, code, seqs):
    s = Setup(gpu, seqs, 2, dim, 16, code, seed=21).fill()
    run(s, 6, trees(s), q=q, out=out, gain=2.0)


@pytest.mark.parametrize("window", [1, 2, 33, 64, 65, 200, 100000])
@pytest.mark.parametrize("seqs", [FEW, MANY])
@pytest.mark.parametrize("given", [False, True])
def test_windows(gpu, window, seqs, given):
    """Counted from a row's position: its depth, or its place."""
    s = Setup(gpu, seqs, 1, 128, 16, "fp8", seed=window).fill()
    sets = trees(s)
    run(s, 4, sets, window, depths(sets, s) if given else None)


def test_any_positions(gpu):
    """Positions that do not ascend, before the start and far past the end."""
    s = Setup(gpu, [(40, 300), (9, 200), (5, 5)], 1, 64, 16, "int8", seed=5).fill()
    far = [0, -5, 1 << 30, 170, -(1 << 31), (1 << 31) - 1, 100, 299]
    run(s, 4, trees(s), 50, [far[i % 8] for i in range(54)])
    run(s, 40, trees(s), 50, [far[i % 8] for i in range(54)])


@pytest.mark.parametrize("window", [(1 << 32) - 1, 1 << 32, 1 << 33, (1 << 63) - 1])
@pytest.mark.parametrize("seqs", [FEW, MANY])
def test_windows_longer_than_any_position(gpu, window, seqs):
    """They hide no key of a row at any position, in either attention."""
    import torch
    s = Setup(gpu, seqs, 1, 64, 16, "int8", seed=8).fill()
    low = -(1 << 31) if window > 1 << 32 else 0
    run(s, 4, trees(s), window, [(low, -1, 0, (1 << 31) - 1)[i % 4] if low else i % 4
                                 for i in range(s.offsets[-1])])
    Q = torch.randn((s.offsets[-1], 4, 64), device="cuda")
    got = gpu.cache_attention(s.cache, s.batch, Q, window=window, out_dtype=torch.float32)
    want = gpu.cache_attention(s.cache, s.batch, Q, out_dtype=torch.float32)
    # (ranges may be cut elsewhere; operands have 22 bits, scores are below 12)
    assert (got - want).abs().max() <= 2.0 ** -17 * want.abs().max()


@pytest.mark.parametrize("seqs", [FEW, MANY, [(100, 1000)]])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_a_chain_is_causal_attention(gpu, seqs, dim):
    import torch
    s = Setup(gpu, seqs, 2, dim, 32, "int8", seed=6).fill().to_gpu()
    T = s.offsets[-1]
    Q = torch.randn((T, 6, dim), device="cuda")
    seen = torch.from_numpy(words_of(trees(s, chain=True), 3)).cuda()
    for window in (0, 40):
        got = gpu.tree_attention(s.cache, s.batch, Q, seen, window=window,
                                 out_dtype=torch.float32)
        want = gpu.cache_attention(s.cache, s.batch, Q, window=window, out_dtype=torch.float32)
        if window:      # (there a window hides rows of the step too)
            short = torch.tensor([n <= 40 for n in s.new for _ in range(n)], device="cuda")
            if not short.any():
                continue
            got, want = got[short], want[short]
        # operands have 22 bits: scores (up to 12 here) are off by 12 x 2^-22 on either
        # side and weights by twice that, of means of at most the largest value
        assert (got - want).abs().max() <= 2.0 ** -17 * want.abs().max()


def test_any_bits(gpu):
    """Rows that see none of the step, all of it, later rows, not themselves; bits past
    the sequence's rows; fewer words than rows."""
    s = Setup(gpu, [(6, 40), (70, 200), (5, 5)], 2, 128, 16, "int8", seed=7).fill()
    sets = [set(), {0, 1, 2, 3, 4, 5}, {5}, {0, 63, 64, 100}, {1, 3}, set(range(192))]
    sets += [set(int(j) for j in s.rng.integers(0, 192, 20)) for _ in range(70)]
    sets += [set(), {4}, {0, 1}, {3, 7}, {64}]
    got, _ = run(s, 4, sets, words=3)
    assert (got[76] == 0).all() and (got[80] == 0).all() and (got[77] != 0).any()
    s2 = Setup(gpu, [(6, 40), (70, 200), (5, 5)], 2, 128, 16, "int8", seed=7).fill()
    run(s2, 4, sets, words=1)


def test_rows_that_see_nothing_are_zeros(gpu):
    """An empty sequence, rows before position 0, rows without bits or past; beside
    rows that see something."""
    s = Setup(gpu, [(2, 0), (8, 3), (1, 40), (40, 40)], 1, 64, 16, "fp8", seed=42).fill()
    sets = [{0}, {0, 1}] + [set(range(i + 1)) for i in range(8)] + [set()]
    sets += [set() if i % 2 else {i} for i in range(40)]
    got, want = run(s, 3, sets)
    assert (got[:7] == 0).all() and (got[12::2] == 0).all()
    assert (np.abs(got[7:11]).max(axis=(1, 2)) > 0).all()
    # many rows, beside a sequence long enough to be cut
    s = Setup(gpu, [(70, 0), (70, 3), (100, 3000), (0, 0), (66, 66)], 4, 64, 16, "int8",
              seed=44).fill()
    sets = trees(s)
    sets[-66:] = [set() if i % 2 else {i} for i in range(66)]
    got, want = run(s, 16, sets)
    assert (got[:70] == 0).all() and (got[70:137] == 0).all() and (got[241::2] == 0).all()


@pytest.mark.parametrize("kv", [1, 4])
@pytest.mark.parametrize("seqs", [[(25, 3000)], [(3, 5000), (40, 2100), (1, 30)], [(130, 2500)]])
def test_long_contexts(gpu, kv, seqs):
    """Keys split over workgroups, and joined."""
    s = Setup(gpu, seqs, kv, 64, 128, "int8", seed=8).fill()
    sets = trees(s)
    run(s, kv, sets)
    s = Setup(gpu, seqs, kv, 64, 128, "int8", seed=8).fill()
    run(s, kv, sets, 700, depths(sets, s))


def test_codes_that_no_row_sees(gpu):
    """Slots behind the sequences hold no numbers, pages before the window point
    nowhere."""
    s = Setup(gpu, [(20, 700), (4, 600)], 1, 128, 16, "fp8", seed=31).fill()
    sets = trees(s)
    kept = s.table.copy()
    at = depths(sets, s)
    s.table[0, :(680 - 99) // 16] = -1
    s.table[1, :(596 - 99) // 16] = s.spare[0]
    got, _ = run(s, 4, sets, 100, at, check=False, q="bf16")
    s2 = Setup(gpu, [(20, 700), (4, 600)], 1, 128, 16, "fp8", seed=31).fill()
    s2.rng = np.random.default_rng(0)
    s.table, s.rng = kept, np.random.default_rng(0)
    a, _ = run(s, 4, sets, 100, at)
    s.table = s.table.copy()
    s.table[0, :(680 - 99) // 16] = -1
    s.rng = np.random.default_rng(0)
    b, _ = run(s, 4, sets, 100, at, check=False)
    assert np.array_equal(a, b) and got.shape == a.shape


def test_unequal_scales(gpu):
    s = Setup(gpu, [(9, 64), (30, 300), (17, 200)], 1, 64, 16, "int8", seed=43).fill()
    for b, j, f in ((0, 1, 2.0 ** -40), (1, 0, 2.0 ** 30), (1, 7, 0.0), (2, 3, 2.0 ** 20)):
        page = s.table[b, j]
        s.host.vs[page] *= np.float32(f)
        if f == 0:
            s.host.v[page] = 0
    s.host.ks[s.table[1, 4]] = 0
    run(s, 4, trees(s))


def test_rows_behind_the_last_sequence(gpu):
    import torch
    s = Setup(gpu, [(3, 30), (40, 90)], 2, 64, 16, "int8", seed=9).fill().to_gpu(n_tokens=50)
    Q = torch.randn((50, 4, 64), device="cuda")
    seen = torch.full((50, 1), -1, dtype=torch.int64, device="cuda")
    out = torch.full((50, 4, 64), 7.0, device="cuda")
    gpu.tree_attention(s.cache, s.batch, Q, seen, out=out)
    assert (out[43:] == 7).all() and (out[:43] != 7).all()


def test_stream_graph_and_workspace(gpu):
    """On another stream; captured, and replayed as sequences grow and trees change."""
    import torch
    s = Setup(gpu, [(12, 1500), (30, 700), (5, 90)], 2, 128, 16, "int8", seed=10).fill().to_gpu()
    T = s.offsets[-1]
    Q = torch.randn((T, 8, 128), device="cuda")
    seen = torch.from_numpy(words_of(trees(s), 1)).cuda()
    at = torch.tensor(depths(trees(s), s), dtype=torch.int32, device="cuda")
    w = gpu.attention_workspace(s.cache, s.batch, 8)
    args = (s.cache, s.batch, Q, seen, at)
    want = gpu.tree_attention(*args, window=600)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = gpu.tree_attention(*args, window=600, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gpu.tree_attention(*args, window=600, workspace=w, out=out)
    for i in range(3):
        s.batch.lengths.sub_(3)
        at.sub_(3)
        seen.copy_(torch.from_numpy(words_of(trees(s), 1)))
        graph.replay()
        assert torch.equal(out, gpu.tree_attention(*args, window=600))
        torch.cuda.synchronize()


def test_cache_offsets_past_32_bits(gpu):
    """Pages whose codes lie 2^31 and 2^32 bytes into the cache."""
    import torch
    n_pages = (1 << 32) // (16 * 64 * 4) + 8
    cache = gpu.KVCache(torch.zeros((n_pages, 4, 16, 64), dtype=torch.uint8, device="cuda"),
                        torch.zeros((n_pages, 4, 64, 16), dtype=torch.uint8, device="cuda"),
                        torch.zeros((n_pages, 4), device="cuda"),
                        torch.zeros((n_pages, 4), device="cuda"))
    rotary = gpu.Rotary(gpu.rotary_frequencies(64))
    seen = torch.tensor([[1], [3], [5], [11]], dtype=torch.int64, device="cuda")
    Q, K, V = (torch.randn((4, 4, 64), device="cuda") for _ in range(3))
    outs = []
    for pages in ([0, 1], [n_pages // 2 + 1, n_pages - 2], [n_pages - 1, 3]):
        batch = gpu.CacheBatch(torch.tensor([pages], dtype=torch.int32, device="cuda"),
                               torch.tensor([18], dtype=torch.int32, device="cuda"),
                               torch.tensor([0, 4], dtype=torch.int32, device="cuda"), 4)
        past = gpu.CacheBatch(batch.page_table, torch.tensor([14], dtype=torch.int32,
                                                             device="cuda"),
                              torch.tensor([0, 14], dtype=torch.int32, device="cuda"), 14)
        g = torch.Generator(device="cuda").manual_seed(1)
        old = torch.randn((14, 4, 64), device="cuda", generator=g)
        gpu.cache_write(cache, past, old, old)
        q = gpu.cache_append(cache, batch, rotary, Q, K, V)
        outs.append(gpu.tree_attention(cache, batch, q, seen))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    assert outs[0].float().abs().max() > 0.1


def test_refusals(gpu):
    import torch
    s = Setup(gpu, [(3, 20), (2, 2)], 2, 128, 16, "int8", seed=11).fill().to_gpu()
    Q = torch.zeros((5, 4, 128), device="cuda")
    seen = torch.zeros((5, 1), dtype=torch.int64, device="cuda")

    def refused(error, match, Q=Q, seen=seen, **kw):
        with pytest.raises(error, match=match):
            gpu.tree_attention(s.cache, s.batch, Q, seen, **kw)

    refused(ValueError, "Q must be", Q=Q[:4])
    refused(ValueError, "seen", seen=seen[:4])
    refused(ValueError, "seen", seen=seen[:, 0])
    refused(ValueError, "seen", seen=seen.int())
    refused(ValueError, "seen", seen=seen.cpu())
    refused(ValueError, "seen", seen=torch.zeros((5, 2), dtype=torch.int64, device="cuda")[:, :1])
    refused(gpu.RRQError, "status", seen=torch.zeros((5, 0), dtype=torch.int64, device="cuda"))
    refused(ValueError, "positions", positions=torch.zeros(5, device="cuda"))
    refused(gpu.RRQError, "status", window=-1)
    refused(gpu.RRQError, "status", scale=float("nan"))
    refused(gpu.RRQError, "status", Q=torch.zeros((5, 3, 128), device="cuda"))
    refused(ValueError, "workspace", workspace=torch.zeros(16, device="cuda"))
    refused(TypeError, "out_dtype", out_dtype=torch.float16)
    refused(ValueError, "out must be", out=torch.zeros((5, 3, 128), device="cuda"))
