"""Which form, tile and key ranges a call of attention takes: each of them at
its edges, within test_gpu_attention's bound. The number of ranges shows in
the workspace's size."""

import numpy as np
import pytest

from oracle import serving as ora
from serving_helpers import Setup, bf16
from test_gpu_attention import _bound, _run

pytestmark = pytest.mark.gpu


def _ranges(s, heads):
    w = s.rrq.attention_workspace(s.cache, s.batch, heads)
    if w is None:
        return 1
    n, rest = divmod(w.numel(), s.offsets[-1] * heads * (s.host.k.shape[3] + 2) * 4)
    assert rest == 0
    return n


@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("longest,least,most", [(2600, 2, 8), (9001, 9, 64)])
def test_few_rows_long_and_short_sequences(gpu, code, dim, longest, least, most):
    """Ranges joined by one wave or four; short sequences stay whole."""
    s = Setup(gpu, [(1, 100), (1, longest), (0, 0), (2, 700), (1, 1), (3, 2)], 1, dim, 32, code,
              seed=dim + longest).fill()
    _run(s, 5, gain=1.5)
    assert least <= _ranges(s, 5) <= most


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [17, 31, 32, 33, 50, 64, 65])
def test_row_tiles_of_each_form(gpu, dim, rows):
    """Rows a sequence on both sides of each tile's and form's limit."""
    s = Setup(gpu, [(rows, 3000), (rows, rows), (rows, 130)], 2, dim, 64, "int8",
              seed=dim + rows).fill()
    _run(s, 2, gain=1.5)


@pytest.mark.parametrize("dim,heads", [(64, 6), (128, 5), (64, 12)])
def test_wide_tiles_of_grouped_heads(gpu, dim, heads):
    s = Setup(gpu, [(5, 2500), (3, 3), (4, 300), (0, 40), (7, 8)], 1, dim, 16, "fp8",
              seed=dim + heads).fill()
    _run(s, heads, q="f32", out="bf16", gain=1.5)


@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_many_rows_in_several_ranges(gpu, code, dim):
    s = Setup(gpu, [(40, 5000), (70, 70), (0, 30), (33, 1800), (1, 900)], 1, dim, 64, code,
              seed=dim).fill()
    _run(s, 4, gain=1.5)
    assert _ranges(s, 4) > 1


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [1, 1500, 4500])
@pytest.mark.parametrize("rows", [1, 24, 150])
def test_windows_in_several_ranges(gpu, dim, window, rows):
    s = Setup(gpu, [(rows, 6000), (1, 10), (rows, 2000)], 1, dim, 128, "int8",
              seed=dim + window).fill()
    _run(s, 2, window=window, gain=1.5)


@pytest.mark.parametrize("rows", [1, 24, 100])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("power", [-12, -25, -45, -100])
def test_most_of_the_weight_on_small_values(gpu, rows, dim, power):
    """All pages but one or two hold values 2^power below theirs: they add
    little to the output, but their weights count in full."""
    s = Setup(gpu, [(rows, 300), (rows, 120), (rows, 3000)], 1, dim, 16, "int8",
              seed=rows + dim).fill()
    for b, kept in enumerate(((7,), (0, 7), (40, 120))):
        for j, page in enumerate(s.table[b]):
            if page >= 0 and j not in kept:
                s.host.vs[page] *= np.float32(2.0 ** power)
    _run(s, 2)


@pytest.mark.parametrize("rows", [6, 100])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("powers", [(0, 30), (0, -40, 3, -20), (0, 65, 10), (-50, 30, -10, 60),
                                    (-70, 0, 10), (None, 0), (None, -30, None, 5)])
def test_rows_keep_their_precision_beside_larger_values(gpu, rows, dim, powers):
    """Rows that see only a sequence's early pages, of small values, beside
    rows of the same tile that see larger ones: each row within its own bound
    (no share of the other rows' size). None: pages of zeros."""
    s = Setup(gpu, [(rows, rows + 60), (rows, rows), (rows, 2500)], 1, dim, 16, "int8",
              seed=rows + dim).fill()
    for table in s.table:
        for j, page in enumerate(table):
            if page >= 0:
                power = powers[j * len(powers) // max(len(table) // 20, 9) % len(powers)]
                s.host.vs[page] *= np.float32(0 if power is None else 2.0 ** power)
                if power is None:
                    s.host.v[page] = 0
    D, T = dim, s.offsets[-1]
    Q = bf16(s.rng.normal(size=(T, 2, D)).astype(np.float32))
    s.to_gpu()
    got = s.rrq.cache_attention(s.cache, s.batch, s.torch.from_numpy(Q).cuda().bfloat16(),
                                out_dtype=s.torch.float32).cpu().numpy()
    want, mean_abs, reach = ora.attention(s.host, s.table, s.lengths, s.offsets, Q, D ** -0.5,
                                          True, 0)
    # _bound's terms without the largest row's: weights below the rounded form's
    # normal range lose 2^-25 each, where the row's largest contribution has a
    # weight of 2^6 at least (n keys: 127 n 2^-31 of its code, taken as over 64)
    d = D ** -0.5 * reach * ((D + 8) * 2.0 ** -24 + 2.0 ** -22)
    rel = np.expm1(2 * d) + 1.01 * 2.0 ** -11 + (max(s.lengths) + 64) * 2.0 ** -23
    bound = rel[..., None] * mean_abs * (1 + 2.0 ** -23) + 2.0 ** -23 * np.abs(want) + 1e-37
    far = np.abs(got - want) > bound + max(s.lengths) * 2.0 ** -30 * mean_abs.max(-1, keepdims=True)
    assert not far.any(), (np.argwhere(far)[:4], (np.abs(got - want) / bound).max())


@pytest.mark.parametrize("rows", [1, 100])
def test_a_strided_page_table(gpu, rows):
    s = Setup(gpu, [(rows, 3000), (rows, 200)], 1, 64, 16, "int8", seed=rows).fill()
    D, T = 64, s.offsets[-1]
    Q = bf16(s.rng.normal(size=(T, 3, D)).astype(np.float32))
    s.to_gpu()
    n, pages = s.table.shape
    wide = s.torch.full((n, pages + 5), 10 ** 9, dtype=s.torch.int32, device="cuda")
    wide[:, 2:2 + pages] = s.batch.page_table
    batch = s.rrq.CacheBatch(wide[:, 2:2 + pages], s.batch.lengths, s.batch.offsets, T)
    got = s.rrq.cache_attention(s.cache, batch, s.torch.from_numpy(Q).cuda().bfloat16(),
                                out_dtype=s.torch.float32).cpu().numpy()
    want, mean_abs, reach = ora.attention(s.host, s.table, s.lengths, s.offsets, Q, D ** -0.5,
                                          True, 0)
    assert (np.abs(got - want) <= _bound(s, Q, want, mean_abs, reach, D ** -0.5, False,
                                         False)).all()


def test_lengths_that_no_table_holds(gpu):
    """A negative length is none; one past the table counts as far as the
    table reaches (the rows' positions stay the ones given)."""
    import torch
    for rows in (1, 60):
        s = Setup(gpu, [(rows, 64), (rows, 64), (rows, 64)], 1, 64, 16, "int8", seed=rows).fill()
        s.to_gpu()
        Q = torch.randn((3 * rows, 2, 64), device="cuda")
        want = s.rrq.cache_attention(s.cache, s.batch, Q, causal=False)
        s.batch.lengths[0] = -2 ** 31
        s.batch.lengths[2] = 2 ** 31 - 1
        got = s.rrq.cache_attention(s.cache, s.batch, Q, causal=False)
        assert (got[:rows] == 0).all() and torch.equal(got[rows:], want[rows:])


def test_refusals_of_tensors(gpu):
    import torch
    s = Setup(gpu, [(2, 40)], 2, 64, 16, "int8", seed=3).fill().to_gpu()
    Q = torch.zeros((2, 4, 64), device="cuda")
    K = torch.zeros((2, 2, 64), device="cuda")
    r = s.rrq
    i32 = dict(dtype=torch.int32, device="cuda")
    for error, call in (
            (TypeError, lambda: r.cache_attention(s.cache, s.batch, Q.half())),
            (ValueError, lambda: r.cache_attention(s.cache, s.batch, Q[:1])),
            (ValueError, lambda: r.cache_attention(s.cache, s.batch, Q[:, :, :32])),
            (ValueError, lambda: r.cache_attention(s.cache, s.batch, Q.transpose(1, 2))),
            (ValueError, lambda: r.cache_attention(s.cache, s.batch, Q.cpu())),
            (ValueError, lambda: r.cache_attention(s.cache, s.batch, Q, out=Q[:1])),
            (TypeError, lambda: r.cache_attention(s.cache, s.batch, Q, out=Q.half())),
            (ValueError, lambda: r.cache_attention(s.cache, s.batch, Q, workspace=Q)),
            (r.RRQError, lambda: r.cache_attention(s.cache, s.batch, Q[:, :3])),
            (r.RRQError, lambda: r.cache_attention(s.cache, s.batch, Q, scale=float("nan"))),
            (r.RRQError, lambda: r.cache_attention(s.cache, s.batch, Q, window=-1)),
            (TypeError, lambda: r.cache_write(s.cache, s.batch, K, K.bfloat16())),
            (ValueError, lambda: r.cache_write(s.cache, s.batch, K, K[:, :1])),
            (ValueError, lambda: r.cache_write(s.cache, s.batch, K[:1], K[:1])),
            (r.RRQError, lambda: r.cache_write(
                s.cache, s.batch, torch.zeros(257, device="cuda")[1:].view(2, 2, 64), K)),
            (ValueError, lambda: r.cache_read(s.cache, s.batch, out=(K, K[:1]))),
            (TypeError, lambda: r.cache_read(s.cache, s.batch, torch.float16)),
            (ValueError, lambda: r.KVCache(s.k, s.k, s.ks, s.vs)),
            (TypeError, lambda: r.KVCache(s.k, s.v, s.ks.double(), s.vs)),
            (TypeError, lambda: r.CacheBatch(s.batch.page_table.long(), s.batch.lengths,
                                             s.batch.offsets, 2)),
            (ValueError, lambda: r.CacheBatch(s.batch.page_table, s.batch.lengths,
                                              torch.zeros(3, **i32), 2)),
            (r.RRQError, lambda: r.KVCache.empty(2, 2, 96) and r.cache_write(
                r.KVCache.empty(2, 2, 96), s.batch, torch.zeros((2, 2, 96), device="cuda"),
                torch.zeros((2, 2, 96), device="cuda"))),
            (ValueError, lambda: r.token_logprobs(Q)),
            (TypeError, lambda: r.token_logprobs(Q[0].half())),
            (ValueError, lambda: r.token_logprobs(Q[0].t())),
            (ValueError, lambda: r.token_logprobs(Q[0], torch.zeros(4, device="cuda"))),
            (r.RRQError, lambda: r.token_logprobs(Q[0], n_top=33)),
            (r.RRQError, lambda: r.token_logprobs(Q[0], n_top=-1))):
        with pytest.raises(error):
            call()
    # nothing was enqueued: the stream still works
    assert (r.cache_attention(s.cache, s.batch, Q) != 55).all()


@pytest.mark.parametrize("rows", [1, 20, 90])
def test_cache_offsets_pass_32_bits(gpu, rows):
    """Pages past 4 GiB of codes (keys and values each) give what the same
    pages give at the start of a small cache."""
    import torch
    s = Setup(gpu, [(rows, 700), (rows, 2000)], 8, 128, 128, "int8", seed=rows).fill().to_gpu()
    Q = torch.randn((s.offsets[-1], 8, 128), device="cuda")
    want = s.rrq.cache_attention(s.cache, s.batch, Q)
    used = s.host.k.shape[0]
    far = 36000
    big = s.rrq.KVCache.empty(far + used, 8, 128, 128, "int8")
    assert big.k_codes[:far].numel() > 2 ** 32
    big.k_codes[far:], big.v_codes[far:] = s.k, s.v
    big.k_scales[far:], big.v_scales[far:] = s.ks, s.vs
    batch = s.rrq.CacheBatch(s.batch.page_table + far, s.batch.lengths, s.batch.offsets,
                             s.offsets[-1])
    assert torch.equal(s.rrq.cache_attention(big, batch, Q), want)


@pytest.mark.parametrize("rows", [1, 20, 200])
def test_a_captured_call_with_ranges(gpu, rows):
    """Write, attention over several ranges and scoring in one graph, replayed
    as lengths change, with eager work and synchronisation between."""
    import torch
    s = Setup(gpu, [(rows, 5000), (rows, 3000)], 1, 128, 64, "fp8", seed=rows).fill().to_gpu()
    T = s.offsets[-1]
    K = torch.empty((T, 1, 128), device="cuda")
    Q = torch.empty((T, 4, 128), device="cuda")
    logits = torch.empty((T, 20000), device="cuda")
    targets = torch.arange(T, device="cuda")
    out = torch.empty((T, 4, 128), device="cuda", dtype=torch.bfloat16)
    w = s.rrq.attention_workspace(s.cache, s.batch, 4)
    assert w is not None
    wl = s.rrq.logprobs_workspace(logits, 6)

    def step():
        s.rrq.cache_write(s.cache, s.batch, K, K)
        s.rrq.cache_attention(s.cache, s.batch, Q, workspace=w, out=out)
        return s.rrq.token_logprobs(logits, targets, 6, workspace=wl)

    g = torch.Generator(device="cuda")
    g.manual_seed(1)

    def fill():
        for t in (K, Q, logits):
            t.normal_(generator=g)

    fill()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for first, second in ((5000, 300), (4000, 2900), (rows, 3000), (4999, rows)):
        s.batch.lengths.copy_(torch.tensor([first, second], dtype=torch.int32))
        fill()
        graph.replay()
        got = [out.clone()] + [t.clone() for t in captured]
        torch.cuda.synchronize()
        want = step()               # the same tokens again: the same codes
        torch.cuda.synchronize()
        assert torch.equal(got[0], out)
        for a, b in zip(got[1:], want):
            assert torch.equal(a, b)
