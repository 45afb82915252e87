"""Token scoring against the oracle in 64 bits.

Bound: a lane adds V / 256 + 96 terms at most (its own, and the joins), each
with an exponential off by 2^-22 and 2^-23 of its exponent's argument (which
matters up to about 40); so with u = 2^-24 the sum l is off by
(V / 256 + 96 + 4 + 80) u of itself, a log probability by that and 4 u of
itself and of the difference to the largest logit; the entropy by the same on l
and on sum p |d|, d the difference to the largest logit. Ids are equal."""

import numpy as np
import pytest

from oracle import serving as ora
from serving_helpers import bf16

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _check(rrq, x, targets, n_top, dtype="f32", stride=None, **kw):
    import torch
    rows, vocab = x.shape
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    stride = vocab if stride is None else stride
    wide = torch.full((rows, stride), float("inf"), device="cuda", dtype=dt)
    wide[:, :vocab] = torch.from_numpy(x).cuda().to(dt)
    t = torch.from_numpy(targets).cuda()
    got = rrq.token_logprobs(wide[:, :vocab], t, n_top, **kw)
    lp, h, ids, top = ora.token_logprobs(x, targets, n_top)
    m = x.astype(np.float64).max(1, keepdims=True)
    d = np.where(np.isneginf(x), 0.0, x - np.where(np.isneginf(m), 0.0, m))
    e = np.where(np.isneginf(x), 0.0, np.exp(d))
    p = e / np.maximum(e.sum(1, keepdims=True), 1e-300)
    mean_d = (p * np.abs(d)).sum(1)
    base = (vocab / 256 + 180) * U
    inside = (targets >= 0) & (targets < vocab)
    dt_ = np.abs(d[np.arange(rows), np.where(inside, targets, 0)])
    for got_, want, bound in (
            (got[0], lp, base + 4 * U * (np.abs(np.where(np.isinf(lp), 0, lp)) + dt_)),
            (got[1], h, base * (2 + 2 * mean_d) + 4 * U * (np.abs(h) + mean_d))):
        g = got_.cpu().numpy().astype(np.float64)
        with np.errstate(invalid="ignore"):
            ok = (g == want) | (np.abs(g - want) <= bound)
        assert ok.all(), (np.argwhere(~ok)[:4], g[~ok][:4], want[~ok][:4])
    if n_top:
        assert np.array_equal(got[2].cpu().numpy(), ids)
        g = got[3].cpu().numpy().astype(np.float64)
        dd = np.abs(np.take_along_axis(d, ids, 1))
        with np.errstate(invalid="ignore"):
            ok = (g == top) | (np.abs(g - top) <= base + 4 * U * (
                np.abs(np.where(np.isinf(top), 0, top)) + dd))
        assert ok.all(), (np.argwhere(~ok)[:4])
    else:
        assert got[2] is None and got[3] is None


def _logits(rng, rows, vocab, dtype):
    x = (rng.normal(size=(rows, vocab)) * 3).astype(np.float32)
    x[rng.random((rows, vocab)) < 1e-3] += 8
    return bf16(x) if dtype == "bf16" else x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 64, 255, 2047, 2048, 2049, 8192, 8193, 33001,
                                   131072])
@pytest.mark.parametrize("rows", [1, 3])
def test_sizes(gpu, dtype, vocab, rows):
    rng = np.random.default_rng(vocab)
    x = _logits(rng, rows, vocab, dtype)
    for n_top in sorted({0, 1, min(5, vocab), min(32, vocab)}):
        _check(gpu, x, rng.integers(0, vocab, rows), n_top, dtype)


@pytest.mark.parametrize("rows", [17, 300, 1300])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_and_strides(gpu, rows, dtype):
    rng = np.random.default_rng(rows)
    x = _logits(rng, rows, 4099, dtype)
    _check(gpu, x, rng.integers(0, 4099, rows), 7, dtype, stride=4101)
    _check(gpu, x, rng.integers(0, 4099, rows), 20, dtype, stride=4099)


def test_orders_that_fill_the_buffer(gpu):
    """Ascending, descending, equal and two-valued rows, every n_top."""
    n = 20000
    up = np.arange(n, dtype=np.float32) / 4096
    two = np.where(np.arange(n) % 3 == 0, 1.0, 0.5).astype(np.float32)
    late = np.zeros(n, np.float32)
    late[-40:] = 3
    x = np.stack([up, up[::-1], np.full(n, 2.5, np.float32), two, late])
    t = np.array([0, n - 1, 77, 3, n - 1])
    for n_top in (1, 2, 31, 32):
        _check(gpu, x, t, n_top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_logits(gpu, dtype):
    rng = np.random.default_rng(5)
    x = _logits(rng, 8, 9001, dtype)
    x[0] = -np.inf                       # nothing left
    x[1, 1:] = -np.inf                   # one left
    x[2, :8000] = -np.inf
    x[3, 5:] = -np.inf                   # fewer left than n_top
    lowest = np.float32(-3.3895314e38)   # the lowest finite value of bfloat16
    x[4, 100:] = lowest
    x[5] = lowest
    x[6, ::2] = -np.inf
    t = np.array([4, 0, 8500, 2, 50, 9000, 1, -1])
    _check(gpu, x, t, 12, dtype)
    _check(gpu, x, np.array([0, 1, 0, 6, 9000, 0, 0, 9001]), 0, dtype)


def test_rows_with_nan_or_infinity(gpu):
    import torch
    rng = np.random.default_rng(6)
    x = _logits(rng, 5, 5000, "f32")
    want = x.copy()
    x[1, 3] = np.nan
    x[2, 4000] = np.inf
    x[3, :] = np.nan
    x[4, :4998] = -np.inf
    x[4, 4998] = np.nan
    lp, h, ids, top = (t.cpu().numpy() for t in gpu.token_logprobs(
        torch.from_numpy(x).cuda(), torch.zeros(5, dtype=torch.int64, device="cuda"), 4))
    assert np.isfinite(lp[0]) and np.isnan(lp[1:4]).all() and np.isnan(h[1:]).sum() >= 3
    assert np.isnan(h[1:4]).all()
    want[1, 3] = -np.inf
    assert np.array_equal(ids[1], np.argsort(-want[1], kind="stable")[:4])
    assert ids[2, 0] == 4000 and np.array_equal(ids[3], [0, 1, 2, 3])
    assert np.array_equal(ids[4], [4999, 0, 1, 2])


def test_without_targets_and_another_stream(gpu):
    import torch
    x = torch.randn((3, 50000), device="cuda")
    t = torch.tensor([1, 2, 3], device="cuda")
    want = gpu.token_logprobs(x, t, 9)
    got = gpu.token_logprobs(x, None, 9)
    assert got[0] is None and all(torch.equal(a, b) for a, b in zip(got[1:], want[1:]))
    w = gpu.logprobs_workspace(x, 9)
    assert w is not None
    w.fill_(0xFF)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = gpu.token_logprobs(x, t, 9, workspace=w, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(gpu.RRQError) as ei:
        gpu.token_logprobs(x, t, 9, workspace=w[:w.numel() - 1])
    assert ei.value.status == gpu.RRQ_ERR_WORKSPACE


def test_large_magnitudes(gpu):
    x = np.zeros((4, 3001), np.float32)
    x[0] = np.linspace(-1e30, 1e30, 3001)
    x[1] = 1e38
    x[1, 7] = -1e38
    x[2] = -1e38
    x[3, 5] = 3e38
    x[3, 6] = -3e38
    _check(gpu, x, np.array([3000, 0, 1, 5]), 5)


def test_no_rows(gpu):
    import torch
    out = gpu.token_logprobs(torch.empty((0, 100), device="cuda"),
                             torch.empty(0, dtype=torch.int64, device="cuda"), 3)
    assert out[0].shape == (0,) and out[2].shape == (0, 3)


def test_row_offsets_pass_32_bits(gpu):
    import torch
    vocab, rows = 70001, 1 << 15             # 4.6e9 bytes of bfloat16
    x = torch.zeros((rows, vocab), dtype=torch.bfloat16, device="cuda")
    x[rows - 1, vocab - 1] = 5.0
    x[rows - 1, 11] = 7.0
    t = torch.full((rows,), vocab - 1, dtype=torch.int64, device="cuda")
    lp, h, ids, top = gpu.token_logprobs(x, t, 2)
    last = np.zeros((1, vocab))
    last[0, vocab - 1], last[0, 11] = 5.0, 7.0
    want = ora.token_logprobs(last, np.array([vocab - 1]), 2)
    assert abs(lp[-1].item() - want[0][0]) < 1e-4 and ids[-1].tolist() == [11, vocab - 1]
    assert ids[0].tolist() == [0, 1] and abs(lp[0].item() + np.log(vocab)) < 1e-4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [3, 4, 5, 8, 9, 11, 2003, 4097, 6143, 6144, 6145, 8195])
def test_ends_of_rows(gpu, dtype, vocab):
    """A row's last block, for rows of less than one block a wave too; what
    lies past a row's end is not a logit."""
    rng = np.random.default_rng(vocab)
    x = _logits(rng, 37, vocab, dtype)
    x[5] = x[5, 0]
    x[6, -1] = 60.0
    x[7, :-1] = -np.inf
    t = rng.integers(0, vocab, 37)
    for n_top in (0, min(3, vocab), min(32, vocab)):
        _check(gpu, x, t, n_top, dtype, vocab + 3)
