"""Attention with a binary32 result: its operands carry 22 bits (queries of
binary32 and the softmax's weights as two parts of 11 bits each).

Bound, with u = 2^-24, A = |scale| R the largest sum of |scale| |q| |k| of the row,
C the query's channels other than 0 (terms of 0 round nothing) and n the keys
that the row sees. A score is off by at most
    d = A (2^-22 [binary32 queries] + 2 C 2^-23 + 5 u)     query's parts, sum, factors
      + (6 A + 135) u                 exponent's argument and what is subtracted from it
      + 28 u                          exponential, logarithm and reciprocal of the scales
weights change by e^(2d) - 1 at most and are rounded by 2^-21 in all; both sums
add 2 n + 64 roundings of 2^-23; weights below the rounded form's range lose
2^-38 of the largest contribution each: n 2^-38 of the largest |v|. With the
result's own 2^-23:
    |out - exact| <= (e^(2d) - 1 + 2^-21 + (2 n + 64) 2^-23) A_v + 2^-23 |out| + n 2^-38 v_max
with A_v the mean of |v| under the weights. Rows of few keys make this a
fraction of the 2^-11 that one rounding to 11 bits costs."""

import numpy as np
import pytest

from oracle import serving as ora
from serving_helpers import Setup, bf16

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
CHANNELS = 4


def _check(s, heads, q, gain=4.0, **kw):
    torch = s.torch
    D, T = s.host.k.shape[3], s.offsets[-1]
    Q = np.zeros((T, heads, D), np.float32)
    at = np.argsort(s.rng.random((T, heads, D)), axis=2)[:, :, :CHANNELS]
    np.put_along_axis(Q, at, (s.rng.normal(size=at.shape) * gain).astype(np.float32), 2)
    if q == "bf16":
        Q = bf16(Q)
    s.to_gpu()
    got = s.rrq.cache_attention(
        s.cache, s.batch, torch.from_numpy(Q).cuda().to(
            torch.bfloat16 if q == "bf16" else torch.float32),
        out_dtype=torch.float32, **kw).cpu().numpy()
    scale = D ** -0.5
    want, mean_abs, reach = ora.attention(s.host, s.table, s.lengths, s.offsets, Q, scale,
                                          kw.get("causal", True), kw.get("window", 0))
    n = np.zeros(T)
    for b, length in enumerate(s.lengths):
        new = s.offsets[b + 1] - s.offsets[b]
        n[s.offsets[b]:s.offsets[b + 1]] = (length - new + 1 + np.arange(new)
                                            if kw.get("causal", True) else length)
    n = n[:, None, None]
    A = scale * reach[..., None]
    d = (A * ((2.0 ** -22 if q == "f32" else 0) + 2 * CHANNELS * 2.0 ** -23 + 5 * U) +
         (6 * A + 135) * U + 28 * U)
    v_max = (127 * 0.03 if s.code == "int8" else 448 * 0.0105)
    bound = ((np.expm1(2 * d) + 2.0 ** -21 + (2 * n + 64) * 2.0 ** -23) * mean_abs *
             (1 + 2.0 ** -23) + 2.0 ** -23 * np.abs(want) + n * 2.0 ** -38 * v_max)
    bad = np.abs(got - want) > bound
    assert not bad.any(), (np.argwhere(bad)[:4], (np.abs(got - want) / bound).max())


@pytest.mark.parametrize("q", ["f32", "bf16"])
@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads", [3, 16, 20])
def test_few_rows(gpu, q, code, dim, heads):
    """One workgroup of many waves, tiles of 16 and of 32 rows."""
    s = Setup(gpu, [(1, 2), (1, 3), (1, 5), (1, 17), (1, 70), (1, 1)], 1, dim, 16, code,
              seed=dim + heads).fill()
    _check(s, heads, q)


@pytest.mark.parametrize("q", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [1, 3, 30])
def test_few_rows_in_several_ranges(gpu, q, dim, rows):
    """Short sequences beside one whose ranges are joined."""
    s = Setup(gpu, [(rows, 3000), (rows, rows), (rows, rows + 1), (rows, rows + 40)], 1, dim, 64,
              "int8", seed=dim + rows).fill()
    _check(s, 5, q)
    assert s.rrq.attention_workspace(s.cache, s.batch, 5) is not None


@pytest.mark.parametrize("q", ["f32", "bf16"])
@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_many_rows(gpu, q, code, dim):
    s = Setup(gpu, [(90, 90), (70, 72), (150, 150)], 8, dim, 32, code, seed=dim).fill()
    _check(s, 16, q)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_many_rows_in_several_ranges(gpu, dim):
    s = Setup(gpu, [(40, 2600), (70, 70), (90, 1500)], 8, dim, 64, "int8", seed=dim).fill()
    _check(s, 16, "f32")
    assert s.rrq.attention_workspace(s.cache, s.batch, 16) is not None


@pytest.mark.parametrize("rows,kv", [(1, 1), (100, 8)])
@pytest.mark.parametrize("causal,window", [(True, 3), (False, 2)])
def test_windows(gpu, rows, kv, causal, window):
    s = Setup(gpu, [(rows, 400), (rows, rows)], kv, 128, 16, "fp8", seed=rows).fill()
    _check(s, 2 * kv, "f32", window=window, causal=causal)
