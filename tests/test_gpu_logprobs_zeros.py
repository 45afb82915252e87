"""Negative zero among the logits: it equals positive zero, so the lower index
comes first. In every form: a block of one wave, several waves, several
segments of a row, and more equal values than a wave's buffer holds. Bounds
are test_gpu_logprobs'."""

import numpy as np
import pytest

from test_gpu_logprobs import _check

pytestmark = pytest.mark.gpu


def _rows(vocab):
    """Rows whose places are decided among zeros of both signs."""
    rng = np.random.default_rng(vocab)
    even = np.arange(vocab) % 2 == 0
    minus, plus = np.float32(-0.0), np.float32(0.0)
    rows = [np.where(even, minus, plus), np.where(even, plus, minus),
            np.where(np.arange(vocab) < vocab // 2, minus, plus),      # all of one sign first
            np.where(rng.random(vocab) < 0.5, minus, plus),
            np.where(np.arange(vocab) < vocab - 1, minus, plus)]
    few = np.where(even, minus, plus)                # some larger, the last places zeros
    few[rng.integers(0, vocab, 3)] = 2.5
    rare = np.full(vocab, np.float32(-1.0))          # zeros above everything else
    rare[rng.integers(0, vocab, 5)] = plus
    rare[rng.integers(0, vocab, 5)] = minus
    tiny = np.where(even, minus, plus)               # numbers next to zero on both sides
    tiny[vocab // 3] = np.float32(2.0 ** -120)
    tiny[vocab // 2] = np.float32(-2.0 ** -120)
    return np.stack(rows + [few, rare, tiny]).astype(np.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [2, 50, 2048, 6200, 40000])
def test_zeros_of_both_signs(gpu, dtype, vocab):
    x = _rows(vocab)
    assert (np.signbit(x) & (x == 0)).any() and (~np.signbit(x) & (x == 0)).any()
    rng = np.random.default_rng(1)
    for n_top in sorted({1, 2, min(7, vocab), min(32, vocab)}):
        _check(gpu, x, rng.integers(0, vocab, len(x)), n_top, dtype)
