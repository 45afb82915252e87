"""Values near the end of binary32's range: a mean of them lies within it,
though their sum does not. Both forms of attention, whole ranges and joined
ones, within test_gpu_attention's bound (relative, so it holds here as it is)."""

import numpy as np
import pytest

from serving_helpers import Setup
from test_gpu_attention import _run

pytestmark = pytest.mark.gpu
# the largest value is below 1.27e38 (int8) and 1.35e38 (e4m3) at scales of 0.5 to 1.5 times these
LARGEST = {"int8": 0.66e36, "fp8": 0.2e36}


def _setup(rrq, seqs, kv, dim, page, code, positive):
    s = Setup(rrq, seqs, kv, dim, page, code, seed=dim + len(seqs)).fill()
    s.host.vs *= np.float32(LARGEST[code] / (0.02 if code == "int8" else 0.007))
    if positive:                # values of one sign: the sum grows with every key
        # (0xFF stands in slots without a token)
        s.host.v[s.host.v != 0xFF] &= 0x7F
    return s


@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows,longest", [(1, 900), (1, 9000), (24, 700), (24, 5000), (100, 4000)])
def test_few_row_tiles(gpu, code, dim, rows, longest):
    s = _setup(gpu, [(rows, longest), (rows, max(rows, 40))], 1, dim, 64, code, True)
    _run(s, 2, scale=0.0)
    _run(s, 2, out="bf16")


@pytest.mark.parametrize("code", ["int8", "fp8"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("longest", [300, 2600])
def test_many_rows(gpu, code, dim, longest):
    s = _setup(gpu, [(100, longest), (70, 70), (60, 100)], 8, dim, 64, code, True)
    _run(s, 8, scale=0.0)
    _run(s, 8, out="bf16")


@pytest.mark.parametrize("rows", [1, 100])
def test_small_scales_beside_them(gpu, rows):
    """Pages of ordinary values beside pages of large ones."""
    s = _setup(gpu, [(rows, 3000), (rows, 200)], 1, 128, 16, "int8", False)
    for table in s.table:
        for j, page in enumerate(table):
            if page >= 0 and j % 3:
                s.host.vs[page] *= np.float32(2.0 ** -60)
    _run(s, 2)
