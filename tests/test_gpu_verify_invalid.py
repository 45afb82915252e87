"""Target rows without a distribution (a NaN, +inf, nothing but -inf), also where what spoils
them is the very token of a rejected child; draft rows without one; what greedy calls make
of such rows."""

import numpy as np
import pytest

from test_gpu_verify import check, make

pytestmark = pytest.mark.gpu

BAD = {"nan": np.float32(np.nan), "inf": np.float32(np.inf)}
# (sequences of four rows, vocabulary): decided with the weights, and by a kernel before
# them (more than 256 blocks of 4096 logits)
FORMS = [(12, 9000), (200, 9000)]


def _walk(kind, seqs, vocab, dtype, bad):
    """Cases whose row 0 is spoilt (sequences 0 mod 4), whose row 1 is, below an
    accepted one (1 mod 4), that has two such tokens (2 mod 4), or none."""
    tree = kind == "tree"
    a, dtype, pad = make([4] * seqs, vocab, dtype, tree=tree, seed=41, sharp=1.0)
    rng = np.random.default_rng(42)
    a["uniforms"][:] = 0.5
    if tree:
        a["parents"][:] = np.tile([-1, 0, 0, 1], seqs)
    for b in range(seqs):
        r = 4 * b
        tokens = rng.choice(vocab, 4, replace=False)
        a["tokens"][r:r + 4] = tokens
        if b % 4 == 0:
            a["logits"][r, tokens[1]] = bad
        elif b % 4 == 1:
            a["logits"][r, tokens[1]] = 30.0
            a["logits"][r + 1, tokens[3 if tree else 2]] = bad
        elif b % 4 == 2:
            a["logits"][r, tokens[1]] = a["logits"][r, tokens[2]] = bad
    return a, dtype, pad


@pytest.mark.parametrize("bad", sorted(BAD))
@pytest.mark.parametrize("kind", ["chain", "tree"])
@pytest.mark.parametrize("seqs,vocab", FORMS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_rejected_token_spoils_its_row(gpu, dtype, seqs, vocab, kind, bad):
    case = _walk(kind, seqs, vocab, dtype, BAD[bad])
    counts, following, _ = check(gpu, case)
    counts, following = counts.tolist(), following.tolist()
    assert counts[0::4] == [0] * (seqs // 4) and following[0::4] == [-1] * (seqs // 4)
    assert counts[1::4] == [1] * (seqs // 4) and following[1::4] == [-1] * (seqs // 4)
    assert counts[2::4] == [0] * (seqs // 4) and following[2::4] == [-1] * (seqs // 4)
    assert min(following[3::4]) >= 0


@pytest.mark.parametrize("bad", sorted(BAD))
def test_spoilt_siblings_far_apart(gpu, bad):
    """The child that spoils the row is tried more than 64 rows before the last one."""
    a, dtype, pad = make([150], 6, tree=True, seed=43, sharp=0.5)
    a["parents"][1:] = 1
    a["parents"][[1, 100, 140]] = 0
    a["tokens"][[1, 100, 140]] = [3, 4, 2]
    a["logits"][0, 3] = BAD[bad]
    counts, following, _ = check(gpu, (a, dtype, pad))
    assert counts.item() == 0 and following.item() == -1


@pytest.mark.parametrize("kind", ["chain", "tree"])
@pytest.mark.parametrize("seqs,vocab", FORMS)
def test_rows_of_minus_infinity(gpu, seqs, vocab, kind):
    a, dtype, pad = _walk(kind, seqs, vocab, "f32", np.float32(0))
    a["logits"][::4] = -np.inf
    counts, following, _ = check(gpu, (a, dtype, pad))
    assert (counts == 0).all() and (following == -1).all()


def test_a_draft_row_without_a_distribution_rejects(gpu):
    """And the next token is drawn from p itself."""
    a, dtype, pad = make([2] * 8, 5000, draft=True, seed=44)
    a["uniforms"][1::2] = 0.0       # (u q < p, were there a q)
    a["draft"][0::4, 0] = -np.inf
    a["draft"][1::4, 0, 77] = np.nan
    a["draft"][2::4, 0, 78] = np.inf
    counts, following, _ = check(gpu, (a, dtype, pad))
    assert counts.tolist() == [0, 0, 0, 1] * 2 and (following >= 0).all()


@pytest.mark.parametrize("vocab", [5, 9000, 70001])
def test_greedy_infinities(gpu, vocab):
    """At a temperature of 0 the first of the largest logits, -inf and +inf being numbers
    as others and a NaN less than any; nothing but NaN: none."""
    a, dtype, pad = make([2] * 5, vocab, seed=45)
    a["tokens"][1::2] = [0, 3, 4, 2, 0]
    a["logits"][0] = -np.inf                # 0, and the draft is it
    a["logits"][2, [3, 4]] = np.inf         # 3
    a["logits"][4] = np.nan
    a["logits"][4, 4] = -np.inf             # 4
    a["logits"][6] = np.nan                 # none
    a["logits"][8, :3] = np.nan             # the largest of the others
    counts, following, paths = check(gpu, (a, dtype, pad), 0.0)
    assert counts.tolist() == [1, 1, 1, 0, 0]
    assert following[3].item() == -1
    assert following[4].item() == 3 + int(np.argmax(a["logits"][8, 3:]))
    assert paths.tolist()[3] == [0, -1]
