"""Pins of the drafting oracle: torch's norms and softmax in 64 bits, closed forms of
rotations, hand-worked walks, distributions by counting. CPU only."""

import itertools

import numpy as np
import pytest
import torch

from oracle import drafting as dra
from oracle import serving as ora


def test_norms_are_torchs():
    rng = np.random.default_rng(0)
    x, y, g = (rng.normal(size=(5, 33)) for _ in range(3))
    w, b, pw = (rng.normal(size=33) for _ in range(3))
    t = [torch.from_numpy(v) for v in (x, y, g, w, b, pw)]
    rms = torch.nn.functional.rms_norm(t[1], (33,), t[5], 1e-3)
    h = t[0] + 0.5 * t[2] * rms
    want = torch.nn.functional.layer_norm(h, (33,), t[3], t[4], 1e-3)
    got, got_h = dra.block_norm(x, y, w, b, "layer", "rms", pw, g, 0.5, 1e-3)
    assert np.allclose(got_h, h.numpy(), rtol=1e-13) and np.allclose(got, want.numpy(), rtol=1e-12)
    got, got_h = dra.block_norm(x, None, None, None, "rms", None, None, None, 1.0, 0.0)
    assert np.array_equal(got_h, x) and np.allclose(np.square(got).mean(1), 1, rtol=1e-14)


def test_norm_errors_bound_binary32():
    """The same formulas in numpy's binary32, sums one by one over at most 89 terms."""
    rng = np.random.default_rng(1)
    f32 = np.float32
    x, y, g = (rng.normal(size=(50, 60)).astype(f32) * f32(3) for _ in range(3))
    w = rng.normal(size=60).astype(f32)

    def norm(v, kind):
        if kind == "layer":
            v = v - np.add.accumulate(v, 1, dtype=f32)[:, -1:] * f32(1 / 60)
        s = np.add.accumulate(v * v, 1, dtype=f32)[:, -1:] * f32(1 / 60) + f32(1e-6)
        return v * (f32(1) / np.sqrt(s))

    for kind, post in itertools.product(("rms", "layer"), ("rms", "layer")):
        h = x + norm(y, post) * w * g * f32(0.3)
        out = norm(h, kind) * w + w
        host = (x, y, w, w, kind, post, w, g, np.float64(f32(0.3)), np.float64(f32(1e-6)))
        want, want_h = dra.block_norm(*host)
        err, err_h = dra.block_norm_error(*host)
        assert out.dtype == f32 and (np.abs(out - want) <= err).all()
        assert (np.abs(h - want_h) <= err_h).all()
        assert (err < 1e-4 * (1 + np.abs(want) + np.abs(w))).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotations(layout):
    """Lengths stay, products depend on distances alone, a quarter turn swaps a pair, what is
    not rotated stays bit for bit."""
    rng = np.random.default_rng(2)
    f = 10000.0 ** (-np.arange(16) / 16)
    x = rng.normal(size=(1, 2, 40)).astype(np.float32)
    at = np.array([0, 3, 1000, 123456])
    r = dra.rotate(np.repeat(x, 4, 0), at, f, layout, 1.0).astype(np.float64)
    assert np.array_equal(r[0], x[0]) and np.array_equal(r[..., 32:], np.repeat(x, 4, 0)[..., 32:])
    assert np.allclose(np.linalg.norm(r, axis=2), np.linalg.norm(x, axis=2), rtol=1e-6)
    s = dra.rotate(np.repeat(x, 4, 0), at + 77, f, layout, 1.0).astype(np.float64)
    dots = (r * s).sum(2)
    assert np.allclose(dots, dots[:1], rtol=1e-5, atol=1e-5)
    quarter = dra.rotate(x, [1], np.full(16, np.pi / 2), layout, 2.0)
    a, b = (x[..., :16], x[..., 16:32]) if layout == "half" else (x[..., :32:2], x[..., 1:32:2])
    qa, qb = ((quarter[..., :16], quarter[..., 16:32]) if layout == "half" else
              (quarter[..., :32:2], quarter[..., 1:32:2]))
    assert np.allclose(qa, -2 * b, atol=1e-6) and np.allclose(qb, 2 * a, atol=1e-6)


def _cache(length, code="int8"):
    rng = np.random.default_rng(3)
    pages = -(-length // 16)
    c = ora.Cache(rng.integers(0, 100, (pages, 2, 16, 8)).astype(np.uint8),
                  rng.integers(0, 100, (pages, 2, 8, 16)).astype(np.uint8),
                  rng.uniform(0.01, 0.02, (pages, 2)).astype(np.float32),
                  rng.uniform(0.01, 0.02, (pages, 2)).astype(np.float32), code)
    return c, [list(range(pages))]


def test_a_chain_is_causal_attention():
    c, table = _cache(50)
    Q = np.random.default_rng(4).normal(size=(7, 4, 8)).astype(np.float32)
    sets = [set(range(i + 1)) for i in range(7)]
    for window in (0, 20):
        got = dra.tree_attention(c, table, [50], [0, 7], Q, sets, None, 0.3, window)
        want = ora.attention(c, table, [50], [0, 7], Q, 0.3, True, window)
        for g, w in zip(got, want):
            assert np.allclose(g, w, rtol=1e-14)


def test_trees_by_a_dense_mask():
    c, table = _cache(40)
    rng = np.random.default_rng(5)
    Q = rng.normal(size=(6, 2, 8)).astype(np.float32)
    sets = [{0}, {0, 1}, {0, 2}, {0, 1, 3}, set(), {5, 9}]
    at = [34, 35, 35, 36, 10, 34]
    got, _, _ = dra.tree_attention(c, table, [40], [0, 6], Q, sets, at, 0.2, 12)
    for h in range(2):
        k, v = (torch.from_numpy(ora.dense(c, table[0], n, h, 40)) for n in ("k", "v"))
        s = 0.2 * torch.from_numpy(Q[:, h].astype(np.float64)) @ k.t()
        seen = torch.zeros(6, 40, dtype=torch.bool)
        for i in range(6):
            for j in range(34):
                seen[i, j] = j > at[i] - 12
            for j in sets[i]:
                if j < 6:
                    seen[i, 34 + j] = True
        p = torch.softmax(s.masked_fill(~seen, float("-inf")), 1)
        assert np.allclose(got[:, h], (p @ v).numpy(), rtol=1e-12)


LOG = np.log


def test_hand_worked_walks():
    """p = (1/2, 1/4, 1/4) after every row."""
    x = np.tile(LOG([0.5, 0.25, 0.25]), (4, 1))
    one = dict(offsets=[0, 4], max_accept=3)
    # u = 0.3 < 1/2 accepts 0; 0.3 >= 1/4 rejects 1, of which (2/3, 0, 1/3) is left; 0.7 draws 2
    c, f, p, _ = dra.verify(x, [9, 0, 1, 0], uniforms=[0.7, 0.3, 0.3, 0.0], **one)
    assert c.tolist() == [1] and f.tolist() == [2] and p.tolist() == [[0, 1, -1, -1]]
    # siblings: 0 rejected (0.6), then 1 has 1/4 of 1/2 left: 0.45 accepts it; then nothing
    # is tried under it and 0.5 draws 1, the first past half
    c, f, p, _ = dra.verify(x, [9, 0, 1, 2], uniforms=[0.5, 0.6, 0.45, 0.0],
                            parents=[-1, 0, 0, 0], **one)
    assert c.tolist() == [1] and f.tolist() == [1] and p.tolist() == [[0, 2, -1, -1]]
    # 0 and 1 rejected: 2 alone is left and accepted at any number
    c, f, p, _ = dra.verify(x, [9, 0, 1, 2], uniforms=[0.2, 0.6, 0.55, 0.99],
                            parents=[-1, 0, 0, 0], **one)
    assert c.tolist() == [1] and f.tolist() == [0] and p.tolist() == [[0, 3, -1, -1]]
    # the draft was sure of 1: 0.2 x 1 < 1/4 accepts it, 0.3 does not and p - q leaves 0 and 2
    q = np.log([[[1e-9, 1.0, 1e-9]] * 3])
    c, f, _, _ = dra.verify(x, [9, 1, 1, 1], uniforms=[0.9, 0.2, 0.3, 0.1], draft=q, **one)
    assert c.tolist() == [1] and f.tolist() == [2]
    # greedy: 0 is the likeliest; at most max_accept
    c, f, p, _ = dra.verify(x, [9, 0, 0, 0], uniforms=[0.9] * 4, offsets=[0, 4], max_accept=2,
                            temperature=0)
    assert c.tolist() == [2] and f.tolist() == [0] and p.tolist() == [[0, 1, 2]]


@pytest.mark.parametrize("given", [False, True])
def test_first_tokens_have_the_targets_distribution(given):
    """Counted over a grid of random numbers, and over the drafted token's own
    distribution: the target's probabilities. The coarser grid, of the drawn tokens, has
    steps of a tenth, and half of one at most is on the wrong side of a border."""
    p = np.array([0.5, 0.2, 0.2, 0.1])
    q = np.array([0.1, 0.3, 0.2, 0.4])
    grid = (np.arange(60) + 0.5) / 60
    mass = np.zeros(4)
    x = np.tile(LOG(p), (2, 1))
    for t in range(4):
        for u1, u0 in itertools.product(grid, grid[::6]):
            c, f, path, _ = dra.verify(x, [9, t], offsets=[0, 2], max_accept=1, uniforms=[u0, u1],
                                       draft=LOG(q)[None, None] if given else None)
            mass[t if c[0] else f[0]] += (q[t] if given else 0.25) / 600
    assert np.abs(mass - p).max() < 0.05
