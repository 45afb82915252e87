"""Pins of the oracle of the cache, attention and token scoring: closed forms,
torch's own e4m3 type, brute force. CPU only."""

import numpy as np
import pytest

from oracle import serving as ora


def test_fp8_values_are_torchs():
    import torch
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(got, ora.fp8_values().astype(np.float32), equal_nan=True)
    assert np.nanmax(ora.fp8_values()) == 448


def test_encode_picks_the_nearest_code():
    import torch
    rng = np.random.default_rng(0)
    y = np.concatenate([rng.normal(size=4000) * 100, rng.normal(size=4000) * 0.01,
                        ora.fp8_values()[:127], [448.0, -448.0, 1e9, -1e9, 0.0, 2.0 ** -10]])
    y = y.astype(np.float32)
    values = ora.fp8_values()
    got = ora.decode(ora.encode(y, "fp8"), "fp8")
    best = np.nanmin(np.abs(values[None, :] - np.clip(y, -448, 448)[:, None]), 1)
    assert np.array_equal(np.abs(got - np.clip(y, -448, 448)), best)
    want = torch.from_numpy(np.clip(y, -448, 448)).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(got, want)
    got = ora.decode(ora.encode(y, "int8"), "int8")
    assert np.array_equal(got, np.clip(np.rint(y), -127, 127))
    assert ora.decode(ora.encode([0.5, 1.5, -2.5, 200], "int8"), "int8").tolist() == [0, 2, -2, 127]
    # between 16 and 18 lies 17, a tie: 16 has the even mantissa; 19 goes to 20
    assert ora.decode(ora.encode([17.0, 19.0, -17.0], "fp8"), "fp8").tolist() == [16, 20, -16]


def _cache(pages, heads, page, dim, code):
    return ora.Cache(np.zeros((pages, heads, page, dim), np.uint8),
                     np.zeros((pages, heads, dim, page), np.uint8),
                     np.full((pages, heads), np.nan, np.float32),
                     np.full((pages, heads), np.nan, np.float32), code)


@pytest.mark.parametrize("code", ["int8", "fp8"])
def test_written_values_lie_within_half_a_step(code):
    rng = np.random.default_rng(1)
    c = _cache(4, 2, 16, 8, code)
    K = rng.normal(size=(37, 2, 8)).astype(np.float32)
    ora.write(c, [[2, 0, 3]], [37], [0, 37], K, -K)
    for h in range(2):
        got = ora.dense(c, [2, 0, 3], "k", h, 37)
        assert np.array_equal(got, -ora.dense(c, [2, 0, 3], "v", h, 37))
        for j, page in enumerate([2, 0, 3]):
            part = slice(16 * j, min(37, 16 * j + 16))
            top = np.abs(K[part, h]).max()
            assert abs(c.ks[page, h] - top / ora.C_MAX[code]) <= 1e-6 * c.ks[page, h]
            step = 0.5 * c.ks[page, h] if code == "int8" else np.abs(K[part, h]) / 16 + 1e-3 * top
            assert (np.abs(got[part] - K[part, h]) <= 1.0001 * step).all()


def test_a_hand_written_page():
    """int8: 127 units of the first write, then a token of twice the range:
    the scale doubles and the codes already there halve (ties to even)."""
    c = _cache(1, 1, 16, 4, "int8")
    s = np.float32(np.float32(127) * (np.float32(1) / np.float32(127)))
    K = np.array([[[127, 3, -1, 0]]], np.float32)
    ora.write(c, [[0]], [1], [0, 1], K, K)
    assert c.ks[0, 0] == s
    assert ora.decode(c.k[0, 0, 0], "int8").tolist() == [127, 3, -1, 0]
    K = np.array([[[254, 0, 2, 1]]], np.float32)
    ora.write(c, [[0]], [2], [0, 1], K, K)
    assert c.ks[0, 0] == 2 * s
    assert ora.decode(c.k[0, 0, 0], "int8").tolist() == [64, 2, 0, 0]
    assert ora.decode(c.v[0, 0, :, 1], "int8").tolist() == [127, 0, 1, 0]


def test_attention_of_equal_keys_is_the_mean():
    c = _cache(3, 1, 16, 4, "int8")
    K = np.ones((40, 1, 4), np.float32)
    V = np.arange(40, dtype=np.float32)[:, None, None] * np.ones((1, 1, 4), np.float32)
    ora.write(c, [[0, 1, 2]], [40], [0, 40], K, V)
    v = ora.dense(c, [0, 1, 2], "v", 0, 40)
    Q = np.random.default_rng(2).normal(size=(3, 2, 4))
    out, mean_abs, _ = ora.attention(c, [[0, 1, 2]], [40], [0, 3], Q, 0.5)
    for i in range(3):
        assert np.allclose(out[i], v[:38 + i].mean(0)) and np.allclose(out[i], mean_abs[i])
    out, _, _ = ora.attention(c, [[0, 1, 2]], [40], [0, 3], Q, 0.5, window=4)
    assert np.allclose(out[1], v[35:39].mean(0))
    out, _, _ = ora.attention(c, [[0, 1, 2]], [40], [0, 3], Q, 0.5, causal=False)
    assert np.allclose(out[0], v.mean(0))


def test_attention_against_torch():
    import torch
    rng = np.random.default_rng(3)
    c = _cache(3, 2, 16, 8, "fp8")
    K, V = (rng.normal(size=(30, 2, 8)).astype(np.float32) for _ in range(2))
    ora.write(c, [[1, 2]], [30], [0, 30], K, V)
    Q = rng.normal(size=(30, 4, 8))
    out, _, _ = ora.attention(c, [[1, 2]], [30], [0, 30], Q, 0.3)
    k, v = (torch.from_numpy(np.stack([ora.dense(c, [1, 2], n, h, 30) for h in (0, 0, 1, 1)]))
            for n in ("k", "v"))
    want = torch.nn.functional.scaled_dot_product_attention(
        torch.from_numpy(Q).transpose(0, 1), k, v, is_causal=True, scale=0.3)
    assert np.allclose(out, want.transpose(0, 1).numpy())


def test_token_logprobs_closed_forms():
    x = np.zeros((3, 8))
    x[1, 3] = np.log(8)                  # probabilities 8/15, 1/15 x 7
    x[2, :6] = -np.inf
    lp, h, ids, top = ora.token_logprobs(x, np.array([0, 3, 1]), 3)
    assert np.allclose(lp[:2], [-np.log(8), np.log(8 / 15)]) and lp[2] == -np.inf
    assert np.allclose(h, [np.log(8), 8 / 15 * np.log(15 / 8) + 7 / 15 * np.log(15), np.log(2)])
    assert ids.tolist() == [[0, 1, 2], [3, 0, 1], [6, 7, 0]]
    assert top[2, 2] == -np.inf and np.isclose(top[1, 0], np.log(8 / 15))
    lp, h, _, _ = ora.token_logprobs(np.full((1, 4), -np.inf), np.array([9]), 0)
    assert lp[0] == 0 and h[0] == 0
    lp, h, _, _ = ora.token_logprobs(np.full((1, 4), -3e38), np.array([2]), 0)
    assert np.isclose(lp[0], -np.log(4)) and np.isclose(h[0], np.log(4))
