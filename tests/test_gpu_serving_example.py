"""The example decoder: every call it makes of the cache, attention and token
scoring, on the values it makes them with, against the oracle within the
bounds of those operators' own tests."""

import importlib.util
import math
import os

import numpy as np
import pytest

from conftest import ROOT
from oracle import serving as ora
from test_gpu_attention import _bound
from test_gpu_logprobs import _check as check_logprobs

pytestmark = pytest.mark.gpu


@pytest.fixture
def example(gpu):
    spec = importlib.util.spec_from_file_location(
        "serve_prefixes", os.path.join(ROOT, "examples", "serve_prefixes.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _host(cache):
    return ora.Cache(*(t.cpu().numpy().copy() for t in (cache.k_codes, cache.v_codes,
                                                        cache.k_scales, cache.v_scales)),
                     cache.code_type)


class _Rows:        # what _bound reads of a setup
    def __init__(self, lengths):
        self.lengths = lengths


@pytest.mark.parametrize("code", ["int8", "fp8"])
def test_every_call_of_the_example(gpu, example, monkeypatch, code):
    import torch
    write, attend, logprobs = gpu.cache_write, gpu.cache_attention, gpu.token_logprobs
    calls = {"write": 0, "attend": 0, "logprobs": 0}

    def index(batch):
        return [t.cpu().numpy() for t in (batch.page_table, batch.lengths, batch.offsets)]

    def checked_write(cache, batch, K, V):
        host = _host(cache)
        write(cache, batch, K, V)
        ora.write(host, *index(batch), K.cpu().numpy(), V.cpu().numpy())
        got = _host(cache)
        with np.errstate(invalid="ignore"):
            assert np.array_equal(got.k, host.k) and np.array_equal(got.v, host.v)
        assert np.array_equal(got.ks.view(np.uint32), host.ks.view(np.uint32))
        assert np.array_equal(got.vs.view(np.uint32), host.vs.view(np.uint32))
        calls["write"] += 1

    def checked_attend(cache, batch, Q):
        out = attend(cache, batch, Q)
        table, lengths, offsets = index(batch)
        q, scale = Q.cpu().numpy(), Q.shape[2] ** -0.5
        want, mean_abs, reach = ora.attention(_host(cache), table, lengths, offsets, q, scale,
                                              True, 0)
        bound = _bound(_Rows(lengths), q, want, mean_abs, reach, scale, True, True)
        assert (np.abs(out.float().cpu().numpy() - want) <= bound).all()
        calls["attend"] += 1
        return out

    def checked_logprobs(logits, targets=None, n_top=0):
        x = logits.cpu().numpy()
        given = np.full(len(x), -1) if targets is None else targets.cpu().numpy()
        monkeypatch.setattr(gpu, "token_logprobs", logprobs)
        check_logprobs(gpu, x, given, n_top)
        monkeypatch.setattr(gpu, "token_logprobs", checked_logprobs)
        calls["logprobs"] += 1
        return logprobs(logits, targets, n_top)

    for name, f in (("cache_write", checked_write), ("cache_attention", checked_attend),
                    ("token_logprobs", checked_logprobs)):
        monkeypatch.setattr(gpu, name, f, raising=False)
    decoder = example.Decoder(vocab=640, hidden=256, layers=2, heads=6, kv_heads=2, dim=64,
                              inner=256, page=16, code_type=code)
    rng = np.random.default_rng(5)
    prompts = [rng.integers(0, 640, n).tolist() for n in (1, 37, 16, 70)]
    texts, drawn, (ids, top) = example.generate(decoder, prompts, 4, 4, chunk=32)
    assert [len(t) for t in texts] == [5, 41, 20, 74] and drawn.shape == (4, 4)
    assert all(t[:len(p)] == p for t, p in zip(texts, prompts))
    assert ids.shape == (4, 5) and (drawn <= 0).all()
    for k in (1, 4):
        means, entropy = example.score(decoder, texts, k)
        assert len(means) == 4 and all(m < 0 for m in means)
        assert 0 < entropy <= math.log(640) + 1e-6
    assert calls == {"write": 2 * (3 + 3 + 2), "attend": 2 * (3 + 3 + 2), "logprobs": 4 + 2}


def test_the_example_repeats_itself(gpu, example):
    import torch
    decoder = example.Decoder(vocab=640, hidden=256, layers=1, heads=6, kv_heads=2, dim=128,
                              inner=256, page=32, code_type="fp8")
    prompts = [[3, 1, 4], [5] * 50]
    a = example.generate(decoder, prompts, 3, 2)
    b = example.generate(decoder, prompts, 3, 2)
    assert a[0] == b[0] and torch.equal(a[1], b[1])
    assert example.score(decoder, a[0], 3) == example.score(decoder, a[0], 3)
