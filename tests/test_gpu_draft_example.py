"""The drafting example: every call it makes, on the values it makes them with,
against the oracle within the bounds of those operators' own tests."""

import importlib.util
import os

import numpy as np
import pytest

from conftest import ROOT
from oracle import drafting as dra
from oracle import serving as ora
from test_gpu_attention import _bound

pytestmark = pytest.mark.gpu


@pytest.fixture
def example(gpu):
    spec = importlib.util.spec_from_file_location(
        "draft_prefixes", os.path.join(ROOT, "examples", "draft_prefixes.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _host(cache):
    return ora.Cache(*(t.cpu().numpy().copy() for t in cache.tensors), cache.code_type)


def _np(t):
    return None if t is None else t.float().cpu().numpy()


def _index(batch):
    return [t.cpu().numpy() for t in (batch.page_table, batch.lengths, batch.offsets)]


class _Rows:        # what _bound reads of a setup
    def __init__(self, lengths):
        self.lengths = lengths


@pytest.mark.parametrize("widths,temperature,code,layout", [
    ((1, 1, 1), 0.8, "int8", "half"), ((3, 2, 1), 0.8, "fp8", "interleaved"),
    ((2, 2), 0.0, "int8", "interleaved"), ((1, 1), 0.0, "fp8", "half")])
def test_every_call_of_the_example(gpu, example, monkeypatch, widths, temperature, code, layout):
    import torch
    norm, append, attend, verify = (gpu.block_norm, gpu.cache_append, gpu.tree_attention,
                                    gpu.verify_drafts)
    calls = {"norm": 0, "append": 0, "attend": 0, "verify": 0, "near": 0}

    def checked_norm(residual, y=None, weight=None):
        out, h = norm(residual, y, weight)
        host = (_np(residual), _np(y), _np(weight), None, "rms", None, None, None, 1.0,
                np.float64(np.float32(1e-6)))
        want, want_h = dra.block_norm(*host)
        err, err_h = dra.block_norm_error(*host)
        assert (np.abs(_np(out) - want) <= err + 2.0 ** -8 * (np.abs(want) + err)).all()
        assert (np.abs(_np(h) - want_h) <= err_h + 2.0 ** -24 * (np.abs(want_h) + err_h)).all()
        calls["norm"] += 1
        return out, h

    def checked_append(cache, batch, rotary, Q, K, V, positions=None):
        host = _host(cache)
        out = append(cache, batch, rotary, Q, K, V, positions)
        want = dra.append(host, *_index(batch),
                          None if positions is None else positions.cpu().numpy(),
                          rotary.frequencies.cpu().numpy(), rotary.layout, rotary.amplitude,
                          _np(Q), _np(K), _np(V))
        got = _host(cache)
        assert np.array_equal(got.k, host.k) and np.array_equal(got.v, host.v)
        assert np.array_equal(got.ks.view(np.uint32), host.ks.view(np.uint32))
        assert np.array_equal(got.vs.view(np.uint32), host.vs.view(np.uint32))
        assert np.array_equal(_np(out), want)
        calls["append"] += 1
        return out

    def checked_attend(cache, batch, Q, seen, positions):
        out = attend(cache, batch, Q, seen, positions)
        table, lengths, offsets = _index(batch)
        q, scale = _np(Q), Q.shape[2] ** -0.5
        sets = [{j for j in range(64) if w >> j & 1} for w in seen[:, 0].tolist()]
        want, mean_abs, reach = dra.tree_attention(_host(cache), table, lengths, offsets, q, sets,
                                                   positions.cpu().numpy(), scale)
        bound = _bound(_Rows(lengths), q, want, mean_abs, reach, scale, True, True)
        assert (np.abs(_np(out) - want) <= bound).all()
        calls["attend"] += 1
        return out

    def checked_verify(logits, tokens, offsets, most, uniforms, draft, parents, t, td):
        got = verify(logits, tokens, offsets, most, uniforms, draft, parents, t, td)
        *want, margin = dra.verify(_np(logits), tokens.cpu().numpy(), offsets.cpu().numpy(), most,
                                   _np(uniforms), _np(draft),
                                   None if parents is None else parents.cpu().numpy(), t, td)
        if margin > 1e-6:
            assert all(np.array_equal(g.cpu().numpy(), w) for g, w in zip(got, want))
        else:
            calls["near"] += 1
        calls["verify"] += 1
        return got

    for name, f in (("block_norm", checked_norm), ("cache_append", checked_append),
                    ("tree_attention", checked_attend), ("verify_drafts", checked_verify)):
        monkeypatch.setattr(gpu, name, f, raising=False)
    decoder = example.Decoder(vocab=640, hidden=256, layers=2, heads=6, kv_heads=2, dim=64,
                              inner=256, page=16, code_type=code, layout=layout)
    rng = np.random.default_rng(5)
    prompts = [rng.integers(0, 640, n).tolist() for n in (1, 37, 16, 70)]
    texts, accepted, steps = example.generate(decoder, prompts, 6, 3, 4, widths, temperature)
    assert all(t[:len(p)] == p and len(t) >= len(p) + 6 for t, p in zip(texts, prompts))
    assert all(0 <= t < 640 for text in texts for t in text)
    assert sum(map(len, texts)) - sum(map(len, prompts)) == accepted + 4 * steps
    assert calls["verify"] == steps and calls["near"] <= 1
    # the drafts' levels and the target, of both layers; prompts besides
    assert calls["attend"] == 2 * (len(widths) + 2) * steps
    kept = 0 if max(widths) == 1 else 2 * 2 * steps
    assert calls["append"] == calls["attend"] + kept + 2 * 2
    assert calls["norm"] == 5 * (calls["attend"] // 2 + 2)
    assert torch.cuda.is_available()


@pytest.mark.parametrize("widths", [(1, 1, 1, 1), (2, 2, 1)])
def test_drafts_of_the_target_itself_are_accepted(gpu, example, widths):
    """Drafting at the verifying prefix: a greedy chain's drafts are the target's own
    choices, and so is a path through the tree, up to logits that two batches' sums
    leave in another order."""
    decoder = example.Decoder(vocab=640, hidden=256, layers=2, heads=6, kv_heads=2, dim=64,
                              inner=256, page=16)
    prompts = [[3, 1, 4], [5] * 50, list(range(100))]
    texts, accepted, steps = example.generate(decoder, prompts, 20, 4, 4, widths, 0.0)
    assert accepted >= 0.8 * steps * len(prompts) * len(widths)
    again = example.generate(decoder, prompts, 20, 4, 4, widths, 0.0)
    assert again == (texts, accepted, steps)
