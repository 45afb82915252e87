"""The drafting example's pages hold every text, however unevenly drafts are accepted."""

import importlib.util
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("widths", [(1, 1, 1), (2, 1)])
def test_texts_stay_within_their_pages(gpu, monkeypatch, widths):
    """One text never gains more than a token a step, the other all drafts: it grows to
    several times the asked length before the first one is done."""
    spec = importlib.util.spec_from_file_location(
        "draft_prefixes", os.path.join(ROOT, "examples", "draft_prefixes.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    verify = gpu.verify_drafts

    def uneven(logits, tokens, offsets, most, uniforms, draft, parents, t, td):
        n = offsets[1].item()
        logits = logits.clone()
        tokens = tokens.clone()
        tokens[1:n] = -1                                # the first text: all rejected
        for j in range(1, n):                           # the second: all accepted
            at = n + (j - 1 if parents is None else parents[n + j].item())
            logits[at] = float("-inf")
            logits[at, tokens[n + j]] = 0.0
        return verify(logits, tokens, offsets, most, uniforms, None, parents, t, td)

    longest = []
    attend = gpu.tree_attention

    def watched(cache, batch, *args, **kw):
        longest.append((int(batch.lengths.max()), batch.page_table.shape[1] * cache.page_size))
        return attend(cache, batch, *args, **kw)

    monkeypatch.setattr(gpu, "verify_drafts", uneven, raising=False)
    monkeypatch.setattr(gpu, "tree_attention", watched, raising=False)
    decoder = example.Decoder(vocab=64, hidden=128, layers=1, heads=2, kv_heads=1, dim=64,
                              inner=128, page=16)
    texts, _, steps = example.generate(decoder, [[1, 2, 3], [4, 5]], 20, 3, 4, widths, 1.0)
    assert steps == 20 and len(texts[0]) == 23
    assert len(texts[1]) == 2 + 20 * (len(widths) + 1)
    assert all(length <= room for length, room in longest), max(longest)
