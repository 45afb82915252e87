"""A refused call enqueues nothing: outputs, cache and batch hold what they held,
and the next call gives what it gave before. Rows of logits that hold no
distribution give no number, in each form of scoring."""

import numpy as np
import pytest

from serving_helpers import Setup

pytestmark = pytest.mark.gpu


def test_refused_calls_change_nothing(gpu):
    import torch
    r = gpu
    s = Setup(r, [(2, 40), (3, 3000)], 2, 64, 16, "int8", seed=3).fill().to_gpu()
    Q = torch.randn((5, 4, 64), device="cuda")
    K = torch.randn((5, 2, 64), device="cuda")
    logits = torch.randn((5, 40000), device="cuda")
    targets = torch.arange(5, device="cuda")
    w = r.attention_workspace(s.cache, s.batch, 4)
    wl = r.logprobs_workspace(logits, 4)
    assert w is not None and wl is not None
    want = [r.cache_attention(s.cache, s.batch, Q), *r.cache_read(s.cache, s.batch),
            *r.token_logprobs(logits, targets, 4)]
    out = torch.full((5, 4, 64), 55.0, device="cuda")
    pair = (torch.full((5, 2, 64), 55.0, device="cuda"), torch.full((5, 2, 64), 55.0, device="cuda"))
    held = [*s.cache.tensors, *s.batch.tensors, out, *pair, w.fill_(0x5A), wl.fill_(0x5A)]
    before = [t.clone() for t in held]
    shifted = torch.zeros(5 * 2 * 64 + 1, device="cuda")[1:].view(5, 2, 64)
    lost = r.RrqCache(*(getattr(s.cache.desc, n) for n, _ in r.RrqCache._fields_))
    lost.v_codes = None
    for error, call in (
            (ValueError, lambda: r.cache_attention(s.cache, s.batch, Q[:1], out=out)),
            (TypeError, lambda: r.cache_attention(s.cache, s.batch, Q.half(), out=out)),
            (TypeError, lambda: r.cache_attention(s.cache, s.batch, Q, out=out,
                                                  out_dtype=torch.bfloat16)),
            (ValueError, lambda: r.cache_attention(s.cache, s.batch, Q, out=out,
                                                   workspace=w.view(-1, 2)[:, 0])),
            (r.RRQError, lambda: r.cache_attention(s.cache, s.batch, Q, out=out,
                                                   workspace=w[:w.numel() - 16])),
            (r.RRQError, lambda: r.cache_attention(s.cache, s.batch, Q, out=out, workspace=w[1:])),
            (r.RRQError, lambda: r.cache_attention(s.cache, s.batch, Q[:, :3], out=out[:, :3]
                                                   .contiguous(), workspace=w)),
            (r.RRQError, lambda: r.cache_attention(s.cache, s.batch, Q, scale=float("inf"),
                                                   out=out, workspace=w)),
            (r.RRQError, lambda: r.cache_attention(s.cache, s.batch, Q, window=-1, out=out,
                                                   workspace=w)),
            (r.RRQError, lambda: r.rrq_cache_attention(lost, s.batch.desc, Q, 0, 256, 64, 4, 0.1,
                                                       1, 0, out, 0, w, w.numel())),
            (ValueError, lambda: r.cache_write(s.cache, s.batch, K, K[:, :1])),
            (TypeError, lambda: r.cache_write(s.cache, s.batch, K, K.bfloat16())),
            (r.RRQError, lambda: r.cache_write(s.cache, s.batch, shifted, K)),
            (r.RRQError, lambda: r.rrq_cache_write(lost, s.batch.desc, K, K, 0, 128, 64, 128, 64)),
            (ValueError, lambda: r.cache_read(s.cache, s.batch, out=(pair[0], pair[1][:1]))),
            (TypeError, lambda: r.cache_read(s.cache, s.batch, torch.bfloat16, out=pair)),
            (r.RRQError, lambda: r.rrq_cache_read(lost, s.batch.desc, *pair, 0)),
            (r.RRQError, lambda: r.token_logprobs(logits, targets, 33, workspace=wl)),
            (r.RRQError, lambda: r.token_logprobs(logits, targets, 4, workspace=wl[:-16])),
            (ValueError, lambda: r.token_logprobs(logits, targets[:4], 4, workspace=wl)),
            (ValueError, lambda: r.token_logprobs(logits, targets.int(), 4, workspace=wl))):
        with pytest.raises(error):
            call()
    torch.cuda.synchronize()
    # (bits: the unused slots of the cache hold NaN scales)
    for a, b in zip(held, before):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
    got = [r.cache_attention(s.cache, s.batch, Q), *r.cache_read(s.cache, s.batch),
           *r.token_logprobs(logits, targets, 4)]
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 5000, 8100, 40000])
def test_rows_without_a_distribution(gpu, dtype, vocab):
    """One wave a row, four, and segments; a NaN or +inf at a row's start,
    middle and end, among numbers and among -inf only."""
    import torch
    rng = np.random.default_rng(vocab)
    rows = []
    for at in (0, vocab // 2, vocab - 1):
        for value in (np.nan, np.inf):
            for rest in ("numbers", "nothing"):
                x = rng.normal(size=vocab).astype(np.float32)
                if rest == "nothing":
                    x[:] = -np.inf
                x[at] = value
                rows.append(x)
    rows.append(np.full(vocab, np.nan, np.float32))
    both = np.full(vocab, -np.inf, np.float32)
    both[1], both[vocab - 2] = np.inf, np.nan
    rows.append(both)
    rows.append(rng.normal(size=vocab).astype(np.float32))       # an ordinary one
    x = torch.from_numpy(np.stack(rows)).cuda()
    x = x.bfloat16() if dtype == "bf16" else x
    n = len(rows)
    for target in (0, vocab // 2, vocab - 1):
        lp, h, ids, top = (t.cpu().numpy() for t in gpu.token_logprobs(
            x, torch.full((n,), target, dtype=torch.int64, device="cuda"), 3))
        assert np.isnan(lp[:-1]).all() and np.isnan(h[:-1]).all() and np.isnan(top[:-1]).all()
        assert np.isfinite(lp[-1]) and np.isfinite(h[-1]) and np.isfinite(top[-1]).all()
        # alternatives by logit all the same; a NaN comes last
        for i, row in enumerate(x.float().cpu().numpy()):
            numbers, none = np.flatnonzero(~np.isnan(row)), np.flatnonzero(np.isnan(row))
            order = numbers[np.argsort(-row[numbers], kind="stable")]
            assert ids[i].tolist() == [*order, *none][:3], i
    lp = gpu.token_logprobs(x, torch.full((n,), -1, dtype=torch.int64, device="cuda"))[0]
    assert (lp == 0).all()
