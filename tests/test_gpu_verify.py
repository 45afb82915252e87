"""rrq_verify_drafts on the GPU against its definition in 64 bits: whole numbers, equal.

Inputs whose decisions come nearer than 1e-6 to their borders would be no test of
equality (a row's sum is good to about 2^-24 behind an acceptance, to 10^-12 behind a
drawn token); `check` asserts that there are none."""

import numpy as np
import pytest

from oracle import drafting as ora

pytestmark = pytest.mark.gpu


def _trees(rng, counts, tree):
    parents = []
    for n in counts:
        for j in range(n):
            parents.append(-1 if j == 0 else int(rng.integers(max(0, j // 3 - 1), j)) if tree
                           else j - 1)
    return parents


def make(counts, vocab, dtype="f32", draft=False, tree=False, max_accept=None, seed=0, sharp=3.0,
         likely=0.6, pad=0):
    """Inputs on the host: logits, drafts of which a share is likely, numbers."""
    rng = np.random.default_rng(seed)
    R, B = sum(counts), len(counts)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(int)
    deepest = max(counts) - 1 if max_accept is None else max_accept

    def rounded(x):
        x = x.astype(np.float32)
        if dtype == "bf16":
            b = x.view(np.uint32).astype(np.uint64)
            x = ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
        return x

    logits = rounded(rng.normal(size=(R, vocab)) * sharp)
    parents = _trees(rng, counts, tree)
    tokens = rng.integers(0, vocab, R)
    q = rounded(rng.normal(size=(B, max(deepest, 0), vocab)) * sharp) if draft else None
    for b in range(B):
        for j in range(1, counts[b]):
            row = offsets[b] + j
            x = logits[offsets[b] + max(parents[row], 0)]
            if rng.random() < likely:
                order = np.argsort(-x)
                tokens[row] = order[min(vocab - 1, int(rng.integers(0, 4)))]
            if draft and j <= deepest:
                q[b, j - 1] = rounded(x + rng.normal(size=vocab) * 0.7)
    return dict(logits=logits, tokens=tokens, offsets=offsets, max_accept=deepest,
                uniforms=rng.random(R).astype(np.float32), draft=q,
                parents=np.array(parents, np.int32) if tree else None), dtype, pad


def upload(case):
    import torch
    a, dtype, pad = case
    dt = torch.float32 if dtype == "f32" else torch.bfloat16

    def matrix(x):
        wide = torch.full((*x.shape[:-1], x.shape[-1] + pad), float("nan"), device="cuda",
                          dtype=dt)
        wide[..., pad // 2:pad // 2 + x.shape[-1]] = torch.from_numpy(x).cuda().to(dt)
        return wide[..., pad // 2:pad // 2 + x.shape[-1]]

    return dict(logits=matrix(a["logits"]), tokens=torch.from_numpy(a["tokens"]).cuda(),
                offsets=torch.tensor(a["offsets"], dtype=torch.int32, device="cuda"),
                max_accept=a["max_accept"], uniforms=torch.from_numpy(a["uniforms"]).cuda(),
                draft=None if a["draft"] is None else matrix(a["draft"]),
                parents=None if a["parents"] is None else torch.from_numpy(a["parents"]).cuda())


def check(rrq, case, temperature=1.0, draft_temperature=1.0, near=1e-6, **kw):
    args = upload(case)
    got = rrq.verify_drafts(**args, temperature=temperature, draft_temperature=draft_temperature,
                            **kw)
    *want, margin = ora.verify(**case[0], temperature=temperature,
                               draft_temperature=draft_temperature)
    assert margin > near, margin
    for g, w, name in zip(got, want, ("counts", "following", "paths")):
        g = g.cpu().numpy()
        bad = np.argwhere(g != w)
        assert bad.size == 0, f"{name}: {len(bad)} differ, first {bad[0]}: {g[tuple(bad[0])]} " \
                              f"for {w[tuple(bad[0])]}"
    return got


VOCABS = [1, 2, 3, 7, 8, 100, 1000, 4095, 4096, 4097, 8191, 8193, 20011, 131072, 150001]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("kind", ["chain", "draft", "tree"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_vocabularies(gpu, vocab, kind, dtype):
    counts = [6, 1, 3, 4] if vocab > 20000 else [6, 1, 0, 3, 9, 2, 5, 7]
    check(gpu, make(counts, vocab, dtype, kind == "draft", kind == "tree", seed=vocab))


@pytest.mark.parametrize("temperature,draft_temperature", [(0.7, 1.0), (1.3, 0.8), (0.05, 3.0),
                                                           (50.0, 50.0), (1e-6, 1e-6)])
@pytest.mark.parametrize("kind", ["chain", "draft", "tree"])
def test_temperatures(gpu, temperature, draft_temperature, kind):
    check(gpu, make([5] * 20, 3001, "f32", kind == "draft", kind == "tree", seed=3), temperature,
          draft_temperature)


@pytest.mark.parametrize("kind", ["chain", "draft", "tree"])
@pytest.mark.parametrize("vocab", [1, 5, 1000, 9000, 70001])
def test_greedy(gpu, kind, vocab):
    case = make([6, 1, 3, 12, 0, 7], vocab, "bf16", kind == "draft", kind == "tree", seed=5,
                likely=0.95, sharp=0.3)     # (many equal logits)
    check(gpu, case, 0.0)


@pytest.mark.parametrize("counts", [[65], [64, 63, 1], [130, 200, 66], [1, 0, 300]])
@pytest.mark.parametrize("kind", ["chain", "draft", "tree"])
def test_many_rows(gpu, counts, kind):
    """Walks over more rows than a wave has lanes."""
    check(gpu, make(counts, 50, "f32", kind == "draft", kind == "tree", seed=len(counts),
                    likely=0.98, sharp=6.0))


def test_long_walks(gpu):
    """Sure tokens: walks go on past 64 rows, accepted in later rounds."""
    a, dtype, pad = make([200, 150], 40, seed=6, sharp=0.1)
    offsets = a["offsets"]
    for b in range(2):
        for j in range(1, [200, 150][b]):
            a["logits"][offsets[b] + j - 1, a["tokens"][offsets[b] + j]] = 30.0
    counts, _, _ = check(gpu, (a, dtype, pad))
    assert counts.tolist() == [199, 149]


@pytest.mark.parametrize("max_accept", [0, 1, 2, 5])
@pytest.mark.parametrize("kind", ["chain", "draft", "tree"])
def test_a_walk_ends_at_its_limit(gpu, max_accept, kind):
    check(gpu, make([7, 1, 4, 7, 7, 7], 30, "f32", kind == "draft", kind == "tree",
                    max_accept=max_accept, seed=8, likely=1.0, sharp=8.0))


def test_longer_paths_than_drafts(gpu):
    check(gpu, make([4, 2], 30, max_accept=9, seed=9))
    check(gpu, make([4, 2], 30, draft=True, max_accept=9, seed=9))


def test_siblings(gpu):
    """Star trees: rejected tokens are taken out, equal ones once."""
    a, dtype, pad = make([40, 90, 3], 12, tree=True, seed=10, sharp=1.0)
    a["parents"][:] = np.where(a["parents"] < 0, -1, 0)
    a["tokens"][:] = np.arange(len(a["tokens"])) % 5
    a["uniforms"][1:40] = 0.99
    a["uniforms"][41:130] = 0.995
    check(gpu, (a, dtype, pad))


def test_siblings_far_apart(gpu):
    """A token that was rejected more than 64 rows earlier."""
    a, dtype, pad = make([150], 6, tree=True, seed=11, sharp=0.5)
    a["parents"][1:] = 1                    # no one's children but row 1's, never reached
    a["parents"][[1, 100, 140]] = 0
    a["tokens"][[1, 100, 140]] = [3, 3, 2]
    a["uniforms"][[0, 1, 100, 140]] = [0.4, 0.97, 0.0, 0.99]
    counts, following, _ = check(gpu, (a, dtype, pad))
    assert counts.item() == 0 and following.item() not in (3, 2)


def test_parents_that_do_not_count(gpu):
    """Parents behind their row, below -1 or past the sequence: no one's children."""
    a, dtype, pad = make([8, 8], 20, tree=True, seed=12, likely=1.0, sharp=6.0)
    a["parents"][[2, 3, 5, 9, 12]] = [2, 7, -5, 100, 1 << 30]
    check(gpu, (a, dtype, pad))


def test_tokens_outside_the_vocabulary(gpu):
    for draft in (False, True):
        a, dtype, pad = make([5, 5, 5], 20, draft=draft, seed=13, likely=1.0, sharp=6.0)
        a["tokens"][[1, 7, 11]] = [-1, 20, 1 << 40]
        check(gpu, (a, dtype, pad))


@pytest.mark.parametrize("pad", [1, 3, 6])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_rows(gpu, pad, dtype):
    check(gpu, make([5, 2, 6], 8200, dtype, draft=True, seed=14, pad=pad))


def test_numbers_at_the_ends(gpu):
    """u = 0 and the largest below 1, and masked tokens at both ends."""
    top = np.float32(1) - np.float32(2) ** -24
    for u in (np.float32(0), top):
        for draft in (False, True):
            a, dtype, pad = make([3] * 8, 5000, draft=draft, seed=15)
            a["logits"][:, :3] = -np.inf
            a["logits"][:, -700:] = -np.inf
            if draft:
                a["draft"][:, :, :3] = -np.inf
                a["draft"][:, :, -700:] = -np.inf
            a["uniforms"][::3] = u
            check(gpu, (a, dtype, pad), near=0 if u else 1e-6)
    # a number that is no number below 1 draws the last token that may be drawn
    a["uniforms"][::3] = 1.0
    a["tokens"][:] = -1
    a["draft"] = None
    _, following, _ = gpu.verify_drafts(**upload((a, dtype, pad)))
    assert (following == 4299).all()


def test_rows_without_a_distribution(gpu):
    a, dtype, pad = make([3] * 6, 9000, seed=16, likely=1.0, sharp=9.0)
    a["uniforms"][1::3] = 0.0
    a["logits"][0] = -np.inf
    a["logits"][3, 8999] = np.nan
    a["logits"][6, 17] = np.inf
    a["logits"][10] = -np.inf               # a later row
    a["logits"][12, :] = np.nan
    a["logits"][15, 1:] = -np.inf           # one token has it all
    a["tokens"][16] = 0
    counts, following, _ = check(gpu, (a, dtype, pad))
    assert counts[[0, 1, 2, 4]].tolist() == [0] * 4 and counts[5] >= 1
    assert following[[0, 1, 2, 4]].tolist() == [-1] * 4
    # the draft's rows
    a, dtype, pad = make([3] * 5, 9000, draft=True, seed=17)
    a["uniforms"][:] = 0.5
    a["draft"][0, 0] = -np.inf
    a["draft"][1, 0, 5] = np.nan
    a["draft"][2, 0, 6] = np.inf
    check(gpu, (a, dtype, pad))
    # greedy: numbers beside others that are none
    a, dtype, pad = make([3] * 6, 9000, seed=16)
    a["logits"][0] = -np.inf
    a["logits"][3, ::2] = np.nan
    a["logits"][6, 17] = np.inf
    a["logits"][12, :] = np.nan
    check(gpu, (a, dtype, pad), 0.0)


def test_a_draft_equal_to_the_target(gpu):
    """Every draft is accepted whatever the number; one of probability 0 is not, and then
    nothing is left of p - q: p itself is drawn from."""
    a, dtype, pad = make([4] * 10, 5000, draft=True, seed=18)
    for b in range(10):
        a["draft"][b] = a["logits"][4 * b:4 * b + 3]
        for j in range(1, 4):
            a["tokens"][4 * b + j] = int(np.argmax(a["logits"][4 * b + j - 1]))
    a["uniforms"][:] = np.minimum(a["uniforms"], 0.999)
    counts, _, _ = check(gpu, (a, dtype, pad))
    assert (counts == 3).all()
    a["logits"][::4, 9] = -np.inf
    a["draft"][:, 0, 9] = -np.inf
    a["tokens"][1::4] = 9
    counts, following, _ = check(gpu, (a, dtype, pad))
    assert (counts == 0).all() and (following >= 0).all()


def test_large_logits(gpu):
    for gain in (1e4, 1e30, 3e37):
        a, dtype, pad = make([4] * 5, 3000, draft=True, seed=19)
        with np.errstate(over="ignore"):        # (the last: some rows hold infinities)
            a["logits"] *= np.float32(gain)
            a["draft"] *= np.float32(gain)
        check(gpu, (a, dtype, pad))
        check(gpu, (a, dtype, pad), gain / 4, gain / 4) if gain < 1e18 else None


@pytest.mark.parametrize("kind", ["chain", "draft", "tree"])
def test_tokens_come_with_the_targets_probabilities(gpu, kind):
    """First tokens of 40000 sequences, accepted or drawn instead, are distributed as the
    target's: within 5 standard deviations of each count."""
    import torch
    B, V = 40000, 6
    rng = np.random.default_rng(20)
    x = rng.normal(size=V) * 1.5
    y = x + rng.normal(size=V)
    p, q = np.exp(x) / np.exp(x).sum(), np.exp(y) / np.exp(y).sum()
    n = 4 if kind == "tree" else 2
    tokens = np.zeros((B, n), np.int64)
    tokens[:, 1] = rng.choice(V, size=B, p=q)
    if kind == "tree":
        tokens[:, 2:] = rng.integers(0, V, (B, 2))
    args = dict(logits=torch.tensor(np.tile(x, (B * n, 1)), dtype=torch.float32, device="cuda"),
                tokens=torch.from_numpy(tokens.reshape(-1)).cuda(),
                offsets=torch.arange(0, B * n + 1, n, dtype=torch.int32, device="cuda"),
                max_accept=1, uniforms=torch.from_numpy(rng.random(B * n).astype(np.float32)).cuda())
    if kind == "draft":
        args["draft"] = torch.tensor(np.tile(y, (B, 1, 1)), dtype=torch.float32, device="cuda")
    if kind == "tree":
        args["parents"] = torch.tensor([-1, 0, 0, 0] * B, dtype=torch.int32, device="cuda")
    counts, following, paths = (t.cpu().numpy() for t in gpu.verify_drafts(**args))
    first = np.where(counts > 0, tokens[np.arange(B), paths[:, 1]], following)
    seen = np.bincount(first, minlength=V)
    assert (np.abs(seen - B * p) < 5 * np.sqrt(B * p * (1 - p))).all(), (seen, B * p)
    assert 0 < counts.mean() < 1


def test_rows_behind_the_last_sequence_and_no_sequences(gpu):
    import torch
    case = make([4, 3], 500, draft=True, seed=21)
    want = gpu.verify_drafts(**upload(case))
    args = upload(case)
    args["logits"] = torch.cat([args["logits"], torch.full((3, 500), float("nan"),
                                                           device="cuda")])
    args["tokens"] = torch.cat([args["tokens"], torch.zeros(3, dtype=torch.int64, device="cuda")])
    args["uniforms"] = torch.cat([args["uniforms"], torch.zeros(3, device="cuda")])
    got = gpu.verify_drafts(**args)
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    args.update(offsets=args["offsets"][:1], draft=None)
    counts, following, paths = gpu.verify_drafts(**args)
    assert counts.shape == (0,) and following.shape == (0,) and paths.shape == (0, 4)
    args.update(logits=args["logits"][:0], tokens=args["tokens"][:0],
                uniforms=args["uniforms"][:0],
                offsets=torch.zeros(3, dtype=torch.int32, device="cuda"))
    counts, following, paths = gpu.verify_drafts(**args)
    assert counts.tolist() == [0, 0] and following.tolist() == [-1, -1] and (paths == -1).all()


def test_rows_past_32_bits(gpu):
    """Logits of more than 2^32 bytes."""
    import torch
    V = 131072
    rows = (1 << 32) // (2 * V) + 6
    logits = torch.zeros((rows, V), dtype=torch.bfloat16, device="cuda")
    tokens = torch.full((rows,), 7, dtype=torch.int64, device="cuda")
    logits[-6:, 7] = 30.0
    logits[-1, 7] = 0.0
    logits[-1, 99] = 30.0
    offsets = torch.tensor([0, rows - 6, rows], dtype=torch.int32, device="cuda")
    u = torch.full((rows,), 0.5, device="cuda")
    counts, following, paths = gpu.verify_drafts(logits, tokens, offsets, 5, u)
    assert counts.tolist()[1] == 5 and following.tolist()[1] == 99
    assert paths[1].tolist() == [0, 1, 2, 3, 4, 5]


def test_stream_graph_and_workspace(gpu):
    """On another stream; captured with its own workspace, and replayed on other logits."""
    import torch
    case = make([5, 3, 6, 1], 20000, draft=True, seed=22)
    args = upload(case)
    want = gpu.verify_drafts(**args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = gpu.verify_drafts(**args, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    w = gpu.verify_workspace(args["logits"], 4, args["draft"])
    w.fill_(255)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = gpu.verify_drafts(**args, workspace=w)
    for i in range(4):
        args["logits"].mul_(0.8)
        args["uniforms"].copy_(args["uniforms"].roll(1))
        graph.replay()
        want = gpu.verify_drafts(**args)
        assert all(torch.equal(g, x) for g, x in zip(got, want))
        torch.cuda.synchronize()


def test_refusals(gpu):
    import torch
    args = upload(make([3, 2], 40, draft=True, seed=23))

    def refused(error, match, **kw):
        with pytest.raises(error, match=match):
            gpu.verify_drafts(**{**args, **kw})

    refused(TypeError, "logits", logits=[1.0])
    refused(ValueError, "GPU", logits=args["logits"].cpu())
    refused(TypeError, "logits must be", logits=args["logits"].half())
    refused(ValueError, "logits must be", logits=args["logits"][0])
    refused(ValueError, "last dimension", logits=args["logits"].t().contiguous().t())
    refused(ValueError, "tokens", tokens=args["tokens"][:4])
    refused(ValueError, "tokens", tokens=args["tokens"].int())
    refused(TypeError, "tokens and uniforms", tokens=None)
    refused(ValueError, "uniforms", uniforms=args["uniforms"].double())
    refused(ValueError, "offsets", offsets=args["offsets"].long())
    refused(ValueError, "offsets", offsets=args["offsets"].cpu())
    refused(ValueError, "offsets", offsets=args["offsets"][:0])
    refused(ValueError, "chain", parents=torch.zeros(5, dtype=torch.int32, device="cuda"))
    refused(ValueError, "parents", draft=None,
            parents=torch.zeros(4, dtype=torch.int32, device="cuda"))
    refused(ValueError, "draft must be", draft=args["draft"][:, :1])
    refused(TypeError, "draft must have", draft=args["draft"].bfloat16())
    refused(ValueError, "draft must be on", draft=args["draft"].cpu())
    refused(ValueError, "max_accept", max_accept=-1)
    refused(gpu.RRQError, "status", temperature=-1.0)
    refused(gpu.RRQError, "status", temperature=float("nan"))
    refused(gpu.RRQError, "status", temperature=1e-30)
    refused(gpu.RRQError, "status", draft_temperature=0.0)
    refused(gpu.RRQError, "status", logits=args["logits"][:1].expand(5, 40))
    refused(ValueError, "workspace", workspace=torch.zeros(16, device="cuda"))
    refused(gpu.RRQError, "workspace", workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
