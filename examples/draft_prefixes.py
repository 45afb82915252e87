"""Drafting with a short prefix of a package and checking with a longer one.

The decoder of serve_prefixes.py, whose packages hold 2 to 8 bit weights, drafts
tokens at a short prefix (a chain, drawn from its distributions, or a tree of its
likeliest tokens) and verifies them at a longer one in a single step over all of
them: what is accepted is distributed as the longer prefix alone would draw it.
Weights are random (there is no checkpoint here), so the text means nothing; the
calls are those of a real decoder.

    python examples/draft_prefixes.py
"""

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_04048_amd as rrq  # noqa: E402
from examples.serve_prefixes import Linear  # noqa: E402


class Decoder:
    """Pre-norm decoder layers with grouped heads, rotary positions and a gated
    feed-forward; norms, rotation and residuals in the library's calls."""

    def __init__(self, vocab=4096, hidden=1024, layers=2, heads=16, kv_heads=4, dim=64,
                 inner=2048, page=64, code_type="int8", layout="half", seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.page = heads, kv_heads, dim, page
        self.code_type = code_type
        self.embed = torch.randn((vocab, hidden), device="cuda", generator=g)
        self.layers = [{"qkv": Linear((heads + 2 * kv_heads) * dim, hidden, g),
                        "out": Linear(hidden, heads * dim, g),
                        "up": Linear(2 * inner, hidden, g),
                        "down": Linear(hidden, inner, g)} for _ in range(layers)]
        # of each block, and of the head
        self.norms = [1 + 0.1 * torch.randn(hidden, device="cuda", generator=g)
                      for _ in range(2 * layers + 1)]
        self.head = Linear(vocab, hidden, g)
        self.rotary = rrq.Rotary(rrq.rotary_frequencies(dim), layout)

    def caches(self, n_pages):
        return [rrq.KVCache.empty(n_pages, self.kv_heads, self.dim, self.page, self.code_type)
                for _ in self.layers]

    def parts(self, qkv):
        """Queries, keys and values of a fused projection's rows."""
        n, m = self.heads, self.heads + self.kv_heads
        return qkv[:, :n], qkv[:, n:m], qkv[:, m:]

    def step(self, caches, batch, tokens, k, positions=None, seen=None):
        """(logits of the batch's new tokens, each layer's fused projection). With
        `seen` the tokens are drafted ones."""
        h = self.embed[tokens]
        x, h = rrq.block_norm(h, weight=self.norms[0])
        fused = []
        for i, (w, cache) in enumerate(zip(self.layers, caches)):
            qkv = w["qkv"](x, k).view(len(tokens), -1, self.dim)
            fused.append(qkv)
            Q = rrq.cache_append(cache, batch, self.rotary, *self.parts(qkv), positions)
            if seen is None:
                a = rrq.cache_attention(cache, batch, Q)
            else:
                a = rrq.tree_attention(cache, batch, Q, seen, positions)
            x, h = rrq.block_norm(h, w["out"](a.view(len(tokens), -1), k), self.norms[2 * i + 1])
            gate, up = w["up"](x, k).chunk(2, -1)
            y = w["down"](torch.nn.functional.silu(gate) * up, k)
            x, h = rrq.block_norm(h, y, self.norms[2 * i + 2])
        return self.head(x, k), fused


class Texts:
    """Sequences and their pages, at one prefix. The last token of a text is not in
    the cache yet: it is the first row of its next step."""

    def __init__(self, decoder, k, n_seqs, max_tokens):
        self.decoder, self.k = decoder, k
        per = -(-max_tokens // decoder.page)
        self.caches = decoder.caches(n_seqs * per)
        order = torch.randperm(n_seqs * per, generator=torch.Generator().manual_seed(1))
        self.table = order.to(torch.int32).view(n_seqs, per).cuda()

    def batch(self, starts, counts):
        """counts[b] tokens of each sequence after its first starts[b]."""
        offsets = [0]
        for n in counts:
            offsets.append(offsets[-1] + n)
        as_ints = dict(dtype=torch.int32, device="cuda")
        lengths = torch.tensor([s + n for s, n in zip(starts, counts)], **as_ints)
        return rrq.CacheBatch(self.table, lengths, torch.tensor(offsets, **as_ints), offsets[-1])

    def run(self, starts, rows, drafts=None):
        """Logits of each sequence's new rows; drafts: their Tree."""
        batch = self.batch(starts, [len(r) for r in rows])
        tokens = torch.tensor([t for r in rows for t in r], dtype=torch.int64, device="cuda")
        positions = seen = None
        if drafts is not None:
            positions = torch.tensor([s + d for s in starts for d in drafts.depth],
                                     dtype=torch.int32, device="cuda")
            seen = torch.tensor([[w] for _ in starts for w in drafts.seen], dtype=torch.int64,
                                device="cuda")
        logits, self.fused = self.decoder.step(self.caches, batch, tokens, self.k, positions, seen)
        return logits

    def keep(self, starts, n_rows, kept):
        """Of the last run's n_rows rows a sequence those of kept[b], in order, become
        its next tokens: a path through a tree does not lie in a row in the cache."""
        batch = self.batch(starts, [len(p) for p in kept])
        rows = torch.tensor([b * n_rows + j for b, p in enumerate(kept) for j in p],
                            dtype=torch.int64, device="cuda")
        for cache, qkv in zip(self.caches, self.fused):
            rrq.cache_append(cache, batch, self.decoder.rotary,
                             *self.decoder.parts(qkv[rows]))


class Tree:
    """The shape of a step's drafts (64 rows at most): row 0, and for each row of a
    level widths[level] children."""

    def __init__(self, widths):
        self.parents, self.depth, self.seen, self.rank = [-1], [0], [1], [0]
        self.levels, last = [[0]], [0]
        for width in widths:
            level = []
            for p in last:
                for rank in range(width):
                    level.append(len(self.parents))
                    self.parents.append(p)
                    self.depth.append(self.depth[p] + 1)
                    self.seen.append(self.seen[p] | 1 << level[-1])
                    self.rank.append(rank)
            self.levels.append(level)
            last = level
        self.seen = [w - (1 << 64) if w >> 63 else w for w in self.seen]
        if len(self.parents) > 64:
            raise ValueError(f"a tree has 64 rows at most, got {len(self.parents)}")

    def upto(self, level):
        """The tree of the first levels."""
        part = object.__new__(Tree)
        n = self.levels[level][-1] + 1
        part.parents, part.depth, part.seen = self.parents[:n], self.depth[:n], self.seen[:n]
        return part


def generate(decoder, prompts, n_new, k_draft=1, k=4, widths=(1, 1, 1, 1), temperature=1.0,
             seed=3):
    """(texts of at least n_new new tokens, accepted drafts, steps). Widths of 1: chains
    drawn from the draft's distributions; else trees of its likeliest tokens."""
    n = len(prompts)
    tree, chain = Tree(widths), max(widths) == 1
    depth, n_rows = len(widths), sum(map(len, Tree(widths).levels))
    # the slowest text gains a token a step, while another may gain all its drafts
    most = max(map(len, prompts)) + n_new * (depth + 1) + n_rows
    draft, target = (Texts(decoder, x, n, most) for x in (k_draft, k))
    texts = [list(p) for p in prompts]
    for side in (draft, target):            # all but the last tokens
        if any(len(t) > 1 for t in texts):
            side.run([0] * n, [t[:-1] for t in texts])
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    offsets = torch.arange(0, n * n_rows + 1, n_rows, dtype=torch.int32, device="cuda")
    parents = None if chain else torch.tensor(tree.parents * n, dtype=torch.int32, device="cuda")
    accepted = steps = 0
    while min(len(t) - len(p) for t, p in zip(texts, prompts)) < n_new:
        starts = [len(t) - 1 for t in texts]
        rows = [[t[-1]] for t in texts]
        given = []                          # the draft's logits, by level
        for level in range(depth + 1):
            logits = draft.run(starts, rows, tree.upto(level)).view(n, -1, len(decoder.embed))
            if level == depth:
                break                       # (the last level's keys and values)
            last = logits[:, tree.levels[level]]
            if chain:
                given.append(last[:, 0])
                u = torch.rand(given[-1].shape, device="cuda", generator=g).clamp_(1e-9)
                x = given[-1] / temperature if temperature > 0 else given[-1]
                noise = -torch.log(-torch.log(u)) if temperature > 0 else 0.0
                new = (x + noise).argmax(-1, keepdim=True)
            else:
                _, _, ids, _ = rrq.token_logprobs(last.reshape(-1, last.shape[-1]),
                                                  n_top=widths[level])
                new = ids.view(n, -1)
            for r, t in zip(rows, new.tolist()):
                r += t
        logits = target.run(starts, rows, tree)
        uniforms = torch.rand(n * n_rows, device="cuda", generator=g)
        counts, following, paths = rrq.verify_drafts(
            logits, torch.tensor([t for r in rows for t in r], device="cuda"), offsets, depth,
            uniforms, torch.stack(given, 1) if chain else None, parents, temperature,
            temperature if temperature > 0 else 1.0)
        kept = [p[:c + 1] for p, c in zip(paths.tolist(), counts.tolist())]
        for side in (draft, target):
            if not chain:
                side.keep(starts, n_rows, kept)
        for text, r, path, t in zip(texts, rows, kept, following.tolist()):
            text += [r[j] for j in path[1:]] + [t]
        accepted += sum(map(len, kept)) - n
        steps += 1
    return texts, accepted, steps


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--new", type=int, default=24, help="tokens drawn a sequence")
    ap.add_argument("--code", choices=sorted(rrq.CODE_TYPES), default="int8")
    ap.add_argument("--temperature", type=float, default=0.7)
    args = ap.parse_args()
    decoder = Decoder(layers=args.layers, code_type=args.code)
    rng = torch.Generator().manual_seed(2)
    prompts = [torch.randint(0, 4096, (n,), generator=rng).tolist() for n in (7, 130, 301, 64)]
    for k in (1, 2, 3):
        for name, widths in (("chains of 4", (1, 1, 1, 1)), ("trees of 4, 2, 1", (4, 2, 1))):
            t0 = time.perf_counter()
            texts, accepted, steps = generate(decoder, prompts, args.new, k, 4, widths,
                                              args.temperature)
            torch.cuda.synchronize()
            new = sum(map(len, texts)) - sum(map(len, prompts))
            print(f"drafts at prefix {k}, {name}: {new} tokens in {steps} steps, "
                  f"{accepted / (steps * len(prompts)):.2f} accepted a step "
                  f"({time.perf_counter() - t0:.2f} s)")


if __name__ == "__main__":
    main()
