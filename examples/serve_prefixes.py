"""A small decoder served from RRQ packages, start to end on one GPU.

Ragged prompts are taken in in chunks over an 8-bit paged cache, tokens are
drawn greedily with their likeliest alternatives, and the text is then scored
at every prefix of the package: how much likelihood the 2, 4, 6 and 8 bit
weights give it. Weights are random (there is no checkpoint here), so the
text means nothing; the calls are those of a real one.

    python examples/serve_prefixes.py
"""

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_04048_amd as rrq  # noqa: E402

GROUP = 128


class Linear:
    """A linear layer held as an RRQ package; k stages of it serve a call."""

    def __init__(self, rows, cols, generator):
        W = torch.randn((rows, cols), device="cuda", generator=generator) * cols ** -0.5
        self.rows, self.cols = rows, cols
        self.package = rrq.construct(W.bfloat16(), GROUP)

    def __call__(self, x, k):
        return rrq.linear(x.bfloat16().contiguous(), *self.package, self.rows, self.cols, GROUP, k)


def norm(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)


def rotate(x, positions):
    """Rotary positions of [tokens, heads, dim]."""
    half = x.shape[-1] // 2
    freq = 10000.0 ** (-torch.arange(half, device=x.device, dtype=torch.float32) / half)
    angle = positions[:, None, None] * freq
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)


class Decoder:
    """Pre-norm decoder layers with grouped heads and a gated feed-forward."""

    def __init__(self, vocab=4096, hidden=1024, layers=2, heads=16, kv_heads=4, dim=64,
                 inner=2048, page=64, code_type="int8", seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.page = heads, kv_heads, dim, page
        self.code_type = code_type
        self.embed = torch.randn((vocab, hidden), device="cuda", generator=g)
        self.layers = [{"qkv": Linear((heads + 2 * kv_heads) * dim, hidden, g),
                        "out": Linear(hidden, heads * dim, g),
                        "up": Linear(2 * inner, hidden, g),
                        "down": Linear(hidden, inner, g)} for _ in range(layers)]
        self.head = Linear(vocab, hidden, g)

    def caches(self, n_pages):
        return [rrq.KVCache.empty(n_pages, self.kv_heads, self.dim, self.page, self.code_type)
                for _ in self.layers]

    def step(self, caches, batch, tokens, positions, k):
        """Logits [tokens, vocab] of the batch's new tokens."""
        x = self.embed[tokens]
        for w, cache in zip(self.layers, caches):
            qkv = w["qkv"](norm(x), k).view(len(tokens), -1, self.dim)
            qk = rotate(qkv[:, :self.heads + self.kv_heads], positions)
            # the values go to the cache as columns of the fused projection
            rrq.cache_write(cache, batch, qk[:, self.heads:],
                            qkv[:, self.heads + self.kv_heads:])
            a = rrq.cache_attention(cache, batch, qk[:, :self.heads])
            x = x + w["out"](a.view(len(tokens), -1), k)
            gate, up = w["up"](norm(x), k).chunk(2, -1)
            x = x + w["down"](torch.nn.functional.silu(gate) * up, k)
        return self.head(norm(x), k)


class Sequences:
    """Texts and their pages; `take` makes the next call's batch."""

    def __init__(self, decoder, n_seqs, max_tokens):
        self.per = -(-max_tokens // decoder.page)
        self.caches = decoder.caches(n_seqs * self.per)
        # pages dealt in any order: a pool hands them out as sequences grow
        order = torch.randperm(n_seqs * self.per, generator=torch.Generator().manual_seed(1))
        self.table = order.to(torch.int32).view(n_seqs, self.per).cuda()
        self.lengths = [0] * n_seqs

    def take(self, counts):
        """The batch of counts[b] further tokens of each sequence, and their
        positions."""
        positions, offsets = [], [0]
        for b, n in enumerate(counts):
            positions += range(self.lengths[b], self.lengths[b] + n)
            offsets.append(offsets[-1] + n)
            self.lengths[b] += n
        as_ints = dict(dtype=torch.int32, device="cuda")
        batch = rrq.CacheBatch(self.table, torch.tensor(self.lengths, **as_ints),
                               torch.tensor(offsets, **as_ints), offsets[-1])
        return batch, torch.tensor(positions, dtype=torch.float32, device="cuda"), offsets


def tokens_of(parts):
    return torch.tensor([t for part in parts for t in part], dtype=torch.int64, device="cuda")


def generate(decoder, prompts, n_new, k, chunk=96, n_top=5):
    """(texts, log probabilities of the drawn tokens, alternatives of the last
    step) from prompts, each taken in in chunks."""
    seqs = Sequences(decoder, len(prompts), max(map(len, prompts)) + n_new)
    texts = [list(p) for p in prompts]
    last = [None] * len(prompts)
    for start in range(0, max(map(len, prompts)), chunk):
        parts = [p[start:start + chunk] for p in prompts]
        batch, positions, offsets = seqs.take([len(p) for p in parts])
        logits = decoder.step(seqs.caches, batch, tokens_of(parts), positions, k)
        for b, part in enumerate(parts):
            if part:
                last[b] = logits[offsets[b + 1] - 1]
    logits = torch.stack(last)
    logprobs = []
    for i in range(n_new):
        _, _, ids, top = rrq.token_logprobs(logits, n_top=n_top)
        for text, t in zip(texts, ids[:, 0].tolist()):
            text.append(t)
        logprobs.append(top[:, 0])
        if i + 1 < n_new:
            batch, positions, _ = seqs.take([1] * len(texts))
            logits = decoder.step(seqs.caches, batch, tokens_of([t[-1:] for t in texts]),
                                  positions, k)
    return texts, torch.stack(logprobs, 1), (ids, top)


def score(decoder, texts, k):
    """(mean log probability of each text's tokens given those before, mean
    entropy) at prefix k: every text in one call."""
    seqs = Sequences(decoder, len(texts), max(map(len, texts)))
    batch, positions, offsets = seqs.take([len(t) for t in texts])
    logits = decoder.step(seqs.caches, batch, tokens_of(texts), positions, k)
    # the last token of a text predicts nothing that is given
    targets = tokens_of([t[1:] + [-1] for t in texts])
    logprob, entropy, _, _ = rrq.token_logprobs(logits, targets)
    means = [logprob[a:b - 1].mean().item() for a, b in zip(offsets, offsets[1:])]
    return means, entropy.mean().item()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--new", type=int, default=24, help="tokens drawn a sequence")
    ap.add_argument("--code", choices=sorted(rrq.CODE_TYPES), default="int8")
    args = ap.parse_args()
    decoder = Decoder(layers=args.layers, code_type=args.code)
    rng = torch.Generator().manual_seed(2)
    prompts = [torch.randint(0, 4096, (n,), generator=rng).tolist() for n in (7, 130, 301, 64)]
    t0 = time.perf_counter()
    texts, logprobs, (ids, top) = generate(decoder, prompts, args.new, 4)
    torch.cuda.synchronize()
    print(f"{len(texts)} sequences, {args.new} tokens each in {time.perf_counter() - t0:.2f} s; "
          f"mean log probability {logprobs.mean().item():.3f}")
    print("last step's alternatives of sequence 0:",
          ", ".join(f"{i}: {p:.3f}" for i, p in zip(ids[0].tolist(), top[0].tolist())))
    for k in (1, 2, 3, 4):
        means, entropy = score(decoder, texts, k)
        print(f"prefix {k} ({2 * k} bits): log probability a token "
              f"{sum(means) / len(means):8.3f}, entropy {entropy:.3f}")


if __name__ == "__main__":
    main()
