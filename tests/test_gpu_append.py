"""rrq_cache_append on the GPU against its definition: rotated queries, codes and
scales bit for bit, and nothing else touched."""

import numpy as np
import pytest

from oracle import drafting as ora
from serving_helpers import Setup, assert_same_blocks, bf16

pytestmark = pytest.mark.gpu

CODES = ["int8", "fp8"]
# (new tokens, length with them) of each sequence
RAGGED = [(1, 1), (5, 21), (0, 9), (40, 40), (3, 130), (17, 33)]


def _frequencies(rot):
    return 10000.0 ** (-np.arange(rot // 2) * 2.0 / rot)


def _rows(rng, n, heads, dim, dtype):
    x = rng.normal(size=(n, heads, dim)).astype(np.float32)
    x *= np.float32(2.0) ** rng.integers(-3, 4, size=(n, heads, 1)).astype(np.float32)
    return bf16(x) if dtype == "bf16" else x


class Case:
    def __init__(self, gpu, seqs, q_heads, heads, dim, page, code, dtype, seed, rot=None,
                 layout="half", amplitude=1.0, positions=None):
        import torch
        self.torch = torch
        self.s = s = Setup(gpu, seqs, heads, dim, page, code, seed=seed).fill(
            [length - n for n, length in seqs])
        n = s.offsets[-1]
        self.Q = _rows(s.rng, n, q_heads, dim, dtype)
        self.K = _rows(s.rng, n, heads, dim, dtype)
        self.V = _rows(s.rng, n, heads, dim, dtype)
        self.dtype = torch.float32 if dtype == "f32" else torch.bfloat16
        self.frequencies = _frequencies(rot or dim)
        self.layout, self.amplitude, self.positions = layout, amplitude, positions
        s.to_gpu()
        self.rotary = gpu.Rotary(torch.from_numpy(self.frequencies).cuda(), layout, amplitude)

    def upload(self):
        """Columns of one fused row, with columns between that are not theirs."""
        t = self.torch
        parts, n = [self.Q, self.K, self.V], len(self.Q)
        wide = t.full((max(n, 1), sum(p.shape[1] + 1 for p in parts), self.Q.shape[2]),
                      float("nan"), device="cuda", dtype=self.dtype)
        out, at = [], 0
        for p in parts:
            wide[:n, at:at + p.shape[1]] = t.from_numpy(p).cuda().to(self.dtype)
            out.append(wide[:n, at:at + p.shape[1]])
            at += p.shape[1] + 1
        return out

    def device_positions(self):
        if self.positions is None:
            return None
        return self.torch.tensor(self.positions, dtype=self.torch.int32, device="cuda")

    def call(self, **kw):
        return self.s.rrq.cache_append(self.s.cache, self.s.batch, self.rotary, *self.upload(),
                                       self.device_positions(), **kw)

    def check(self, **kw):
        s = self.s
        got = self.call(**kw)
        self.torch.cuda.synchronize()
        want = ora.append(s.host, s.table, s.lengths, s.offsets, self.positions, self.frequencies,
                          self.layout, self.amplitude, self.Q, self.K, self.V)
        want = bf16(want) if self.dtype == self.torch.bfloat16 else want
        assert_same_blocks(got.float().cpu().numpy(), want, "queries")
        assert_same_blocks(s.ks.cpu().numpy(), s.host.ks, "key scales")
        assert_same_blocks(s.vs.cpu().numpy(), s.host.vs, "value scales")
        assert_same_blocks(s.k.cpu().numpy(), s.host.k, "key codes")
        assert_same_blocks(s.v.cpu().numpy(), s.host.v, "value codes")
        return got


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("q_heads,heads,dim,page,rot", [
    (1, 1, 64, 16, 64), (6, 3, 128, 32, 128), (5, 2, 256, 64, 256), (7, 2, 64, 128, 8),
    (3, 1, 256, 16, 72), (2, 2, 128, 128, 64)])
def test_append_equals_the_definition(gpu, code, dtype, layout, q_heads, heads, dim, page, rot):
    Case(gpu, RAGGED, q_heads, heads, dim, page, code, dtype, dim + page, rot, layout).check()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_positions(gpu, layout):
    """Positions of long contexts, negative ones and the ends of the type, in 64 bits;
    an amplitude."""
    n = sum(k for k, _ in RAGGED)
    far = [0, 1, -1, 131071, -131071, 1 << 20, 123456789, (1 << 31) - 1, -(1 << 31)]
    Case(gpu, RAGGED, 4, 2, 128, 64, "int8", "f32", 3, layout=layout, amplitude=1.1386294,
         positions=[far[i % len(far)] + (i // len(far) if i % len(far) < 7 else 0)
                    for i in range(n)]).check()


def test_exact_turns(gpu):
    """Frequencies of whole and quarter turns, and zero: cosines and sines next to 0 and
    1, and keys that stay."""
    import torch
    c = Case(gpu, RAGGED, 4, 2, 64, 32, "fp8", "f32", 4, rot=16)
    c.frequencies = np.array([0.0, np.pi / 2, np.pi, 2 * np.pi, np.pi / 4, 1.0, 3.0, 1e-9])
    c.rotary = gpu.Rotary(torch.from_numpy(c.frequencies).cuda())
    got = c.check()
    want = torch.from_numpy(c.Q).cuda()
    assert torch.equal(got[..., 0], want[..., 0]) and torch.equal(got[..., 8], want[..., 8])


@pytest.mark.parametrize("code", CODES)
def test_equals_rotation_then_write(gpu, code):
    """The calls it stands for: torch's rotation in 64 bits, then cache_write."""
    import torch
    c = Case(gpu, RAGGED, 4, 2, 128, 64, code, "f32", 5)
    K = torch.from_numpy(ora.rotate(c.K, ora.places(c.s.lengths, c.s.offsets), c.frequencies,
                                    "half", 1.0)).cuda()
    V = torch.from_numpy(c.V).cuda()
    got = c.call()
    codes = [t.clone() for t in c.s.cache.tensors]
    c.s.to_gpu()
    gpu.cache_write(c.s.cache, c.s.batch, K, V)
    for a, b in zip(codes, c.s.cache.tensors):
        assert_same_blocks(a.cpu().numpy(), b.cpu().numpy(), "cache")
    assert got.shape == c.Q.shape


@pytest.mark.parametrize("n", [1, 300, 1500, 9000])
def test_many_tokens(gpu, n):
    """Groups of one token and of several, whole and not."""
    Case(gpu, [(n, n + 3), (7, 7)], 5, 1, 64, 64, "int8", "bf16", n, rot=32).check()


def test_repeated_call_and_in_place(gpu):
    import torch
    c = Case(gpu, RAGGED, 4, 2, 128, 16, "int8", "bf16", 6)
    want = c.check()
    codes = [t.clone() for t in c.s.cache.tensors]
    Q, K, V = c.upload()
    Q = Q.contiguous()
    got = gpu.cache_append(c.s.cache, c.s.batch, c.rotary, Q, K, V, out=Q)
    assert got is Q and torch.equal(got, want)
    for a, b in zip(codes, c.s.cache.tensors):
        assert_same_blocks(a.cpu().numpy(), b.cpu().numpy(), "cache")


def test_rows_outside_the_offsets_and_pages(gpu):
    """Rows before the first and behind the last sequence stay as they are; pages out of
    range and positions past the table are not written."""
    import torch
    c = Case(gpu, [(3, 20), (6, 40), (2, 2)], 4, 2, 64, 16, "int8", "f32", 7)
    s = c.s
    n = s.offsets[-1]
    before = [t.clone() for t in s.cache.tensors]
    table = torch.from_numpy(s.table).cuda()
    table[0, 1] = s.cache.n_pages           # the page of the first sequence's new tokens
    table[2, 0] = -1
    lengths = torch.tensor([20, 100, 2], dtype=torch.int32, device="cuda")    # past its table
    offsets = torch.tensor([2, 5, 11, 13], dtype=torch.int32, device="cuda")
    batch = gpu.CacheBatch(table, lengths, offsets, n + 6)
    pad = [torch.cat([torch.full((2,) + x.shape[1:], 5.0), torch.from_numpy(x),
                      torch.full((4,) + x.shape[1:], 5.0)]).cuda() for x in (c.Q, c.K, c.V)]
    out = torch.full_like(pad[0], 7.0)
    gpu.cache_append(s.cache, batch, c.rotary, *pad, out=out)
    assert (out[:2] == 7).all() and (out[2 + n:] == 7).all()
    want = ora.rotate(c.Q, ora.places([20, 100, 2], [0, 3, 9, 11]), c.frequencies, "half", 1.0)
    assert_same_blocks(out[2:2 + n].cpu().numpy(), want, "queries")
    for a, b in zip(before, s.cache.tensors):
        assert_same_blocks(a.cpu().numpy(), b.cpu().numpy(), "cache")


def test_nothing_to_do(gpu):
    c = Case(gpu, [(0, 5), (0, 0)], 4, 2, 64, 16, "int8", "f32", 8)
    before = [t.clone() for t in c.s.cache.tensors]
    assert c.call().shape == (0, 4, 64)
    for a, b in zip(before, c.s.cache.tensors):
        assert_same_blocks(a.cpu().numpy(), b.cpu().numpy(), "cache")


def test_stream_and_graph(gpu):
    """On another stream; captured, and replayed as the sequences grow."""
    import torch
    c = Case(gpu, [(1, 30), (1, 17), (1, 100)], 4, 2, 128, 16, "int8", "f32", 9)
    s = c.s
    Q, K, V = (t.contiguous() for t in c.upload())
    args = (s.cache, s.batch, c.rotary, Q, K, V)
    want = gpu.cache_append(*args)
    codes = [t.clone() for t in s.cache.tensors]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = gpu.cache_append(*args, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    for a, b in zip(codes, s.cache.tensors):
        assert_same_blocks(a.cpu().numpy(), b.cpu().numpy(), "cache")
    out = torch.empty_like(Q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gpu.cache_append(*args, out=out)
    for i in range(3):
        s.batch.lengths.sub_(1)
        K.mul_(1.25)
        graph.replay()
        replayed = [t.clone() for t in s.cache.tensors]
        want = gpu.cache_append(*args)
        assert torch.equal(out, want)
        torch.cuda.synchronize()
        for a, b in zip(replayed, s.cache.tensors):
            assert_same_blocks(a.cpu().numpy(), b.cpu().numpy(), "cache")


def test_refusals(gpu):
    import torch
    c = Case(gpu, [(3, 20), (2, 2)], 4, 2, 128, 16, "int8", "f32", 10)
    s = c.s
    Q, K, V = c.upload()
    before = [t.clone() for t in s.cache.tensors]

    def refused(error, match, Q=Q, K=K, V=V, positions=None, rotary=c.rotary, **kw):
        with pytest.raises(error, match=match):
            gpu.cache_append(s.cache, s.batch, rotary, Q, K, V, positions, **kw)

    refused(ValueError, "Q must be", Q=Q[:4])
    refused(ValueError, "K must be", K=K[:, :1])
    refused(ValueError, "V must be", V=V[..., :64])
    refused(ValueError, "K must be on", K=K.cpu())
    refused(TypeError, "one dtype", V=V.bfloat16())
    refused(TypeError, "Q must be", Q=Q.half(), K=K.half(), V=V.half())
    refused(ValueError, "positions", positions=torch.zeros(4, dtype=torch.int32, device="cuda"))
    refused(ValueError, "positions", positions=torch.zeros(5, dtype=torch.int64, device="cuda"))
    refused(ValueError, "positions", positions=torch.zeros(5, dtype=torch.int32))
    refused(ValueError, "out must be", out=torch.empty((5, 3, 128), device="cuda"))
    refused(TypeError, "out", out=torch.empty((5, 4, 128), device="cuda").bfloat16())
    f = c.rotary.frequencies
    refused(gpu.RRQError, "status", rotary=gpu.Rotary(f[:2]))          # of 4 channels
    refused(gpu.RRQError, "status", rotary=gpu.Rotary(torch.cat([f, f])))
    refused(gpu.RRQError, "status", rotary=gpu.Rotary(f, amplitude=float("nan")))
    with pytest.raises(ValueError, match="layout"):
        gpu.Rotary(f, "whole")
    with pytest.raises(TypeError, match="float64"):
        gpu.Rotary(f.float())
    with pytest.raises(ValueError, match="GPU"):
        gpu.Rotary(f.cpu())
    with pytest.raises(ValueError, match="contiguous"):
        gpu.Rotary(f[::2])
    torch.cuda.synchronize()
    for a, b in zip(before, s.cache.tensors):
        assert_same_blocks(a.cpu().numpy(), b.cpu().numpy(), "cache")
