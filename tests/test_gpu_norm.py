"""rrq_block_norm on the GPU against its definition in 64 bits."""

import numpy as np
import pytest

from oracle import drafting as ora

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}


def _np(t):
    return None if t is None else t.detach().float().cpu().numpy()


def make(rows, cols, r="f32", y="f32", gate="", post="", bias=False, weight=True, seed=0, pad=0):
    """Arguments of block_norm; pad: columns around each matrix's, rows strided."""
    import torch
    g = torch.Generator().manual_seed(seed)
    types = _types()

    def matrix(dtype, gain, mean=0.0):
        x = torch.randn((rows, cols + 2 * pad), generator=g) * gain + mean
        x = x.to(types[dtype]).cuda()
        return x[:, pad:pad + cols]

    def vector(gain, mean, dtype="f32"):
        return (torch.randn(cols, generator=g) * gain + mean).to(types[dtype]).cuda()

    far = torch.where(torch.rand(cols, generator=g) < 0.02, 20.0, 1.0).cuda()
    residual = matrix(r, 1.0, 0.1)
    residual.copy_(residual.float() * far)
    a = dict(residual=residual, y=matrix(y, 0.7, 0.05) if y else None,
             weight=vector(0.1, 1.0) if weight else None, bias=vector(0.1, 0.0) if bias else None,
             post=post or None, post_weight=vector(0.1, 1.0) if post else None,
             gate={"": lambda: None, "vector": lambda: vector(0.3, 0.5, y),
                   "rows": lambda: matrix(y, 0.3, 0.5)}[gate]())
    return a


def check(rrq, a, kind="rms", scale=1.0, eps=1e-6, out="bf16", rows=slice(None), **kw):
    got, h = rrq.block_norm(**a, kind=kind, scale=scale, eps=eps, out_dtype=_types()[out], **kw)
    host = dict(residual=_np(a["residual"]), y=_np(a["y"]), weight=_np(a["weight"]),
                bias=_np(a["bias"]), kind=kind, post=a["post"], post_weight=_np(a["post_weight"]),
                gate=_np(a["gate"]), scale=np.float64(np.float32(scale)),
                eps=np.float64(np.float32(eps)))
    want, want_h = ora.block_norm(**host)
    err, err_h = ora.block_norm_error(**host)
    r_type = "f32" if a["residual"].dtype == _types()["f32"] else "bf16"
    for g, w, e, t, name in ((got, want, err, out, "out"), (h, want_h, err_h, r_type, "h")):
        g, w, e = _np(g).astype(np.float64)[rows], w[rows], e[rows]
        off = np.abs(g - w)
        # the result's own rounding is of a value off by e
        allowed = e + HALF[t] * (np.abs(w) + e)
        bad = np.argwhere(~(off <= allowed))
        assert bad.size == 0, f"{name}: {len(bad)} off, first {bad[0]}: {g[tuple(bad[0])]} " \
                              f"for {w[tuple(bad[0])]} +- {allowed[tuple(bad[0])]}"
    return got, h


@pytest.mark.parametrize("cols", [1, 2, 7, 8, 9, 63, 64, 65, 500, 513, 4095, 4096, 4097, 5120,
                                  8200, 20000, 33001, 65536])
@pytest.mark.parametrize("kind,post,gate", [("rms", "", ""), ("layer", "rms", "rows"),
                                            ("rms", "layer", "vector")])
def test_sizes(gpu, cols, kind, post, gate):
    check(gpu, make(3, cols, gate=gate, post=post, bias=cols % 2 == 1, seed=cols), kind)


def test_one_element_layer(gpu):
    """(x - x) / sqrt(0 + eps): the bias alone."""
    a = make(5, 1, post="layer", bias=True)
    got, h = gpu.block_norm(**a, kind="layer", out_dtype=_types()["f32"])
    assert np.array_equal(_np(got), np.broadcast_to(_np(a["bias"]), (5, 1)))
    assert np.array_equal(_np(h), _np(a["residual"]))


@pytest.mark.parametrize("r", ["f32", "bf16"])
@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [96, 4096, 4103])
def test_types(gpu, r, y, out, cols):
    check(gpu, make(5, cols, r, y, gate="rows", post="rms", bias=True, seed=3), "rms", 0.25, out=out)


@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("r,y", [("f32", "bf16"), ("bf16", "f32")])
def test_strided_rows(gpu, pad, r, y):
    """Columns of wider tensors, at any alignment of their type; what lies beside
    them plays no part."""
    a = make(7, 1001, r, y, gate="rows", pad=pad, seed=pad)
    want = check(gpu, a)
    for name in ("residual", "y", "gate"):
        wide = a[name]._base
        wide[:, :pad] = float("nan")
        wide[:, -pad:] = float("nan")
    got = check(gpu, a)
    assert all((g == w).all() for g, w in zip(got, want))


def test_without_weights_and_without_y(gpu):
    a = make(9, 768, weight=False, gate="vector")
    check(gpu, a, "layer", out="f32")
    a = make(9, 768, y=None, bias=True)
    got, h = check(gpu, a, "layer", out="f32")
    assert h is a["residual"]


def test_many_rows(gpu):
    check(gpu, make(3000, 260, "bf16", "bf16", gate="rows", post="layer"), "rms")


def test_more_rows_than_workgroups(gpu):
    """Every row of 2^20 and some is done, the last as the first."""
    import torch
    rows = (1 << 20) + 70
    a = make(70, 8, gate="rows", post="rms")
    want, want_h = gpu.block_norm(**a)
    far = {k: torch.zeros((rows, 8), device="cuda", dtype=a[k].dtype)
           for k in ("residual", "y", "gate")}
    for t, name in ((far[k], k) for k in far):
        t[:70] = a[name]
        t[-70:] = a[name]
    got, h = gpu.block_norm(**{**a, **far})
    for part in (slice(0, 70), slice(rows - 70, rows)):
        assert torch.equal(got[part], want) and torch.equal(h[part], want_h)
    assert (h[70:-70] == 0).all() and (got[70:-70] == 0).all()


def test_no_rows(gpu):
    import torch
    x = torch.empty((0, 64), device="cuda")
    out, h = gpu.block_norm(x, x)
    assert out.shape == h.shape == (0, 64)


def test_zeros_and_eps(gpu):
    """Rows of zeros, and rows whose mean square is far below and above eps."""
    import torch
    a = make(6, 384, gate="", post="rms")
    a["residual"][0] = 0
    a["y"][0] = 0
    a["residual"][1:3] *= 1e-6
    a["y"][1:4] *= 1e-6
    a["residual"][4:] *= 1e12
    check(gpu, a, "rms", eps=1e-5, out="f32")
    check(gpu, a, "layer", eps=1e-5, out="f32")
    got, _ = gpu.block_norm(torch.zeros((2, 64), device="cuda"), eps=0.0)
    assert torch.isnan(got).all()           # 0 / 0


def test_large_mean(gpu):
    """A row far from zero: differences to the mean, not a difference of squares."""
    a = make(4, 1000, weight=False)
    a["residual"] += 3000.0
    check(gpu, a, "layer", out="f32")


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_bad_row_stays_alone(gpu, bad):
    a = make(5, 700, gate="rows", post="layer")
    a["residual"][1, 3] = bad
    a["y"][3, 699] = bad
    with np.errstate(all="ignore"):
        check(gpu, a, "layer", rows=[0, 2, 4])


def test_in_place(gpu):
    import torch
    a = make(11, 2049, "bf16", "bf16", gate="vector")
    want, want_h = gpu.block_norm(**a)
    kept = a["residual"].clone()
    x = torch.empty_like(want)
    got, h = gpu.block_norm(**a, out=(x, a["residual"]))
    assert got is x and h is a["residual"]
    assert torch.equal(got, want) and torch.equal(h, want_h)
    assert not torch.equal(h, kept)


def test_neighbours_stay(gpu):
    """Outputs end where they end."""
    import torch
    a = make(3, 261, gate="rows")
    x = torch.full((5, 261), 7.0, device="cuda", dtype=torch.bfloat16)
    h = torch.full((5, 261), 7.0, device="cuda")
    gpu.block_norm(**a, out=(x[1:4], h[1:4]))
    for t in (x, h):
        assert (t[0] == 7).all() and (t[4] == 7).all()


def test_stream_and_graph(gpu):
    """A call on another stream, and one captured and replayed on other inputs."""
    import torch
    a = make(40, 1024, gate="rows", post="rms")
    want, want_h = gpu.block_norm(**a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, h = gpu.block_norm(**a, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(h, want_h)
    graph = torch.cuda.CUDAGraph()
    out = (torch.zeros_like(want), torch.zeros_like(want_h))
    with torch.cuda.graph(graph):
        gpu.block_norm(**a, out=out)
    for i in range(3):
        a["y"].mul_(1.5)
        graph.replay()
        want, want_h = gpu.block_norm(**a)
        assert torch.equal(out[0], want) and torch.equal(out[1], want_h)
        torch.cuda.synchronize()


def test_refusals(gpu):
    import torch
    a = make(4, 64, gate="rows", post="rms")
    f32 = torch.float32

    def refused(error, match, **kw):
        with pytest.raises(error, match=match):
            gpu.block_norm(**{**a, **kw})

    refused(ValueError, "GPU", residual=a["residual"].cpu())
    refused(TypeError, "torch.Tensor", residual=[1.0])
    refused(ValueError, "y must be on", y=a["y"].cpu())
    refused(ValueError, "y must be", y=a["y"][:3])
    refused(TypeError, "y must be", y=a["y"].half())
    refused(TypeError, "residual must be", residual=a["residual"].double())
    refused(ValueError, "last dimension", residual=a["residual"].t().contiguous().t())
    refused(ValueError, "weight", weight=a["weight"].bfloat16())
    refused(ValueError, "weight", weight=a["weight"][:63])
    refused(ValueError, "bias", bias=torch.zeros((1, 64), device="cuda"))
    refused(ValueError, "kind", kind="batch")
    refused(ValueError, "post", post="none")
    refused(ValueError, "need y", y=None)
    refused(ValueError, "post_weight needs post", post=None)
    refused(TypeError, "gate", gate=a["gate"].bfloat16())
    refused(ValueError, "gate", gate=a["gate"][:, :63])
    refused(ValueError, "gate", gate=a["gate"][:1].expand(4, 64))
    refused(TypeError, "out_dtype", out_dtype=torch.float16)
    refused(gpu.RRQError, "status", eps=-1.0)
    refused(gpu.RRQError, "status", scale=float("inf"))
    refused(gpu.RRQError, "status", residual=a["residual"][:1].expand(4, 64))
    x = torch.empty((4, 64), device="cuda")
    refused(TypeError, "out\\[1\\]", out=(x, x.bfloat16()))
    refused(ValueError, "contiguous", out=(x, torch.empty((4, 128), device="cuda")[:, :64]))
    refused(TypeError, "out\\[0\\]", out=(x, x.clone()), out_dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="residual itself"):
        gpu.block_norm(x, out=(x.clone(), x.clone()))
    with pytest.raises(gpu.RRQError):
        gpu.block_norm(torch.zeros((1, 65537), device="cuda", dtype=f32))
