"""The recurrent block's operators on the GPU against float64 (ops_reference.py), with its bounds.

Sizes cover one step and one row, odd widths, every layout of the kernels (time in pieces or not,
vectors or single elements, the row kernels' widths up to those read again for each statistic), masks that
leave a sequence or a row empty, values that are not finite in masked places, strides and streams.
"""
import numpy as np
import pytest

from . import ops_reference as ref
from .helpers import log

pytestmark = pytest.mark.gpu

PRECS = ["fp32", "bf16"]


def torch_():
    import torch
    return torch


def dtype(prec):
    return {"fp32": torch_().float32, "bf16": torch_().bfloat16}[prec]


def gpu(a, prec="fp32"):
    return torch_().from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(dtype(prec))


def host(t):
    return t.detach().double().cpu().numpy()


def check(name, got, want, prec):
    """Within the reference's bound and the output's one rounding; twice that, for the second-order
    terms that the bounds leave out."""
    value, bound = want
    g = host(got) if not isinstance(got, np.ndarray) else got
    assert g.shape == value.shape, (name, g.shape, value.shape)
    tol = 2 * ref.rounded(value, bound, prec)
    bad = ~(np.abs(g - value) <= tol)
    assert not bad.any(), "%s: %d of %d elements, worst %.3g of its bound" % (
        name, bad.sum(), bad.size, np.nanmax(np.abs(g - value)[bad] / tol[bad]))


# ----------------------------------------------------------------------------- scan

def scan_inputs(rng, B, T, D, prec, resets, ragged):
    t = dict(f=gpu(rng.standard_normal((B, T, D)) * 2 + 1, prec), v=gpu(rng.standard_normal((B, T, D)), prec),
             dy=gpu(rng.standard_normal((B, T, D)), prec), h0=gpu(rng.standard_normal((B, D))),
             dhT=gpu(rng.standard_normal((B, D))))
    reset = (rng.random((B, T)) < 0.1).astype(np.uint8) if resets else None
    lengths = None
    if ragged:
        lengths = rng.integers(0, T + 1, B).astype(np.int32)
        lengths[0] = 0
        if B > 1:
            lengths[-1] = T
    return t, reset, lengths


def scan_check(t, reset, lengths, prec, layout=lambda x: x, **kw):
    from paper_2312_06126_amd import ops
    torch = torch_()
    r = None if reset is None else torch.from_numpy(reset).cuda()
    n = None if lengths is None else torch.from_numpy(lengths).cuda()
    f, v, dy = (layout(t[k]) for k in ("f", "v", "dy"))
    y, hT, saved = ops.scan(f, v, t["h0"], reset=r, lengths=n, save=True, **kw)
    y2, hT2 = ops.scan(f, v, t["h0"], reset=r, lengths=n, **kw)
    df, dv, dh0 = ops.scan_backward(f, v, dy, saved, dhT=t["dhT"], reset=r, lengths=n, **kw)
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(hT, hT2)
    want = ref.scan(host(t["f"]), host(t["v"]), host(t["h0"]), reset, lengths, host(t["dy"]), host(t["dhT"]))
    for name, got, p in (("y", y, prec), ("hT", hT, "fp32"), ("df", df, prec), ("dv", dv, prec), ("dh0", dh0, "fp32")):
        check(name, got, want[name], p)
    return y, hT, df, dv, dh0


SCANS = [(1, 1, 1), (3, 1, 5), (16, 1, 256), (2, 7, 3), (5, 16, 8), (2, 17, 12), (3, 50, 64), (2, 64, 200), (1, 63, 4), (1, 64, 4),
         (1, 65, 4), (2, 129, 7), (1, 1000, 1), (1, 1000, 36), (7, 333, 20), (1, 4099, 8), (130, 40, 513), (70, 33, 1024), (2, 1500, 40),
         (1, 3001, 7), (4, 1024, 72), (3, 520, 257), (2, 2100, 4096), (600, 18, 900)]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("shape", SCANS, ids=str)
def test_scan(shape, prec):
    log("scan %s %s" % (shape, prec))
    rng = np.random.default_rng(sum(shape))
    for resets, ragged in ((False, False), (True, True)):
        scan_check(*scan_inputs(rng, *shape, prec, resets, ragged), prec)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("shape", [(3, 50, 64), (1, 700, 40), (4, 130, 9), (1, 1300, 24), (600, 17, 904)], ids=str)
def test_scan_layouts(shape, prec):
    """Time-major arrays, parts of one projection, rows at odd distances and unaligned starts give the
    results of contiguous ones."""
    torch = torch_()
    rng = np.random.default_rng(5)
    B, T, D = shape
    t, reset, lengths = scan_inputs(rng, *shape, prec, True, True)

    def time_major(x):
        return x.transpose(0, 1).contiguous().transpose(0, 1)

    def part(x):
        w = torch.full((B, T, 3 * D), float("nan"), dtype=x.dtype, device="cuda")
        w[..., D:2 * D] = x
        return w[..., D:2 * D]

    def odd(x):
        w = torch.full((B, T + 2, D + 3), float("nan"), dtype=x.dtype, device="cuda")
        w[:, 1:T + 1, 1:D + 1] = x
        return w[:, 1:T + 1, 1:D + 1]

    for layout in (time_major, part, odd):
        log("scan %s %s %s" % (layout.__name__, shape, prec))
        scan_check(t, reset, lengths, prec, layout)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("T", [6, 300])
def test_scan_masked_values_do_not_matter(prec, T):
    """Infinities and NaN behind a sequence's length and in the state in front of an episode start, in
    either direction; forget gates of +-inf."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(6)
    B, D = 4, 24
    t, _, _ = scan_inputs(rng, B, T, D, prec, False, False)
    reset = np.zeros((B, T), np.uint8)
    reset[:, T // 2] = 1
    lengths = np.array([T, T - 2, T // 2 + 1, 0], np.int32)
    clean = {k: x.clone() for k, x in t.items()}
    for b in range(B):
        for k in ("f", "v", "dy"):
            t[k][b, lengths[b]:] = float("nan")
            t[k][b, lengths[b] + 1:] = float("inf")
    t["v"][0, T // 2 - 1] = float("inf")    # reaches only the steps before the episode start
    t["h0"][1] = float("nan")
    t["f"][2, T // 2 + 0] = float("-inf")   # a = 0
    t["f"][1, T // 2 + 1] = float("inf")    # a = 1
    clean["f"][2, T // 2] = -200.0
    clean["f"][1, T // 2 + 1] = 200.0
    r, n = torch.from_numpy(reset).cuda(), torch.from_numpy(lengths).cuda()
    y, hT, saved = ops.scan(t["f"], t["v"], t["h0"], reset=r, lengths=n, save=True)
    df, dv, dh0 = ops.scan_backward(t["f"], t["v"], t["dy"], saved, dhT=t["dhT"], reset=r, lengths=n)
    want = ref.scan(host(clean["f"]), host(clean["v"]), host(clean["h0"]), reset, lengths, host(clean["dy"]), host(clean["dhT"]))
    s = slice(T // 2, T)
    for name, got in (("y", y), ("df", df), ("dv", dv)):
        check(name, got[:, s], tuple(w[:, s] for w in want[name]), prec)
    check("hT", hT, want["hT"], "fp32")
    # The gradient that a NaN behind an episode start would carry back stays there.
    t["dy"][0, T - 1] = float("nan")
    df, dv, dh0 = ops.scan_backward(clean["f"], clean["v"], t["dy"], ops.scan(clean["f"], clean["v"], clean["h0"], reset=r,
                                                                             lengths=n, save=True)[2],
                                    dhT=t["dhT"], reset=r, lengths=n)
    assert torch.isnan(dv[0, T // 2:]).all() and torch.isfinite(dv[0, :T // 2]).all() and torch.isfinite(dh0).all()


def test_scan_in_steps_equals_the_sequence():
    """Samplers' steps with the state updated in place, on a stream of their own, against one call over the
    sequence; also replayed from a HIP graph."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(7)
    B, T, D = 16, 12, 256
    t, reset, _ = scan_inputs(rng, B, T, D, "bf16", True, False)
    r = torch.from_numpy(reset).cuda()
    y, hT = ops.scan(t["f"], t["v"], t["h0"], reset=r)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    h = t["h0"].clone()
    torch.cuda.synchronize()
    steps = [ops.scan(t["f"][:, i:i + 1], t["v"][:, i:i + 1], h, reset=r[:, i:i + 1], hT=h, stream=side)[0] for i in range(T)]
    side.synchronize()
    assert torch.equal(torch.cat(steps, 1), y) and torch.equal(h, hT)

    h.copy_(t["h0"])
    f1, v1, r1, y1 = t["f"][:, :1].clone(), t["v"][:, :1].clone(), r[:, :1].clone(), torch.empty_like(y[:, :1].contiguous())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.scan(f1, v1, h, reset=r1, hT=h, out=y1)
    h.copy_(t["h0"])
    for i in range(T):
        f1.copy_(t["f"][:, i:i + 1])
        v1.copy_(t["v"][:, i:i + 1])
        r1.copy_(r[:, i:i + 1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y1, y[:, i:i + 1])
    assert torch.equal(h, hT)


def test_scan_optional_arguments_and_differences():
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(8)
    B, T, D = 3, 200, 16
    t, reset, lengths = scan_inputs(rng, B, T, D, "fp32", True, True)
    r, n = torch.from_numpy(reset).cuda(), torch.from_numpy(lengths).cuda()
    y, hT, saved = ops.scan(t["f"], t["v"], save=True)
    df, dv, dh0 = ops.scan_backward(t["f"], t["v"], None, saved)
    assert not df.any() and not dv.any() and not dh0.any()
    df, dv, dh0 = ops.scan_backward(t["f"], t["v"], t["dy"], saved)
    want = ref.scan(host(t["f"]), host(t["v"]), None, None, None, host(t["dy"]))
    for name, got in (("y", y), ("hT", hT), ("df", df), ("dv", dv), ("dh0", dh0)):
        check(name, got, want[name], "fp32")
    # Gradient along a direction against the difference of float32 forward calls, summed in 64 bits. The
    # difference quotient over 2e = 2^-6 is off by e^2 times third derivatives (sums of N = 9600 terms of
    # order 1: sqrt(N) e^2 = 6e-3) and by float32 rounding of N outputs (sqrt(N) 2^-24 * 4 / 2e = 1.5e-3).
    y, hT, saved = ops.scan(t["f"], t["v"], t["h0"], reset=r, lengths=n, save=True)
    df, dv, dh0 = ops.scan_backward(t["f"], t["v"], t["dy"], saved, dhT=t["dhT"], reset=r, lengths=n)
    e = 2.0 ** -7
    for k, g in (("f", df), ("v", dv), ("h0", dh0)):
        d = torch.from_numpy(rng.choice([-1.0, 1.0], t[k].shape).astype(np.float32)).cuda()
        sides = []
        for sign in (1, -1):
            i = dict(t, **{k: t[k] + sign * e * d})
            yy, hh = ops.scan(i["f"], i["v"], i["h0"], reset=r, lengths=n)
            sides.append((yy.double() * t["dy"].double()).sum() + (hh.double() * t["dhT"].double()).sum())
        diff, dot = float(sides[0] - sides[1]) / (2 * e), float((g.double() * d.double()).sum())
        assert abs(diff - dot) <= 0.05, (k, diff, dot)


def test_scan_refuses():
    from paper_2312_06126_amd import ops
    from paper_2312_06126_amd.spz import SPZ_EINVAL, SpzError
    torch = torch_()
    f = torch.zeros((2, 3, 4), device="cuda")
    bad = [dict(f=f.cpu(), v=f), dict(f=f.half(), v=f.half()), dict(f=f[0], v=f[0]), dict(f=f, v=f[:, :2]), dict(f=f, v=f.bfloat16()),
           dict(f=f, v=f.cpu()), dict(f=f, v=f.transpose(1, 2)), dict(f=f, v=f, h0=f[:, 0, :3]), dict(f=f, v=f, h0=f[:, 0].bfloat16()),
           dict(f=f, v=f, reset=torch.zeros((2, 3), device="cuda")), dict(f=f, v=f, lengths=torch.zeros(2, device="cuda")),
           dict(f=f, v=f, out=f[:1].expand(2, 3, 4)), dict(f=f, v=f, hT=f[0])]
    for kw in bad:
        with pytest.raises(SpzError) as e:
            ops.scan(**kw)
        assert e.value.code == SPZ_EINVAL
    with pytest.raises(SpzError):
        ops.scan_backward(f, f, f, None)
    with pytest.raises(SpzError):
        ops.scan_backward(f, f, f, torch.zeros(3, device="cuda"))


# ----------------------------------------------------------------------------- block norm and dropout

def block_inputs(rng, R, D, prec, vectors=True, masked=False):
    t = {k: gpu(rng.standard_normal((R, D)) + m, prec) for k, m in (("x", 0.0), ("h", 0.3), ("z", 0.0))}
    for k in ("w_post", "w_pre", "scale", "b_post", "b_pre"):
        t[k] = gpu(rng.standard_normal(D) * 0.3 + (0.0 if k[0] == "b" else 1.0)) if vectors else None
    g = {k: gpu(rng.standard_normal((R, D)), prec) for k in ("dx_out", "du")}
    valid = (rng.random(R) < 0.7).astype(np.uint8) if masked else None
    return t, g, valid


def block_check(t, g, valid, prec, post, pre, gate, drop=None, eps=1e-5, **kw):
    from paper_2312_06126_amd import ops
    torch = torch_()
    v = None if valid is None else torch.from_numpy(valid).cuda()
    opts = dict(post=post, pre=pre, gate=gate, eps=eps, drop=drop, valid=v, **kw)
    x_out, u = ops.block_norm(**t, **opts)
    grads = ops.block_norm_backward(g["dx_out"], g["du"], **t, **opts)
    again = ops.block_norm_backward(g["dx_out"], g["du"], **t, **opts)
    torch.cuda.synchronize()
    h = {k: None if x is None else host(x) for k, x in t.items()}
    gg = {k: None if x is None else host(x) for k, x in g.items()}
    factor = ref.drop_factor(t["x"].shape, *drop) if drop else None
    want = ref.block_norm(**h, post=post, pre=pre, gate_kind=gate, eps=eps, factor=factor, valid=valid, **gg)
    if t["h"] is not None:
        check("x_out", x_out, want["x_out"], prec)
    if pre != "none":
        check("u", u, want["u"], prec)
    for k, got in grads.items():
        if got is None:
            continue
        assert torch.equal(got, again[k]), k
        if k in want and not (post == "none" and k in ("dw_post", "db_post")) and not (pre == "none" and k in ("dw_pre", "db_pre")):
            check(k, got, want[k], prec if k in ("dx", "dh", "dz") else "fp32")


# Widths on both sides of each row layout's end, in vectors and single elements.
WIDTHS = [1, 3, 8, 64, 127, 128, 130, 256, 257, 393, 512, 516, 1000, 1024, 1030, 2048, 2056, 4100, 4104, 8192, 8200, 16384, 16392]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("width", WIDTHS)
def test_block_norm(width, prec):
    rng = np.random.default_rng(width)
    for rows, post, pre, gate, drop, masked in ((5, "layer", "layer", "sigmoid", (0.1, 7, 1, 2), True),
                                                (3, "rms", "rms", "silu", None, False)):
        log("block_norm %d x %d %s %s" % (rows, width, prec, post))
        block_check(*block_inputs(rng, rows, width, prec, masked=masked), prec, post, pre, gate, drop)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("rows,width", [(1, 64), (3000, 256), (1100, 72), (4099, 5), (2500, 136)])
def test_block_norm_many_rows(rows, width, prec):
    rng = np.random.default_rng(rows)
    log("block_norm %d x %d %s" % (rows, width, prec))
    block_check(*block_inputs(rng, rows, width, prec, masked=True), prec, "rms", "layer", "silu", (0.25, 1 << 40, 3, 4))


@pytest.mark.parametrize("post,pre,gate,block,vectors", [
    ("none", "rms", "none", True, True), ("rms", "none", "sigmoid", True, True), ("none", "layer", "silu", True, False),
    ("layer", "none", "none", True, False), ("rms", "rms", "none", False, True), ("rms", "layer", "silu", False, False)])
def test_block_norm_parts(post, pre, gate, block, vectors):
    rng = np.random.default_rng(11)
    for width in (40, 393):
        t, g, valid = block_inputs(rng, 9, width, "fp32", vectors, True)
        if not block:
            t["h"] = None
        block_check(t, g, valid, "fp32", post, pre, gate, None if not block else (0.5, 3, 2, 1))
        for missing in ("dx_out", "du"):
            block_check(t, dict(g, **{missing: None}), valid, "fp32", post, pre, gate)


def test_block_norm_masked_rows_and_zero_rows():
    """Rows that are masked may hold anything; rows of zeros have finite norms; no rows give zero sums."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(12)
    t, g, valid = block_inputs(rng, 40, 96, "fp32", masked=True)
    for group in (t, g):
        for k, x in group.items():
            if x.dim() == 2:
                x[torch.from_numpy(valid).cuda() == 0] = float("nan")
    t["h"][int(np.flatnonzero(valid)[0])] = 0.0
    block_check(t, g, valid, "fp32", "layer", "rms", "silu")
    grads = ops.block_norm_backward(g["dx_out"], g["du"], **t, gate="silu", valid=torch.zeros(40, dtype=torch.uint8, device="cuda"))
    for x in grads.values():
        assert not x.any()
    none = {k: x[:0] if x.dim() == 2 else x for k, x in t.items()}
    grads = ops.block_norm_backward(g["dx_out"][:0], g["du"][:0], **none, gate="silu")
    for k, x in grads.items():
        assert not x.any() and x.shape == ((0, 96) if k in ("dx", "dh", "dz") else (96,))
    closed = dict(t, h=torch.ones_like(t["h"]), x=torch.ones_like(t["x"]), z=torch.full_like(t["z"], float("-inf")))
    x_out, _ = ops.block_norm(**closed, gate="silu")
    assert torch.equal(x_out, closed["x"])


def test_block_norm_strides_and_streams():
    torch = torch_()
    rng = np.random.default_rng(13)
    for prec in PRECS:
        t, g, valid = block_inputs(rng, 33, 64, prec, masked=True)

        def apart(x, start):
            if x is None or x.dim() != 2:
                return x
            w = torch.full((33, 64 + 8 + start), float("nan"), dtype=x.dtype, device="cuda")
            w[:, start:64 + start] = x
            return w[:, start:64 + start]

        for start in (0, 1, 8):
            tt, gg = {k: apart(x, start) for k, x in t.items()}, {k: apart(x, start) for k, x in g.items()}
            torch.cuda.synchronize()
            block_check(tt, gg, valid, prec, "rms", "layer", "sigmoid", (0.1, 5, 6, 7), stream=torch.cuda.Stream())
        one = dict(t, x=t["x"][:1].expand(33, 64))
        block_check(one, g, valid, prec, "rms", "rms", "silu")


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (3, 8), (5, 393), (256, 64), (77, 1030)], ids=str)
def test_dropout(shape, prec):
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(14)
    x = gpu(rng.standard_normal(shape), prec)
    for p, seed, step, tensor in ((0.0, 1, 2, 3), (0.1, (1 << 63) + 5, 0xFFFFFFFF, 9), (0.5, 0, 0, 0), (1.0, 1, 1, 1)):
        factor = ref.drop_factor(shape, p, seed, step, tensor)
        want = host(x) * factor
        got = ops.dropout(x, p, seed, step, tensor)
        check("y", got, (want, 2 * ref.U * np.abs(want)), prec)
        assert np.array_equal(host(got) == 0, (factor == 0) | (host(x) == 0))
        # Rows apart, unaligned, and in place.
        w = torch.full((shape[0], shape[1] + 5), 7.0, dtype=x.dtype, device="cuda")
        part = w[:, 1:shape[1] + 1]
        part.copy_(x)
        assert torch.equal(ops.dropout(part, p, seed, step, tensor, out=part), got)
        assert bool((w[:, 0] == 7).all()) and bool((w[:, shape[1] + 1:] == 7).all())
    x[0, 0] = float("nan")
    assert not ops.dropout(x, 1.0, 1, 1, 1).any()


def test_dropout_past_32_bits():
    """The last elements of an array of more than 2^32 take the words of their 64-bit index."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rows, width = 4099, 1 << 20
    x = torch.ones((rows, width), dtype=torch.bfloat16, device="cuda")
    y = ops.dropout(x, 0.25, 11, 12, 13, out=x)
    tail = host(y[-1, -64:])
    torch.cuda.synchronize()
    first = rows * width - 64
    u = np.uint64
    blocks = np.arange(first // 8, first // 8 + 8, dtype=np.uint64)
    from oracle import philox
    w = np.stack(philox.block(blocks, u(12), u(5), u(13), u(11), u(0)), 1)
    words = np.stack([w & u(0xFFFF), w >> u(16)], 2).reshape(-1)
    assert np.array_equal(tail != 0, words >= 16384)


def test_block_norm_refuses():
    from paper_2312_06126_amd import ops
    from paper_2312_06126_amd.spz import SPZ_EINVAL, SpzError
    torch = torch_()
    x = torch.zeros((4, 8), device="cuda")
    w = torch.ones(8, device="cuda")
    bad = [dict(x=x.cpu()), dict(x=x[0]), dict(x=x, h=x[:3]), dict(x=x, h=x.bfloat16()), dict(x=x, post="batch"), dict(x=x, gate="relu"),
           dict(x=x, h=x, gate="silu"), dict(x=x, w_pre=w[:4]), dict(x=x, w_pre=w.bfloat16()), dict(x=x, valid=w[:4]),
           dict(x=x, pre="none"), dict(x=x, eps=0.0), dict(x=x, h=x, drop=(1.5, 1, 2, 3)), dict(x=x.t().contiguous().t())]
    for kw in bad:
        with pytest.raises(SpzError) as e:
            ops.block_norm(**kw)
        assert e.value.code == SPZ_EINVAL
    for kw in (dict(p=2.0), dict(p=0.5, out=x[:2])):
        with pytest.raises(SpzError):
            ops.dropout(x, seed=1, step=2, **kw)


# ----------------------------------------------------------------------------- 8-bit product

def quant_check(x, wq, sw, bias, prec, weights, **kw):
    from paper_2312_06126_amd import ops
    y = ops.quant_linear(x, weights, bias=None if bias is None else gpu(bias), **kw)
    q, s = ref.quant_rows(x.float().cpu().numpy())
    terms = s.astype(np.float64)[:, None] * sw.astype(np.float64)[None] * (q @ wq.T.astype(np.float64))
    want = terms if bias is None else terms + bias
    # The sum as float32, two scales, their product, the addition: 6 roundings of the term, 1 of the result.
    check("y", y, (want, 8 * ref.U * np.abs(terms) + 2 * ref.U * np.abs(want)), prec)
    return y


QUANTS = [(1, 1, 1), (1, 32, 32), (16, 256, 64), (3, 31, 33), (33, 33, 31), (16, 1024, 1024), (100, 393, 400), (300, 64, 34), (257, 1000, 130),
          (64, 1030, 70), (129, 2500, 300), (5, 4096, 96), (513, 96, 1), (2049, 40, 260), (1000, 768, 512), (4100, 512, 264),
          (33000, 64, 136), (32700, 48, 72), (32768, 1024, 600), (17000, 2048, 200), (16500, 100, 540), (8300, 33, 33),
          (8200, 2080, 80), (1100, 4096, 2100), (70, 4128, 40), (300, 6000, 200)]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("shape", QUANTS, ids=str)
def test_quant_linear(shape, prec):
    from paper_2312_06126_amd import ops
    torch = torch_()
    log("quant %s %s" % (shape, prec))
    M, K, N = shape
    rng = np.random.default_rng(sum(shape))
    x = gpu(np.maximum(rng.standard_normal((M, K)), -0.2), prec)
    if M > 2:
        x[1] = 0.0
    wf = gpu(rng.standard_normal((N, K)))
    q, s = ops.quant_rows(wf)
    wq, sw = ref.quant_rows(wf.cpu().numpy())
    assert np.array_equal(host(q), wq) and np.array_equal(s.cpu().numpy(), sw)
    weights = ops.quant_pack(q, s)
    bias = rng.standard_normal(N).astype(np.float32)
    y = quant_check(x, wq, sw, bias, prec, weights)
    quant_check(x, wq, sw, None, prec, weights)
    # Rows apart and unaligned, into rows apart.
    xx = torch.full((M, K + 3), float("nan"), dtype=x.dtype, device="cuda")
    xx[:, 1:K + 1] = x
    yy = torch.full((M, N + 2), 5.0, dtype=x.dtype, device="cuda")
    ops.quant_linear(xx[:, 1:K + 1], weights, bias=gpu(bias), out=yy[:, 1:N + 1])
    assert torch.equal(yy[:, 1:N + 1], y)
    assert bool((yy[:, 0] == 5).all()) and bool((yy[:, N + 1] == 5).all())


@pytest.mark.parametrize("prec", PRECS)
def test_quant_rows_values(prec):
    """Ties to even, the extremes, zeros, tiny rows, and rows that are not finite."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    x = np.zeros((8, 40), np.float32)
    x[0, :6] = [127.0, 0.5, 1.5, 2.5, -0.5, -126.5]     # scale 1: halves go to even
    x[1, 7] = -3.0
    x[3] = 1e-30
    x[4, 39] = 3e38
    x[5, 3], x[5, 4] = 1.0, np.inf
    x[6, 3], x[6, 4] = 1.0, np.nan
    x[7] = np.linspace(-1, 1, 40)
    t = gpu(x, prec)
    q, s = ops.quant_rows(t)
    wq, ws = ref.quant_rows(t.float().cpu().numpy())
    assert np.array_equal(host(q), wq) and np.array_equal(s.cpu().numpy(), ws, equal_nan=True)
    w = ops.quant_pack(torch.ones((3, 40), dtype=torch.int8, device="cuda"), torch.ones(3, device="cuda"))
    y = ops.quant_linear(t, w)
    assert torch.isnan(y[5:7]).all() and torch.isfinite(y[torch.tensor([0, 1, 2, 3, 4, 7], device="cuda")]).all()
    e, f = ops.quant_rows(t[:, :0])
    assert e.shape == (8, 0) and not f.any()


def test_quant_rows_like_torch():
    """The integers and scales of 20 million elements are those of the same formula in torch on the GPU."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    x = torch.randn((100000, 200), generator=gen, device="cuda")
    q, s = ops.quant_rows(x)
    want = x.abs().amax(1) / 127.0
    assert torch.equal(s, want) and torch.equal(q.float(), torch.round(x / want[:, None]))
    w = ops.quant_pack(torch.eye(200, dtype=torch.int8, device="cuda"), torch.ones(200, device="cuda"))
    assert torch.equal(ops.quant_linear(x, w), torch.round(x / want[:, None]) * want[:, None])


def test_quant_largest_sums_and_empty_inner():
    """Sums of the greatest length stay exact in 32 bits; no inputs leave the bias."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    K = 131072
    x = torch.ones((2, K), device="cuda")
    w = ops.quant_pack(torch.full((1, K), 127, dtype=torch.int8, device="cuda"), torch.ones(1, device="cuda"))
    y = ops.quant_linear(x, w)
    assert np.allclose(host(y), 127.0 * K, rtol=1e-6)
    bias = torch.arange(5, dtype=torch.float32, device="cuda")
    w = ops.quant_pack(torch.zeros((5, 0), dtype=torch.int8, device="cuda"), torch.ones(5, device="cuda"))
    assert torch.equal(ops.quant_linear(torch.zeros((3, 0), device="cuda"), w, bias=bias), bias.expand(3, 5))


def test_quant_refuses():
    from paper_2312_06126_amd import ops
    from paper_2312_06126_amd.spz import SPZ_EINVAL, SpzError
    torch = torch_()
    x = torch.zeros((4, 8), device="cuda")
    q, s = ops.quant_rows(x)
    w = ops.quant_pack(q, s)
    for call in (lambda: ops.quant_linear(x[:, :7], w), lambda: ops.quant_linear(x.half(), w), lambda: ops.quant_linear(x, w, bias=s[:2]),
                 lambda: ops.quant_linear(x, w, out=x[:, :4].bfloat16()), lambda: ops.quant_pack(x, s), lambda: ops.quant_pack(q, s[:2]),
                 lambda: ops.quant_pack(q, None), lambda: ops.quant_linear(x, w._replace(outer=64)), lambda: ops.quant_rows(x[0])):
        with pytest.raises(SpzError) as e:
            call()
        assert e.value.code == SPZ_EINVAL


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("shape", [(129, 500, 1100), (256, 260, 1024), (257, 260, 1024), (96, 700, 4000), (300, 500, 1100), (270, 200, 1500),
                                   (300, 4096, 4001), (3000, 1025, 2100), (3000, 2048, 1500), (8200, 1000, 2000), (16400, 300, 100),
                                   (16400, 100, 130), (16400, 1700, 65), (20000, 1024, 130), (300, 5000, 200)], ids=str)
def test_quant_ways(shape, prec):
    """Each way of spreading a product, at shares that do not divide, against exact sums. Rounded to 24 bits: the
    sum, the product of the scales, the result; then once to the output's bits."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    M, K, N = shape
    rng = np.random.default_rng(31)
    x = gpu(rng.standard_normal((M, K)).astype(np.float32), prec)
    q, s = ops.quant_rows(x)
    wq, ws = ops.quant_rows(gpu(rng.standard_normal((N, K)).astype(np.float32)))
    bias = gpu(rng.standard_normal(N).astype(np.float32))
    room = torch.full((M + 2, N + 3), 7.0, dtype=x.dtype, device="cuda")
    y = room[1:M + 1, 1:N + 1]
    ops.quant_linear(x, ops.quant_pack(wq, ws), bias=bias, out=y)
    product = (q.double() @ wq.double().t().contiguous()) * s.double()[:, None] * ws.double()
    want = product + bias.double()
    bound = 2.0 ** -22 * (product.abs() + want.abs()) + (2.0 ** -8 if prec == "bf16" else 2.0 ** -24) * 1.01 * want.abs() + 1e-37
    assert bool(((y.double() - want).abs() <= bound).all())
    y.fill_(7.0)
    assert bool((room == 7.0).all())


# ----------------------------------------------------------------------------- across the operators

def test_offsets_past_32_bits():
    """Rows 2^32 elements apart give what the same rows side by side give."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(21)
    B, T, D, far = 2, 40, 64, 1 << 32
    big = torch.empty(far + T * D, dtype=torch.bfloat16, device="cuda")
    f = gpu(rng.standard_normal((B, T, D)), "bf16")
    v = gpu(rng.standard_normal((B, T, D)), "bf16")
    apart = big.as_strided((B, T, D), (far, D, 1))
    apart.copy_(f)
    y, hT, saved = ops.scan(f, v, save=True)
    y2, hT2, saved2 = ops.scan(apart, v, save=True)
    assert torch.equal(y, y2) and torch.equal(hT, hT2)
    for a, b in zip(ops.scan_backward(f, v, y, saved), ops.scan_backward(apart, v, y, saved2)):
        assert torch.equal(a, b)
    ops.scan(f, v, out=apart)                  # now the far rows are outputs
    assert torch.equal(apart, y)
    rows = big.as_strided((B, D), (far, 1))
    x = rows.contiguous()
    h = v[0, :B].contiguous()
    for a, b in zip(ops.block_norm(x, h), ops.block_norm(rows, h)):
        assert torch.equal(a, b)
    assert torch.equal(ops.block_norm_backward(x, h, x, h)["dx"], ops.block_norm_backward(rows, h, rows, h)["dx"])
    w = ops.quant_pack(*ops.quant_rows(gpu(rng.standard_normal((48, D)))))
    assert torch.equal(ops.quant_linear(x, w), ops.quant_linear(rows, w))
    assert all(torch.equal(a, b) for a, b in zip(ops.quant_rows(x), ops.quant_rows(rows)))


@pytest.mark.parametrize("rows,inner", [(40, 4096), (33000, 512)])
def test_graphs_replay_the_eager_results(rows, inner):
    """A captured block (8-bit product, norm with dropout and gradients, scan in pieces) on new inputs, replayed
    between eager work: every replay equals the eager calls."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(22)
    D = 64
    w = ops.quant_pack(*ops.quant_rows(gpu(rng.standard_normal((D, inner)))))
    ones = torch.ones(D, device="cuda")
    x = torch.empty((rows, inner), dtype=torch.bfloat16, device="cuda")
    history = torch.empty((1, 4096, D), dtype=torch.bfloat16, device="cuda")

    def block():
        u = ops.quant_linear(x, w)
        x_out, n = ops.block_norm(u, u, u, w_post=ones, scale=ones, w_pre=ones, gate="silu", drop=(0.2, 1, 2, 3))
        g = ops.block_norm_backward(x_out, n, u, u, u, w_post=ones, scale=ones, w_pre=ones, gate="silu", drop=(0.2, 1, 2, 3))
        y, hT, saved = ops.scan(history, history, save=True)
        df, dv, dh0 = ops.scan_backward(history, history, y, saved)
        return [u, x_out, n, y, hT, df, dv, dh0, ops.dropout(n, 0.5, 4, 5, 6)] + list(g[k] for k in ("dx", "dh", "dz", "dw_post", "dscale", "dw_pre"))

    x.normal_()
    history.normal_()
    block()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = block()
    for i in range(4):
        x.copy_(gpu(rng.standard_normal((rows, inner)), "bf16"))
        history.copy_(gpu(rng.standard_normal((1, 4096, D)), "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, block()):
            assert torch.equal(a, b), i
        torch.cuda.synchronize()
