"""Every way that the recurrent block's operators have of spreading a call, in vectors and single elements, against
float64: which way a shape takes is asked of the library, so that a changed rule cannot leave one without a test."""
import ctypes

import numpy as np
import pytest

from . import ops_reference as ref
from .helpers import log
from .test_gpu_ops import PRECS, block_inputs, check, gpu, host, scan_check, scan_inputs, torch_

pytestmark = pytest.mark.gpu

SERIAL, TILES, PIECES, VECTORS = 0, 1, 2, 4


def scan_way(f, backward):
    """The library's way for tensors laid out as f is (spzt_scan_way)."""
    from paper_2312_06126_amd import spz
    B, T, D = f.shape
    a = spz.ScanArgs(batch=B, steps=T, width=D, prec=int(f.dtype == torch_().bfloat16))
    for k in ("f", "v", "y", "dy", "df", "dv"):
        setattr(a, k, f.data_ptr())
        setattr(a, k + "_batch", f.stride(0))
        setattr(a, k + "_step", f.stride(1))
    return spz.load().spzt_scan_way(ctypes.byref(a), int(backward))


def pieces_of(B, T, D):
    from paper_2312_06126_amd import spz
    return spz.load().spz_scan_workspace(ctypes.byref(spz.ScanArgs(batch=B, steps=T, width=D)), 0) // (16 * B * D)


def contiguous(x):
    return x


def time_major(x):
    return x.transpose(0, 1).contiguous().transpose(0, 1)


def part(x):
    """The middle third of a projection, NaN on either side."""
    D = x.shape[-1]
    w = torch_().full((*x.shape[:-1], 3 * D), float("nan"), dtype=x.dtype, device="cuda")
    w[..., D:2 * D] = x
    return w[..., D:2 * D]


def odd(x):
    """Rows at odd distances from an unaligned start."""
    B, T, D = x.shape
    w = torch_().full((B, T + 2, D + 3), float("nan"), dtype=x.dtype, device="cuda")
    w[:, 1:T + 1, 1:D + 1] = x
    return w[:, 1:T + 1, 1:D + 1]


# Time in pieces, of whole and partial segments; 1100 pieces are more than scan_join holds in registers. Layouts of
# the vector form first; odd() takes vectors away.
LONG = [((1, 4096, 64), contiguous, True), ((2, 6000, 40), contiguous, True), ((1, 35200, 8), contiguous, True),
        ((1, 9001, 12), contiguous, True), ((3, 2000, 40), time_major, True), ((2, 3000, 100), part, True),
        ((1, 35200, 7), contiguous, False), ((2, 3001, 33), time_major, False), ((2, 3000, 100), odd, False)]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("shape,layout,vectors", LONG, ids=lambda p: getattr(p, "__name__", str(p)))
def test_scan_in_pieces(shape, layout, vectors, prec):
    rng = np.random.default_rng(sum(shape))
    B, T, D = shape
    for resets, lengths in ((False, None), (True, [T - 3 - b * (T // 3) for b in range(B)])):
        t, reset, _ = scan_inputs(rng, *shape, prec, resets, False)
        log("scan in %d pieces %s %s %s" % (pieces_of(*shape), layout.__name__, shape, prec))
        for back in (False, True):
            assert scan_way(layout(t["f"]), back) == PIECES + VECTORS * vectors
        if reset is not None:
            reset[:, 1:] = rng.random((B, T - 1)) < 0.002    # some pieces start no episode, as most do
        scan_check(t, reset, None if lengths is None else np.array(lengths, np.int32), prec, layout)
    assert pieces_of(1, 35200, 8) > 1024 and pieces_of(1, 35200, 7) > 1024


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("shape,vectors", [((1, 4096, 64), True), ((2, 3001, 33), False)], ids=str)
def test_scan_in_pieces_masked_values_do_not_matter(shape, vectors, prec):
    """Infinities and NaN in front of an episode start and behind a sequence's end stay on their side of it, through
    the maps of the pieces between."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    B, T, D = shape
    rng = np.random.default_rng(61)
    t, _, _ = scan_inputs(rng, *shape, prec, False, False)
    assert scan_way(t["f"], False) == scan_way(t["f"], True) == PIECES + VECTORS * vectors
    cut, end = T // 2 + 3, T - 700
    reset = np.zeros((B, T), np.uint8)
    reset[:, cut] = 1
    lengths = np.full(B, end, np.int32)
    r, n = torch.from_numpy(reset).cuda(), torch.from_numpy(lengths).cuda()
    want = ref.scan(host(t["f"]), host(t["v"]), host(t["h0"]), reset, lengths, host(t["dy"]), host(t["dhT"]))
    bad = {k: x.clone() for k, x in t.items()}
    for k in ("f", "v", "dy"):
        bad[k][:, end:] = float("nan")
        bad[k][:, end + 40:] = float("inf")
    bad["v"][:, 100] = float("inf")      # the state is not finite from here to the episode start
    bad["h0"][:, 0] = float("nan")
    y, hT, saved = ops.scan(bad["f"], bad["v"], bad["h0"], reset=r, lengths=n, save=True)
    df, dv, dh0 = ops.scan_backward(bad["f"], bad["v"], bad["dy"], saved, dhT=t["dhT"], reset=r, lengths=n)
    assert not torch.isfinite(y[:, 100:cut]).any() and not torch.isfinite(y[:, :cut, 0]).any()
    for name, got in (("y", y), ("df", df), ("dv", dv)):
        check(name, got[:, cut:], tuple(w[:, cut:] for w in want[name]), prec)
    check("hT", hT, want["hT"], "fp32")
    check("dv", dv, want["dv"], prec)     # takes no state
    check("dh0", dh0, want["dh0"], "fp32")
    # A NaN behind the episode start does not come back past it.
    bad = dict(t, dy=t["dy"].clone(), dhT=torch.full_like(t["dhT"], float("nan")))
    saved = ops.scan(t["f"], t["v"], t["h0"], reset=r, lengths=n, save=True)[2]
    df, dv, dh0 = ops.scan_backward(t["f"], t["v"], bad["dy"], saved, dhT=bad["dhT"], reset=r, lengths=n)
    assert torch.isnan(dv[:, cut:end]).all() and not dv[:, end:].any()
    for name, got in (("df", df), ("dv", dv)):
        check(name, got[:, :cut], tuple(w[:, :cut] for w in want[name]), prec)
    check("dh0", dh0, want["dh0"], "fp32")


def test_scan_shapes_take_every_way():
    """The shapes of the scan's tests, here and in test_gpu_ops, in either direction."""
    from .test_gpu_ops import SCANS
    torch = torch_()
    shapes = SCANS + [s for s, layout, _ in LONG if layout is contiguous]
    for back in (False, True):
        ways = {scan_way(torch.empty(s, device="cuda"), back) for s in shapes}
        assert ways == {w + v for w in (SERIAL, TILES, PIECES) for v in (0, VECTORS)}, (back, ways)


# ----------------------------------------------------------------------------- block norm

def chunked_reference(t, g, valid, factor, **opts):
    """ref.block_norm over 64 rows at a time. Its bound of a sum over R rows counts R + 64 roundings, here 128: more than
    the kernel's, whose threads add their own rows (up to 5 here), up to 16 threads' sums, a thread's share of the workgroups
    (up to 32) and 32 such shares one after the other."""
    R = len(t["x"])
    out = {}
    for r in range(0, R, 64):
        rows = slice(r, r + 64)
        cut = lambda d: {k: None if x is None else x[rows] if x.ndim == 2 else x for k, x in d.items()}
        o = ref.block_norm(**cut(t), factor=factor[rows], valid=valid[rows], **cut(g), **opts)
        for k, (v, e) in o.items():
            out.setdefault(k, []).append((v, e))
    return {k: tuple(np.concatenate(p) if p[0].ndim == 2 else np.sum(p, 0) for p in zip(*parts)) for k, parts in out.items()}


# Rows of each layout (16, 32, 64 lanes, a workgroup, two chunks a thread, read again) such that a thread takes four or five.
ROWS = [(34000, 64), (27000, 61), (17000, 200), (14000, 201), (8000, 400), (7000, 393), (3500, 1000), (3500, 1001), (1800, 2048),
        (900, 2050), (900, 4104), (900, 4100), (450, 8208), (450, 8193)]


def groups_of(rows, width):
    """Rows that the backward kernel takes at once: its workgroups (of which the workspace holds sums) by rows of each."""
    from paper_2312_06126_amd import spz
    n = spz.load().spz_block_norm_workspace(ctypes.byref(spz.BlockNormArgs(rows=rows, width=width, eps=1e-6))) // (20 * width)
    return n * (16 if width <= 128 else 8 if width <= 256 else 4 if width <= 512 else 1)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("rows,width", ROWS)
def test_block_norm_gradients_over_rows(rows, width, prec):
    """Threads that take several rows: all outputs and gradients against float64, masks and dropout on."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    assert rows > 3 * groups_of(rows, width)
    log("block_norm %d x %d %s" % (rows, width, prec))
    rng = np.random.default_rng(rows + width)
    t, g, valid = block_inputs(rng, rows, width, prec, masked=True)
    drop = (0.1, 7, 1, 2)
    opts = dict(post="layer", pre="rms", gate="silu", eps=1e-5)
    grads = ops.block_norm_backward(g["dx_out"], g["du"], **t, **opts, drop=drop, valid=torch.from_numpy(valid).cuda())
    opts["gate_kind"] = opts.pop("gate")
    want = chunked_reference({k: host(x) for k, x in t.items()}, {k: host(x) for k, x in g.items()}, valid,
                             ref.drop_factor((rows, width), *drop), **opts)
    for k, got in grads.items():
        check(k, got, want[k], prec if k in ("dx", "dh", "dz") else "fp32")


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("rows,width", ROWS)
def test_block_norm_sums_take_every_row_once(rows, width, prec):
    """Sums of small integers are exact: a row that is left out or taken twice shows in db_pre, db_post and dscale. For dw_pre
    and dw_post the gradient is zero in all rows but one, at each place of the loop over rows."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    stride = groups_of(rows, width)
    rng = np.random.default_rng(rows)
    log("block_norm sums %d x %d %s" % (rows, width, prec))
    whole = lambda lo, hi: gpu(rng.integers(lo, hi + 1, (rows, width)), prec)
    valid = (rng.random(rows) < 0.9)
    live = torch.from_numpy(valid).cuda()
    zero, one = torch.zeros(width, device="cuda"), torch.ones(width, device="cuda")
    x, h, d = whole(-4, 4), whole(-3, 3), whole(-2, 2)
    total = lambda p: torch.where(live[:, None], p.double(), 0.0).sum(0)
    # No gradient through the pre norm reaches db_pre, none through the post norm dscale or db_post.
    g = ops.block_norm_backward(None, d, x, b_pre=zero, pre="layer", valid=live)
    assert torch.equal(g["db_pre"].double(), total(d))
    g = ops.block_norm_backward(d, None, x, h, scale=one, post="none", pre="none", valid=live)
    assert torch.equal(g["dscale"].double(), total(d.double() * h.double()))
    g = ops.block_norm_backward(d, None, x, h, b_post=zero, pre="none", valid=live)
    assert torch.equal(g["db_post"].double(), total(d))
    for k in sorted({0, 1, stride - 1, stride, 2 * stride, 2 * stride + 1, 3 * stride, rows - 1}):
        only = torch.zeros_like(d)
        only[k] = 1.0
        g = ops.block_norm_backward(None, only, x, h, None, one, None, None, one, post="rms", pre="rms")
        w = ref.block_norm(host(x[k:k + 1]), host(h[k:k + 1]), w_post=host(one), w_pre=host(one), du=host(only[k:k + 1]))
        for name in ("dw_pre", "dw_post"):
            check(name, g[name], w[name], "fp32")
