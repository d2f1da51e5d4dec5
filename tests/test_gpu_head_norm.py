"""Head norms with rotation on the GPU against float64 (more_ops_reference.py), with its bounds."""
import numpy as np
import pytest

from . import more_ops_reference as ref
from .helpers import log
from .test_gpu_ops import PRECS, check, gpu, host, torch_

pytestmark = pytest.mark.gpu


def inputs(rng, rows, heads, heads_k, dim, prec):
    t = dict(q=gpu(rng.standard_normal((rows, heads, dim)) * 1.5 + 0.2, prec), dq=gpu(rng.standard_normal((rows, heads, dim)), prec))
    if heads_k is not None:
        t.update(k=gpu(rng.standard_normal((rows, heads_k, dim)) * 0.5, prec), dk=gpu(rng.standard_normal((rows, heads_k, dim)), prec))
    for n in ("w_q", "b_q", "w_k", "b_k"):
        t[n] = gpu(rng.standard_normal(dim) * 0.3 + (n[0] == "w"))
    return t


def check_call(t, prec, kind="rms", pairs="halves", positions=None, freqs=None, valid=None, vectors=("w_q", "b_q", "w_k", "b_k"), layout=lambda x: x,
               out=None, back_out=None, **kw):
    from paper_2312_06126_amd import ops
    torch = torch_()
    names = [n for n in vectors if n[2] == "q" or "k" in t]
    a = dict({n: t[n] for n in names}, norm=kind, eps=1e-5, pairs=pairs, **kw)
    if freqs is not None:
        a.update(positions=torch.from_numpy(positions.astype(np.int32)).cuda(), freqs=torch.from_numpy(freqs).cuda())
    if valid is not None:
        a["valid"] = torch.from_numpy(valid).cuda()
    q, k = layout(t["q"]), layout(t["k"]) if "k" in t else None
    yq, yk = ops.head_norm(q, k, out=out, **a)
    g = ops.head_norm_backward(layout(t["dq"]), layout(t["dk"]) if "k" in t else None, q, k, out=back_out, **a)
    torch.cuda.synchronize()
    for part, y in (("q", yq), ("k", yk))[:2 if "k" in t else 1]:
        opt = {n[0]: host(t[n]) for n in names if n[2] == part}
        want = ref.head_norm(host(t[part]), kind=kind, eps=1e-5, positions=positions, freqs=freqs, pairs=pairs, valid=valid,
                             dy=host(t["d" + part]), **opt)
        check(part, y, want["y"], prec)
        check("d" + part, g["d" + part], want["dx"], prec)
        for n in "wb":
            name = "d%s_%s" % (n, part)
            if n in opt:
                check(name, g[name], want["d" + n], "fp32")
            else:
                assert g.get(name) is None
    return yq, yk, g


def freqs_of(half, base=100.0):
    return np.array([base ** (-i / max(half, 1)) for i in range(half)])


SHAPES = [(1, 1, 1, 1), (1, 1, 0, 2), (3, 2, 1, 5), (16, 4, 4, 64), (5, 3, 2, 24), (7, 4, 1, 40), (130, 5, 5, 39), (33, 16, 4, 64), (9, 2, 2, 128),
          (20, 3, 3, 256), (4, 2, 1, 200), (300, 1, 1, 8), (6, 2, 3, 512), (3, 2, 1, 1023), (2, 1, 1, 1024), (2000, 3, 2, 16), (11, 7, 3, 96), (700, 8, 8, 32)]


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_head_norm(shape, prec):
    log("head_norm %s %s" % (shape, prec))
    rng = np.random.default_rng(sum(shape))
    rows, heads, heads_k, dim = shape
    positions = rng.integers(0, 2000, rows)
    for kind, pairs, half, masked in (("rms", "halves", dim // 2, False), ("layer", "neighbours", dim // 3, True), ("none", "halves", dim // 4, True),
                                      ("rms", "neighbours", dim // 2, True), ("layer", "halves", 0, False)):
        valid = (rng.random(rows) < 0.7).astype(np.uint8) if masked else None
        t = inputs(rng, rows, heads, heads_k, dim, prec)
        check_call(t, prec, kind, pairs, positions if half else None, freqs_of(half) if half else None, valid)


@pytest.mark.parametrize("prec", PRECS)
def test_head_norm_without_keys_or_vectors(prec):
    rng = np.random.default_rng(1)
    t = inputs(rng, 40, 4, None, 64, prec)
    check_call(t, prec)
    check_call(t, prec, vectors=())
    t = inputs(rng, 40, 4, 2, 64, prec)
    check_call(t, prec, vectors=("w_q",), positions=np.arange(40), freqs=freqs_of(32))
    check_call(t, prec, kind="layer", vectors=("b_k", "w_k"))


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_head_norm_far_and_negative_positions(prec, pairs):
    """Positions up to the type's ends, where a float32 angle would be off by whole turns."""
    rng = np.random.default_rng(2)
    positions = np.array([0, 1, -1, 2 ** 24 + 1, 10 ** 9 + 7, 2 ** 31 - 1, -2 ** 31, 123456789])
    t = inputs(rng, len(positions), 2, 2, 64, prec)
    check_call(t, prec, "rms", pairs, positions, freqs_of(32, 10000.0))


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("shape", [(50, 4, 2, 64), (50, 3, 3, 40), (13, 2, 2, 39)], ids=str)
def test_head_norm_layouts(shape, prec):
    """Parts of one projection, heads in front of the rows, odd distances and starts; outputs in place and into parts."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(3)
    rows, heads, heads_k, dim = shape
    t = inputs(rng, *shape, prec)
    positions, freqs = rng.integers(0, 500, rows), freqs_of(dim // 2)

    def odd(x):
        w = torch.full((rows + 2, x.shape[1] + 1, dim + 3), float("nan"), dtype=x.dtype, device="cuda")
        w[1:rows + 1, 1:, 1:dim + 1] = x
        return w[1:rows + 1, 1:, 1:dim + 1]

    def heads_first(x):
        return x.transpose(0, 1).contiguous().transpose(0, 1)

    for layout in (odd, heads_first):
        log("head_norm %s %s %s" % (layout.__name__, shape, prec))
        check_call(t, prec, positions=positions, freqs=freqs, layout=layout)
        outs = tuple(odd(torch.zeros_like(t[n])) for n in "qk")
        backs = tuple(heads_first(torch.zeros_like(t[n])) for n in "qk")
        check_call(t, prec, "layer", "neighbours", positions, freqs, layout=layout, out=outs, back_out=backs)
    a = dict(w_q=t["w_q"], w_k=t["w_k"], positions=torch.from_numpy(positions.astype(np.int32)).cuda(), freqs=torch.from_numpy(freqs).cuda())
    want = ops.head_norm(t["q"], t["k"], **a)
    grads = ops.head_norm_backward(t["dq"], t["dk"], t["q"], t["k"], **a)
    q, k, dq, dk = (t[n].clone() for n in ("q", "k", "dq", "dk"))
    ops.head_norm(q, k, out=(q, k), **a)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    ops.head_norm_backward(dq, dk, t["q"], t["k"], out=(dq, dk), **a)
    assert torch.equal(dq, grads["dq"]) and torch.equal(dk, grads["dk"])


@pytest.mark.parametrize("prec", PRECS)
def test_head_norm_masked_rows_and_absent_gradients(prec):
    """NaN in masked rows (positions too far to matter) reaches nothing; all rows masked; no gradient of one part."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(4)
    t = inputs(rng, 12, 3, 2, 48, prec)
    valid = np.ones(12, np.uint8)
    valid[[0, 5, 11]] = 0
    for n in ("q", "k", "dq", "dk"):
        t[n][0], t[n][5], t[n][11] = float("nan"), float("inf"), float("-inf")
    clean = {n: x.clone() for n, x in t.items()}
    for n in ("q", "k", "dq", "dk"):
        clean[n][[0, 5, 11]] = 0.0
    a = dict(w_q=t["w_q"], w_k=t["w_k"], valid=torch.from_numpy(valid).cuda(), norm="layer")
    y, g = ops.head_norm(t["q"], t["k"], **a), ops.head_norm_backward(t["dq"], t["dk"], t["q"], t["k"], **a)
    y0, g0 = ops.head_norm(clean["q"], clean["k"], **a), ops.head_norm_backward(clean["dq"], clean["dk"], clean["q"], clean["k"], **a)
    assert torch.equal(y[0], y0[0]) and torch.equal(y[1], y0[1]) and not y[0][[0, 5, 11]].any()
    for n in g:
        assert g[n] is None or (torch.equal(g[n], g0[n]) and torch.isfinite(g[n].float()).all())
    a["valid"] = torch.zeros(12, dtype=torch.bool, device="cuda")
    y, g = ops.head_norm(t["q"], t["k"], **a), ops.head_norm_backward(t["dq"], t["dk"], t["q"], t["k"], **a)
    assert not y[0].any() and not y[1].any() and not any(x.any() for x in g.values() if x is not None)
    a["valid"] = None
    g = ops.head_norm_backward(None, clean["dk"], clean["q"], clean["k"], **a)
    g0 = ops.head_norm_backward(clean["dq"], clean["dk"], clean["q"], clean["k"], **a)
    assert not g["dq"].any() and not g["dw_q"].any() and torch.equal(g["dk"], g0["dk"]) and torch.equal(g["dw_k"], g0["dw_k"])


def test_head_norm_offsets_past_32_bits():
    """Rows 2^31 elements and more from the first one."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(7)
    t = inputs(rng, 5, 2, 2, 64, "bf16")
    a = dict(w_q=t["w_q"], w_k=t["w_k"], positions=torch.arange(5, dtype=torch.int32, device="cuda"), freqs=ops.rotation_freqs(64))
    want, grads = ops.head_norm(t["q"], t["k"], **a), ops.head_norm_backward(t["dq"], t["dk"], t["q"], t["k"], **a)
    step = 900_000_000
    wide = torch.empty(5 * step, dtype=torch.bfloat16, device="cuda")

    def far(x, at):
        return wide[at:].as_strided((5, 2, 64), (step, 64, 1)).copy_(x)

    q, k, dq, dk = (far(t[n], 1000 * i) for i, n in enumerate(("q", "k", "dq", "dk")))
    outs = tuple(far(torch.zeros_like(t["q"]), 5000 + 1000 * i) for i in range(4))
    got, g = ops.head_norm(q, k, out=outs[:2], **a), ops.head_norm_backward(dq, dk, q, k, out=outs[2:], **a)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert all(grads[n] is None or torch.equal(g[n], grads[n]) for n in grads)
    del wide


def test_head_norm_of_nothing():
    from paper_2312_06126_amd import ops
    torch = torch_()
    for shape in ((0, 4, 64), (5, 0, 64), (5, 4, 0)):
        q = torch.ones(shape, device="cuda")
        w = torch.ones(shape[2], device="cuda")
        y, k = ops.head_norm(q, w_q=w)
        g = ops.head_norm_backward(q, None, q, w_q=w)
        assert y.shape == q.shape and k is None and not g["dw_q"].any()


def test_head_norm_gradient_against_differences():
    """Float32, one direction: the change of a weighted sum of the outputs, in float64 from the kernel's rounded outputs, is the
    gradients' product with it (steps of 1/32: 2^-10 of the second order, roundings 2^-24 * 32 of the sum's terms)."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(5)
    t = inputs(rng, 8, 2, 2, 40, "fp32")
    a = dict(norm="layer", pairs="neighbours", positions=torch.arange(8, dtype=torch.int32, device="cuda"), freqs=torch.from_numpy(freqs_of(15)).cuda())
    x = {n: t[n] for n in ("q", "k", "w_q", "b_q", "w_k", "b_k")}
    g = ops.head_norm_backward(t["dq"], t["dk"], **x, **a)
    for n in x:
        d = gpu(rng.standard_normal(x[n].shape))
        h = 1.0 / 32

        def loss(s):
            yq, yk = ops.head_norm(**dict(x, **{n: x[n] + s * d}), **a)
            return float((yq.double() * t["dq"].double()).sum() + (yk.double() * t["dk"].double()).sum())

        diff = (8 * (loss(h) - loss(-h)) - (loss(2 * h) - loss(-2 * h))) / (12 * h)
        dot = float((g["d" + n].double() * d.double()).sum())
        size = float((g["d" + n].double() * d.double()).abs().sum())
        assert abs(diff - dot) < 2e-3 * size + 1e-4, (n, diff, dot)


@pytest.mark.parametrize("prec", PRECS)
def test_head_norm_streams_and_graphs(prec):
    """On another stream, and captured and replayed with eager work between the replays: the same bits."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(6)
    t = inputs(rng, 200, 4, 2, 64, prec)
    a = dict(w_q=t["w_q"], w_k=t["w_k"], positions=torch.arange(200, dtype=torch.int32, device="cuda"), freqs=ops.rotation_freqs(64))
    want = ops.head_norm(t["q"], t["k"], **a)
    grads = ops.head_norm_backward(t["dq"], t["dk"], t["q"], t["k"], **a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = ops.head_norm(t["q"], t["k"], **a, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ops.head_norm(t["q"], t["k"], **a)
        g = ops.head_norm_backward(t["dq"], t["dk"], t["q"], t["k"], **a)
    for _ in range(3):
        for x in (*y, *(x for x in g.values() if x is not None)):
            x.fill_(7.0)
        graph.replay()
        again = ops.head_norm_backward(t["dq"], t["dk"], t["q"], t["k"], **a)
        torch.cuda.synchronize()
        assert torch.equal(y[0], want[0]) and torch.equal(y[1], want[1])
        for n in grads:
            assert grads[n] is None or (torch.equal(g[n], grads[n]) and torch.equal(again[n], grads[n]))
