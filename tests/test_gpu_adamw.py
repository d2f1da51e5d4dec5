"""AdamW over many tensors on the GPU against float64 (more_ops_reference.py), with its bounds; the 8-bit codes against
the definition's own rounding."""
import numpy as np
import pytest

from . import more_ops_reference as ref
from .helpers import log
from .ops_reference import U, rounded
from .test_gpu_ops import PRECS, check, dtype, gpu, host, torch_

pytestmark = pytest.mark.gpu
SEED = 0xFEDCBA9876543210


def make(rng, sizes, prec, gprec, bits, copies=False, **kw):
    from paper_2312_06126_amd import ops
    torch = torch_()
    params = [gpu(rng.standard_normal(n), prec) for n in sizes]
    grads = [gpu(rng.standard_normal(n) * 10.0 ** rng.uniform(-4, 0), gprec) for n in sizes]
    to = [torch.full((n if isinstance(n, int) else tuple(n),), 9.0, dtype=torch.bfloat16, device="cuda") if i % 2 == 0 else None
          for i, n in enumerate(sizes)] if copies else None
    opt = ops.AdamW(params, bits=bits, copies=to, weight_decay=[0.1 * (i % 3) for i in range(len(sizes))], seed=SEED, **kw)
    return params, grads, opt


def fill(rng, opt, bits):
    """Moments of a run some steps old."""
    torch = torch_()
    n = opt.m.numel()
    m, r = rng.standard_normal(n) * 0.01, np.abs(rng.standard_normal(n)) * 0.02
    if bits == 32:
        opt.m.copy_(gpu(m))
        opt.v.copy_(gpu(r * r))
        return
    s = rng.uniform(1e-6, 1e-4, n // 256)
    opt.m_scale.copy_(gpu(s))
    opt.v_scale.copy_(gpu(s[::-1].copy()))
    opt.m.copy_(gpu(np.clip(m * 2e4, -448, 448)).to(torch.float8_e4m3fn))
    opt.v.copy_(gpu(np.clip(r * 1e4, 0, 448)).to(torch.float8_e4m3fn))


def codes(t):
    return t.view(torch_().uint8).cpu().numpy()


def state_of(opt, bits):
    """Moments as float64, with m and v's own values."""
    if bits == 32:
        return host(opt.m), host(opt.v)
    m = ref.e4m3(codes(opt.m)) * host(opt.m_scale).repeat(256)
    return m, (ref.e4m3(codes(opt.v)) * host(opt.v_scale).repeat(256)) ** 2


def check_rounding(name, got, scale, value, bound, words, floor):
    """Codes and scale of one block against the definition: the code is that of some x within the arithmetic's error."""
    most = np.abs(value).max()
    i = int(np.abs(value).argmax())
    assert abs(scale - most / 448) <= 2 * (bound.max() / 448 + 2 * U * most / 448) + 1e-44, (name, scale, most / 448, i)
    got = ref.e4m3(got)
    if scale == 0:
        assert not got.any()
        return
    x = np.abs(value) / scale
    e = 2 * bound / scale + 4 * U * x
    lo, hi = ref.round_random(np.maximum(x - e, 0.0), words), ref.round_random(x + e, words)
    if floor:
        lo, hi = (np.where(x + e > 0, np.maximum(z, 2.0 ** -9), z) for z in (lo, hi))
        lo = np.where(x - e > 0, lo, 0.0)
    a = np.abs(got)
    assert np.all((a >= lo) & (a <= hi)), (name, np.flatnonzero((a < lo) | (a > hi))[:5])
    assert np.mean(lo != hi) < 0.01
    sure = (np.abs(value) > bound) & (got != 0)
    assert np.all(np.sign(got[sure]) == np.sign(value[sure]))


def check_step(rng, params, grads, opt, bits, prec, t, lr, clip=None, betas=(0.9, 0.99), eps=1e-6, step=None, lr_arg=None):
    torch = torch_()
    before = [host(p) for p in params]
    m0, v0 = state_of(opt, bits)
    raw = (codes(opt.m).copy(), codes(opt.v).copy()) if bits == 8 else (host(opt.m), host(opt.v))
    scales = (host(opt.m_scale), host(opt.v_scale)) if bits == 8 else None
    versions = [p._version for p in params]
    opt.step(grads, step=t if step is None else step, lr=lr if lr_arg is None else lr_arg, betas=betas, eps=eps,
             grad_scale=None if clip is None else torch.full((1,), clip, device="cuda"))
    torch.cuda.synchronize()
    seen = np.zeros(opt.m.numel(), bool)
    for i, (p, g) in enumerate(zip(params, grads)):
        n, at = p.numel(), opt.places[i]
        if g is None:
            assert np.array_equal(host(p), before[i]) and p._version == versions[i]
            continue
        assert n == 0 or p._version > versions[i]
        sl = slice(at, at + n)
        seen[sl] = True
        gx = host(g).reshape(-1) * (1.0 if clip is None else float(np.float32(clip)))
        want = ref.adamw(before[i].reshape(-1), gx, m0[sl], v0[sl], t, float(np.float32(lr)), betas[0], betas[1], eps, float(np.float32(opt.weight_decay[i])))
        check("p%d" % i, host(p).reshape(-1), want["p"], prec)
        if opt.copies[i] is not None:
            check("copy%d" % i, host(opt.copies[i]).reshape(-1), want["p"], "bf16")
        if bits == 32:
            check("m%d" % i, host(opt.m)[sl], want["m"], "fp32")
            check("v%d" % i, host(opt.v)[sl], want["v"], "fp32")
            continue
        wm, wv = ref.moment_words(np.arange(at, at + n), SEED, t)
        for b in range(at, at + n, 256):
            c = slice(b, min(b + 256, at + n))
            o = slice(b - at, c.stop - at)
            check_rounding("m%d block %d" % (i, b), codes(opt.m)[c], host(opt.m_scale)[b // 256], want["m"][0][o], want["m"][1][o], wm[o], False)
            check_rounding("v%d block %d" % (i, b), codes(opt.v)[c], host(opt.v_scale)[b // 256], want["r"][0][o], want["r"][1][o], wv[o], True)
    now = (codes(opt.m), codes(opt.v)) if bits == 8 else (host(opt.m), host(opt.v))
    for a, b in zip(raw, now):
        assert np.array_equal(a[~seen], b[~seen])       # what no tensor holds stays
    if bits == 8:
        blocks = seen.reshape(-1, 256).any(1)
        for a, b in zip(scales, (opt.m_scale, opt.v_scale)):
            assert np.array_equal(a[~blocks], host(b)[~blocks])


SIZES = [[1], [255, 256, 257], [2048, 2049, 7, 4096 + 3], [5, 0, 1000, 1, 300000, 9]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gprec", PRECS)
@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_adamw(sizes, prec, gprec, bits):
    log("adamw %s %s %s %d" % (sizes, prec, gprec, bits))
    rng = np.random.default_rng(sum(sizes) + bits)
    params, grads, opt = make(rng, sizes, prec, gprec, bits, copies=prec == "fp32")
    check_step(rng, params, grads, opt, bits, prec, 1, 1e-2)                    # from zeros
    fill(rng, opt, bits)
    for t, clip in ((2, None), (41, 0.37), (100000, 1.0)):
        check_step(rng, params, grads, opt, bits, prec, t, 3e-3, clip)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_many_tensors_of_mixed_types(bits):
    """More tensors than one launch takes, in both types, some without a gradient, with shapes."""
    from paper_2312_06126_amd import ops
    rng = np.random.default_rng(3)
    sizes = [int(n) for n in rng.integers(0, 700, 150)]
    params = [gpu(rng.standard_normal(n), PRECS[i % 2]) for i, n in enumerate(sizes)]
    params[7], params[8] = gpu(rng.standard_normal((30, 41))), gpu(rng.standard_normal((3, 5, 7)), "bf16")
    grads = [gpu(rng.standard_normal(tuple(p.shape)) * 0.1, PRECS[i % 3 % 2]) for i, p in enumerate(params)]
    opt = ops.AdamW(params, bits=bits, weight_decay=0.01, seed=SEED)
    fill(rng, opt, bits)
    for i in range(0, 150, 13):
        grads[i] = None
    torch = torch_()
    before, (m0, v0) = [host(p).reshape(-1) for p in params], state_of(opt, bits)
    opt.step(grads, step=5, lr=1e-3)
    torch.cuda.synchronize()
    for i, (p, g) in enumerate(zip(params, grads)):
        if g is None:
            assert np.array_equal(host(p).reshape(-1), before[i])
            continue
        sl = slice(opt.places[i], opt.places[i] + p.numel())
        want = ref.adamw(before[i], host(g).reshape(-1), m0[sl], v0[sl], 5, float(np.float32(1e-3)), 0.9, 0.999, 1e-8, float(np.float32(0.01)))
        check("p%d" % i, host(p).reshape(-1), want["p"], "fp32" if p.dtype == torch.float32 else "bf16")


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_steps_and_rates_on_the_device(bits):
    """Step count, rate and gradient scale in tensors, in a captured graph that counts its own steps: each replay is
    the eager step of that number, bit for bit where the corrections are."""
    torch = torch_()
    rng = np.random.default_rng(4)
    params, grads, opt = make(rng, [1000, 77, 5000], "fp32", "bf16", bits)
    fill(rng, opt, bits)
    t, lr, clip = torch.tensor([6], device="cuda"), torch.tensor(1e-2, device="cuda"), torch.full((1,), 0.5, device="cuda")
    saved = [x.clone() for x in (*params, opt.m, opt.v) + ((opt.m_scale, opt.v_scale) if bits == 8 else ())]

    def restore():
        for x, y in zip((*params, opt.m, opt.v) + ((opt.m_scale, opt.v_scale) if bits == 8 else ()), saved):
            x.copy_(y)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.add_(1)
        opt.step(grads, step=t, lr=lr, grad_scale=clip)
    restore()
    t.fill_(6)
    got = []
    for i in range(4):
        lr.fill_(1e-2 / (i + 1))
        graph.replay()
        got.append([p.clone() for p in params])
        torch.cuda.synchronize()
    restore()
    for i in range(4):
        opt.step(grads, step=7 + i, lr=float(np.float32(1e-2 / (i + 1))), grad_scale=clip)
        for p, q in zip(params, got[i]):
            assert torch.allclose(p, q, rtol=4 * U, atol=2e-2 * 16 * U)    # corrections from the device's own powers: an ulp each
    restore()
    check_step(rng, params, grads, opt, bits, "fp32", 9, 1e-2, 0.5, step=torch.tensor(9, device="cuda"), lr_arg=torch.tensor([1e-2], device="cuda"))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_places_past_32_bits(bits):
    """Moments behind 2^32 + elements of others: the second tensor, against the same one by itself (32 bits) or its definition."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(8)
    big = torch.zeros((1 << 32) + 512, dtype=torch.bfloat16, device="cuda")
    small = gpu(rng.standard_normal(1000))
    opt = ops.AdamW([big, small], bits=bits, seed=SEED)
    at = opt.places[1]
    assert at == (1 << 32) + 512
    g = gpu(rng.standard_normal(1000) * 0.1)
    before = host(small)
    opt.step([None, g], step=3, lr=1e-2)
    torch.cuda.synchronize()
    zero = np.zeros(1000)
    want = ref.adamw(before, host(g), zero, zero, 3, float(np.float32(1e-2)), 0.9, 0.999, 1e-8, 0.0)
    check("p", host(small), want["p"], "fp32")
    if bits == 32:
        check("m", host(opt.m[at:at + 1000]), want["m"], "fp32")
        check("v", host(opt.v[at:at + 1000]), want["v"], "fp32")
    else:
        wm, wv = ref.moment_words(np.arange(at, at + 1000), SEED, 3)
        for b in range(0, 1000, 256):
            c, i = slice(b, min(b + 256, 1000)), (at + b) // 256
            check_rounding("m", codes(opt.m[at:at + 1000])[c], float(opt.m_scale[i]), want["m"][0][c], want["m"][1][c], wm[c], False)
            check_rounding("v", codes(opt.v[at:at + 1000])[c], float(opt.v_scale[i]), want["r"][0][c], want["r"][1][c], wv[c], True)
    del opt, big


def test_adamw_rounding_is_fair():
    """Moments that change by a hundredth a step in 8 bits: after 400 steps the mean follows the exact moments, which rounding to
    nearest would leave where they are. 4096 elements; the root's standard deviation is below 0.2 of itself (steps
    of at most an eighth, forgotten at 1 - beta), so the mean's is 0.004: 0.05 is over ten of them."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    p = torch.zeros(4096, device="cuda")
    opt = ops.AdamW([p], bits=8, seed=5)
    g = torch.ones(4096, device="cuda")
    g[::256] = 3.0
    v = np.zeros(1)
    for t in range(1, 401):
        s = 1.0 if t <= 200 else 1.3
        opt.step([g * s], step=t, lr=0.0, betas=(0.99, 0.99))
        v = 0.99 * v + 0.01 * s * s
    got = ref.e4m3(codes(opt.v)) * host(opt.v_scale).repeat(256)
    got_m = ref.e4m3(codes(opt.m)) * host(opt.m_scale).repeat(256)
    rest = np.ones(4096, bool)
    rest[::256] = False
    m = 0.0
    for t in range(1, 401):
        m = 0.99 * m + 0.01 * (1.0 if t <= 200 else 1.3)
    assert abs(np.mean(got[rest] ** 2) / v[0] - 1) < 0.1 and abs(got_m[rest].mean() / m - 1) < 0.05


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_values_that_are_not_finite(bits):
    """They reach their own element, and in 8 bits their block's scale; everything else is as without them."""
    torch = torch_()
    rng = np.random.default_rng(6)
    params, grads, opt = make(rng, [1000, 300], "fp32", "fp32", bits)
    fill(rng, opt, bits)
    base = [x.clone() for x in (*params, opt.m.float(), opt.v.float())]
    state = [opt.m.clone(), opt.v.clone()] + ([opt.m_scale.clone(), opt.v_scale.clone()] if bits == 8 else [])
    opt.step(grads, step=3, lr=1e-2)
    want = [x.clone() for x in (*params, opt.m.float(), opt.v.float())]
    for p, b in zip(params, base):
        p.copy_(b)
    for x, y in zip((opt.m, opt.v, opt.m_scale, opt.v_scale), state):
        x.copy_(y)
    grads[0][300], grads[0][700] = float("nan"), float("inf")
    opt.step(grads, step=3, lr=1e-2)
    bad = torch.zeros(1000, dtype=torch.bool, device="cuda")
    bad[[300, 700]] = True
    assert torch.equal(params[1], want[1]) and torch.equal(params[0][~bad], want[0][~bad]) and not torch.isfinite(params[0][bad]).any()
    if bits == 8:
        assert torch.isnan(opt.m_scale[[1, 2]]).all() and torch.isfinite(opt.m_scale[[0, 3]]).all()
        assert not opt.m[256:768].float().any() and torch.equal(opt.m[768:].float(), want[2][768:]) and torch.equal(opt.m[:256].float(), want[2][:256])
    # All zeros stay zeros, and nothing is divided by them.
    for g in grads:
        g.zero_()
    opt.m.zero_()
    opt.v.zero_()
    if bits == 8:
        opt.m_scale.zero_()
        opt.v_scale.zero_()
    before = params[1].clone()
    opt.step(grads, step=1, lr=1e-2)
    assert torch.equal(params[1], before - torch.tensor(1e-2 * np.float32(0.1)).to(before) * before) or torch.allclose(params[1], before * (1 - 1e-3), rtol=4 * U)
    assert not opt.m.float().any() and not opt.v.float().any()


def test_adamw_refusals():
    from paper_2312_06126_amd import ops
    from paper_2312_06126_amd.spz import SPZ_EINVAL, SpzError
    torch = torch_()
    a, b = torch.ones(300, device="cuda"), torch.ones(20, device="cuda")
    opt = ops.AdamW([a, b])
    g = [torch.ones_like(a), torch.ones_like(b)]
    ok = dict(step=1, lr=1e-3)
    wide = torch.ones((4, 6), device="cuda")
    moved = torch.ones(8, device="cuda")
    other = ops.AdamW([moved])
    moved.data = torch.ones(8, device="cuda")
    leaf = torch.ones(300, device="cuda", requires_grad=True)
    for call in (lambda: ops.AdamW([]), lambda: ops.AdamW([a.cpu()]), lambda: ops.AdamW([a.half()]), lambda: ops.AdamW([wide.t()]),
                 lambda: ops.AdamW([a, a]), lambda: ops.AdamW([a, a[5:9]]), lambda: ops.AdamW([a], bits=16), lambda: ops.AdamW([a], weight_decay=[1, 2]),
                 lambda: ops.AdamW([a], weight_decay="x"), lambda: ops.AdamW([a], weight_decay=float("nan")), lambda: ops.AdamW([a], copies=[a]),
                 lambda: ops.AdamW([a], copies=[a.bfloat16()[:5]]), lambda: ops.AdamW([a.bfloat16()], copies=[a.bfloat16()]),
                 lambda: ops.AdamW([a], copies=[]), lambda: ops.AdamW([leaf * 2]),
                 lambda: opt.step([g[0]], **ok), lambda: opt.step(g[0], **ok), lambda: opt.step([g[0], g[0]], **ok), lambda: opt.step([g[0].double(), g[1]], **ok),
                 lambda: opt.step([g[0], g[1].cpu()], **ok), lambda: opt.step([g[0], 1.0], **ok), lambda: opt.step([leaf, g[1]], **ok),
                 lambda: opt.step(g, step=0, lr=1e-3), lambda: opt.step(g, step=None, lr=1e-3), lambda: opt.step(g, step=1, lr="a"),
                 lambda: opt.step(g, step=1, lr=float("inf")), lambda: opt.step(g, **ok, betas=(1.0, 0.9)), lambda: opt.step(g, **ok, betas=0.9),
                 lambda: opt.step(g, **ok, betas=(0.9, float("nan"))), lambda: opt.step(g, **ok, eps=-1.0), lambda: opt.step(g, **ok, grad_scale=2.0),
                 lambda: opt.step(g, step=torch.ones(1, device="cuda"), lr=1e-3), lambda: opt.step(g, step=torch.ones(2, dtype=torch.int64, device="cuda"), lr=1e-3),
                 lambda: opt.step(g, step=torch.ones(1, dtype=torch.int64), lr=1e-3), lambda: opt.step(g, **ok, grad_scale=torch.ones(1)),
                 lambda: other.step([torch.ones(8, device="cuda")], **ok)):
        with pytest.raises(SpzError) as e:
            call()
        assert e.value.code == SPZ_EINVAL
    opt.m = torch.zeros(5, device="cuda")
    with pytest.raises(SpzError):
        opt.step(g, **ok)
    # Leaves that require a gradient are what a learner holds.
    opt = ops.AdamW([leaf])
    opt.step([torch.ones_like(leaf)], **ok)
    assert (leaf < 1.0).all()
