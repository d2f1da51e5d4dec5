"""Head norms, linear attention and AdamW without a GPU: struct layouts, refusals before any device call, workspace sizes,
and the float64 references against differences."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from . import more_ops_reference as ref
from .test_ops_abi import ODD, PTR, ROOT, directional, lib  # noqa: F401


def test_struct_layouts_match_the_header(tmp_path):
    from paper_2312_06126_amd import spz
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not installed")
    mirrors = (("spz_head_norm_args", spz.HeadNormArgs), ("spz_linear_attention_args", spz.LinearAttentionArgs),
               ("spz_adamw_tensor", spz.AdamwTensor), ("spz_adamw_args", spz.AdamwArgs))
    body = "".join('printf("%%zu\\n", offsetof(%s, %s));' % (c, f) for c, m in mirrors for f, _ in m._fields_)
    body += "".join('printf("%%zu\\n", sizeof(%s));' % c for c, _ in mirrors)
    src = tmp_path / "layout.c"
    src.write_text('#include "%s"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) { %s return 0; }'
                   % (os.path.join(ROOT, "include", "spz.h"), body))
    subprocess.run([gcc, str(src), "-o", str(tmp_path / "layout")], check=True)
    got = [int(s) for s in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()]
    want = [getattr(m, f).offset for _, m in mirrors for f, _ in m._fields_] + [ctypes.sizeof(m) for _, m in mirrors]
    assert got == want
    text = open(os.path.join(ROOT, "include", "spz.h")).read()
    assert "#define SPZ_ADAMW_BLOCK %d" % spz.ADAMW_BLOCK in text
    for name, v in spz.PAIRS.items():
        assert "#define SPZ_PAIRS_%s %d" % (name.upper(), v) in text


def head_args(**kw):
    from paper_2312_06126_amd import spz
    a = spz.HeadNormArgs(rows=4, heads_q=3, heads_k=2, dim=16, pairs=8, positions=PTR, freqs=PTR, eps=1e-6, norm=1,
                         **{n: PTR for n in ("q", "k", "q_out", "k_out", "dq_out", "dk_out", "dq", "dk")})
    for n in ("q", "k", "q_out", "k_out", "dq_out", "dk_out", "dq", "dk"):
        setattr(a, n + "_row", 48)
        setattr(a, n + "_head", 16)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("back,bad,word", [
    (None, dict(prec=5), "precision"), (None, dict(rows=-1), "extent"), (None, dict(heads_q=1 << 31), "extent"), (None, dict(dim=1025), "dim"),
    (None, dict(dim=-1), "dim"), (None, dict(pairs=9), "pairs"), (None, dict(pairs=-1), "pairs"), (None, dict(norm=3), "norm"),
    (None, dict(layout=2), "layout"), (None, dict(eps=0.0), "eps"), (None, dict(eps=float("nan")), "eps"), (None, dict(q=None), "NULL q"),
    (None, dict(k=None), "NULL q or k"), (None, dict(positions=None), "positions"), (None, dict(freqs=None), "positions"), (None, dict(q=PTR + ODD), "aligned"),
    (None, dict(freqs=PTR + 4), "aligned"), (None, dict(positions=PTR + 2), "aligned"), (None, dict(b_k=PTR + ODD), "aligned"), (None, dict(k_head=-1), "stride"),
    (None, dict(rows=1 << 30, heads_q=1 << 20), "range"), (False, dict(q_out=None), "NULL output"), (False, dict(k_out_head=15), "overlap"),
    (False, dict(q_out_row=47), "overlap"), (True, dict(dq_head=8), "overlap"), (True, dict(dk_row=16), "overlap"), (True, dict(dq_out_row=-3), "stride")])
def test_head_norm_refusals(lib, back, bad, word):  # noqa: F811
    from paper_2312_06126_amd import spz
    a = head_args(**bad)
    if back in (None, False):
        assert lib.spz_head_norm_forward(ctypes.byref(a), None) == spz.SPZ_EINVAL
        assert word in lib.spz_last_error(None).decode()
    if back in (None, True):
        assert lib.spz_head_norm_backward(ctypes.byref(a), PTR, 1 << 40, None) == spz.SPZ_EINVAL
        assert word in lib.spz_last_error(None).decode()


def test_head_norm_needs_its_workspace(lib):  # noqa: F811
    from paper_2312_06126_amd import spz
    a = head_args()
    need = lib.spz_head_norm_workspace(ctypes.byref(a))
    assert need > 0
    assert lib.spz_head_norm_backward(ctypes.byref(a), None, need, None) == spz.SPZ_ESIZE
    assert lib.spz_head_norm_backward(ctypes.byref(a), PTR, need - 1, None) == spz.SPZ_ESIZE
    assert lib.spz_head_norm_backward(ctypes.byref(a), PTR + 8, need, None) == spz.SPZ_EINVAL
    assert lib.spz_head_norm_workspace(None) == spz.SPZ_EINVAL and lib.spz_head_norm_forward(None, None) == spz.SPZ_EINVAL


def attention_args(**kw):
    from paper_2312_06126_amd import spz
    a = spz.LinearAttentionArgs(batch=2, steps=8, heads=3, key_width=16, value_width=8, scale=0.25,
                                **{n: PTR for n in ("q", "k", "v", "y", "dy", "dq", "dk", "dv", "rate", "state", "last", "dlast", "dstate")})
    for n, w in (("q", 16), ("k", 16), ("v", 8), ("y", 8), ("dy", 8), ("dq", 16), ("dk", 16), ("dv", 8)):
        for s, v in (("_batch", 24 * w), ("_step", 3 * w), ("_head", w)):
            setattr(a, n + s, v)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("back,bad,word", [
    (None, dict(prec=2), "precision"), (None, dict(batch=-1), "extent"), (None, dict(steps=1 << 31), "extent"), (None, dict(heads=-4), "extent"), (None, dict(heads=65537), "extent"),
    (None, dict(key_width=257), "width"), (None, dict(value_width=300), "width"), (None, dict(value_width=-1), "width"), (None, dict(scale=float("inf")), "scale"),
    (None, dict(scale=float("nan")), "scale"), (None, dict(batch=1 << 30, heads=1 << 20), "range"), (None, dict(batch=1 << 20, steps=1 << 30), "range"),
    (None, dict(q=None), "NULL"), (None, dict(v=None), "NULL"), (None, dict(k=PTR + ODD), "aligned"), (None, dict(rate=PTR + 2), "aligned"),
    (None, dict(lengths=PTR + 1), "aligned"), (None, dict(state=PTR + ODD), "aligned"), (None, dict(v_head=-1), "stride"), (None, dict(q_batch=1 << 60), "stride"),
    (None, dict(reset=PTR, reset_step=-1), "stride"), (False, dict(y=None), "NULL y"), (False, dict(y_head=7), "overlap"), (False, dict(y_step=23), "overlap"),
    (False, dict(y_batch=24 * 8 - 1), "overlap"), (True, dict(dq=None), "NULL dq"), (True, dict(dv=None), "NULL dq, dk or dv"), (True, dict(dk_head=0), "overlap"),
    (True, dict(dq_step=16), "overlap"), (True, dict(dv_batch=8), "overlap"), (True, dict(dy_step=-8), "stride"), (True, dict(dlast=PTR + 2), "aligned"),
    (False, dict(y_batch=1 << 41, batch=1 << 22, steps=1, heads=1, key_width=1, value_width=1), "overlap")])
def test_attention_refusals(lib, back, bad, word):  # noqa: F811
    from paper_2312_06126_amd import spz
    a = attention_args(**bad)
    for direction, call in ((False, lib.spz_linear_attention_forward), (True, lib.spz_linear_attention_backward)):
        if back in (None, direction):
            assert call(ctypes.byref(a), PTR, 1 << 50, None) == spz.SPZ_EINVAL
            assert word in lib.spz_last_error(None).decode()


def test_attention_needs_its_workspace(lib):  # noqa: F811
    from paper_2312_06126_amd import spz
    a = attention_args(batch=1, steps=4096)
    for n in ("q", "k", "v", "y", "dy", "dq", "dk", "dv"):
        setattr(a, n + "_batch", 4096 * getattr(a, n + "_step"))
    for back, call in ((0, lib.spz_linear_attention_forward), (1, lib.spz_linear_attention_backward)):
        need = lib.spz_linear_attention_workspace(ctypes.byref(a), back)
        assert need > 0
        assert call(ctypes.byref(a), None, need, None) == spz.SPZ_ESIZE
        assert call(ctypes.byref(a), PTR, need - 1, None) == spz.SPZ_ESIZE
        assert call(ctypes.byref(a), PTR + 4, need, None) == spz.SPZ_EINVAL
    assert lib.spz_linear_attention_workspace(None, 0) == spz.SPZ_EINVAL


def test_attention_output_orders(lib):  # noqa: F811
    """Whatever the order of the outer dimensions, one whose stride is an element short of what it steps over is refused."""
    from itertools import permutations
    n, names = dict(batch=3, steps=70, heads=4), dict(batch="y_batch", steps="y_step", heads="y_head")
    for order in permutations(n):
        for short in order:
            stride, span = {}, 8
            for d in order:
                stride[names[d]] = span - (d == short)
                span += (n[d] - 1) * stride[names[d]]
            a = attention_args(**n, **stride)
            assert lib.spz_linear_attention_forward(ctypes.byref(a), PTR, 1 << 50, None) == -1
            assert b"overlap" in lib.spz_last_error(None), (order, short)


def adamw_args(one=None, **kw):
    from paper_2312_06126_amd import spz
    t = dict(p=PTR, g=PTR, copy=None, n=300, at=256, weight_decay=0.1)
    t.update(one or {})
    host = (spz.AdamwTensor * 2)(spz.AdamwTensor(p=PTR, g=PTR, n=256, at=0), spz.AdamwTensor(**t))
    a = spz.AdamwArgs(count=2, moments=768, tensors=ctypes.addressof(host), m=PTR, v=PTR, m_scale=PTR, v_scale=PTR, step=1, lr=1e-3, beta1=0.9,
                      beta2=0.999, eps=1e-8, bits=8)
    for k, v in kw.items():
        setattr(a, k, v)
    return a, host


@pytest.mark.parametrize("tensor,bad,word", [
    ({}, dict(bits=16), "bits"), ({}, dict(p_prec=3), "precision"), ({}, dict(g_prec=-1), "precision"), ({}, dict(count=-1), "count"), ({}, dict(moments=700), "moments"),
    ({}, dict(moments=-256), "moments"), ({}, dict(beta1=1.0), "beta"), ({}, dict(beta2=-0.1), "beta"), ({}, dict(beta2=float("nan")), "beta"), ({}, dict(eps=-1.0), "eps"),
    ({}, dict(lr=float("inf")), "lr"), ({}, dict(step=0), "step"), ({}, dict(tensors=None), "NULL"), ({}, dict(m=None), "NULL"), ({}, dict(v_scale=None), "NULL"),
    ({}, dict(m=PTR + 4), "aligned"), ({}, dict(step_at=PTR + 4), "aligned"), ({}, dict(lr_at=PTR + 2), "aligned"), ({}, dict(reserved=1), "reserved"),
    (dict(at=255), {}, "outside"), (dict(at=512, n=257), {}, "outside"), (dict(at=-256), {}, "outside"), (dict(n=-1), {}, "outside"), (dict(n=1 << 62), {}, "outside"),
    (dict(p=None), {}, "NULL p"), (dict(g=None), {}, "NULL p"), (dict(p=PTR + 2), {}, "aligned"), (dict(copy=PTR + 1), {}, "aligned"),
    (dict(weight_decay=float("inf")), {}, "weight_decay")])
def test_adamw_refusals(lib, tensor, bad, word):  # noqa: F811
    a, host = adamw_args(tensor, **bad)
    assert lib.spz_adamw(ctypes.byref(a), None) == -1
    assert word in lib.spz_last_error(None).decode(), lib.spz_last_error(None)
    del host


def test_empty_calls_need_no_arrays(lib):  # noqa: F811
    from paper_2312_06126_amd import spz
    a = spz.HeadNormArgs(rows=0, heads_q=2, dim=8, eps=1e-6, norm=1, q_out_row=16, q_out_head=8)
    assert lib.spz_head_norm_forward(ctypes.byref(a), None) == 0
    b = spz.LinearAttentionArgs(batch=0, steps=5, heads=2, key_width=8, value_width=8, scale=1.0)
    assert lib.spz_linear_attention_forward(ctypes.byref(b), None, 0, None) == 0
    assert lib.spz_linear_attention_backward(ctypes.byref(b), None, 0, None) == 0
    c = spz.AdamwArgs(count=0, step=1, lr=1e-3, bits=32)
    assert lib.spz_adamw(ctypes.byref(c), None) == 0
    assert lib.spz_adamw(None, None) == -1 and lib.spz_linear_attention_forward(None, None, 0, None) == -1


# ----------------------------------------------------------------------------- references against differences

@pytest.mark.parametrize("kind,pairs,half", [("rms", "halves", 3), ("layer", "neighbours", 2), ("none", "halves", 1), ("layer", "halves", 0)])
def test_head_norm_reference_gradients(kind, pairs, half):
    rng = np.random.default_rng(0)
    x = dict(x=rng.standard_normal((4, 2, 7)), w=rng.standard_normal(7), b=rng.standard_normal(7))
    dy = rng.standard_normal((4, 2, 7))
    opt = dict(kind=kind, eps=1e-3, pairs=pairs, valid=np.array([1, 0, 1, 1]), positions=np.array([0, 5, 300, -2]) if half else None,
               freqs=np.array([1.0, 0.3, 0.01])[:half] if half else None)
    o = ref.head_norm(**x, **opt, dy=dy)
    directional(lambda i: float((ref.head_norm(**i, **opt)["y"][0] * dy).sum()), x, {n: o["d" + n][0] for n in x}, rng)


def test_attention_reference_gradients():
    rng = np.random.default_rng(1)
    B, T, H, K, V = 3, 9, 2, 4, 3
    x = {n: rng.standard_normal((B, T, H, w)) for n, w in (("q", K), ("k", K), ("v", V))}
    x["state"] = rng.standard_normal((B, H, K, V))
    dy, dlast = rng.standard_normal((B, T, H, V)), rng.standard_normal((B, H, K, V))
    opt = dict(rate=np.array([0.0, 0.4]), scale=0.7, reset=rng.random((B, T)) < 0.3, lengths=np.array([9, 0, 5]))
    o = ref.attention(**x, **opt, dy=dy, dlast=dlast)

    def loss(i):
        f = ref.attention(**i, **opt)
        return float((f["y"][0] * dy).sum() + (f["last"][0] * dlast).sum())

    directional(loss, x, {n: o["d" + n][0] for n in x}, rng)


def test_codes_and_rounding_of_the_reference():
    torch = pytest.importorskip("torch")
    every = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(every).view(torch.float8_e4m3fn).double().numpy()
    got = ref.e4m3(every)
    assert np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)]) and np.array_equal(np.isnan(got), np.isnan(want))
    rng = np.random.default_rng(2)
    values = np.sort(got[(every < 127)])
    words = np.arange(65536)
    for x in list(rng.uniform(0, 448, 20)) + list(2.0 ** rng.uniform(-12, -5, 20)) + [0.0, 448.0, 2.0 ** -6, 2.0 ** -9]:
        z = ref.round_random(np.full(65536, x), words)
        lo = values[values <= x].max()
        hi = values[values >= x].min()
        assert set(np.unique(z)) <= {lo, hi}
        assert abs(z.mean() - x) <= (hi - lo) * 2.0 ** -15 + 2.0 ** -29


def test_adamw_reference_is_torchs():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(3)
    p = torch.from_numpy(rng.standard_normal(50)).requires_grad_()
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    x, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = rng.standard_normal(50)
        p.grad = torch.from_numpy(g)
        opt.step()
        o = ref.adamw(x, g, m, v, t, 1e-2, 0.8, 0.95, 1e-6, 0.1)
        x, m, v = o["p"][0], o["m"][0], o["v"][0]
        assert np.allclose(x, p.detach().numpy(), rtol=1e-12, atol=1e-13)
