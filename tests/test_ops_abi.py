"""The recurrent block's operators without a GPU: struct layouts, refusals before any device call,
workspace sizes, and the float64 references against differences."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from . import ops_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ODD = 3                     # an address that is aligned to nothing
PTR = 1 << 20               # an address that is never followed: every call here is refused


@pytest.fixture(scope="module")
def lib():
    from paper_2312_06126_amd import spz
    return spz.load()


def test_struct_layouts_match_the_header(tmp_path):
    from paper_2312_06126_amd import spz
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not installed")
    mirrors = (("spz_scan_args", spz.ScanArgs), ("spz_block_norm_args", spz.BlockNormArgs))
    body = "".join('printf("%%zu\\n", offsetof(%s, %s));' % (c, f) for c, m in mirrors for f, _ in m._fields_)
    body += "".join('printf("%%zu\\n", sizeof(%s));' % c for c, _ in mirrors)
    src = tmp_path / "layout.c"
    src.write_text('#include "%s"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) { %s return 0; }'
                   % (os.path.join(ROOT, "include", "spz.h"), body))
    subprocess.run([gcc, str(src), "-o", str(tmp_path / "layout")], check=True)
    got = [int(s) for s in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()]
    want = [getattr(m, f).offset for _, m in mirrors for f, _ in m._fields_] + [ctypes.sizeof(m) for _, m in mirrors]
    assert got == want


def scan_args(**kw):
    from paper_2312_06126_amd import spz
    a = spz.ScanArgs(batch=4, steps=8, width=16, f=PTR, v=PTR, y=PTR, df=PTR, dv=PTR, saved=PTR)
    for k in ("f", "v", "y", "dy", "df", "dv"):
        setattr(a, k + "_batch", 128)
        setattr(a, k + "_step", 16)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad,word", [
    (dict(prec=2), "precision"), (dict(batch=-1), "extent"), (dict(steps=1 << 31), "extent"),
    (dict(batch=1 << 30, width=1 << 30), "range"), (dict(f=None), "NULL"), (dict(v=None), "NULL"),
    (dict(f=PTR + ODD), "aligned"), (dict(h0=PTR + ODD), "aligned"), (dict(lengths=PTR + ODD), "aligned"),
    (dict(f_step=-1), "stride"), (dict(v_batch=1 << 60), "stride"), (dict(reset=PTR, reset_step=-4), "stride")])
def test_scan_refusals_of_both_directions(lib, bad, word):
    from paper_2312_06126_amd import spz
    a = scan_args(**bad)
    for call in (lib.spz_scan_forward, lib.spz_scan_backward):
        assert call(ctypes.byref(a), None, 0, None) == spz.SPZ_EINVAL
        assert word in lib.spz_last_error(None).decode()


@pytest.mark.parametrize("call,bad,word", [
    ("forward", dict(y=None), "NULL y"), ("forward", dict(y=PTR + 1), "aligned"), ("forward", dict(y_step=15), "overlap"),
    ("forward", dict(y_batch=127), "overlap"), ("forward", dict(hT=PTR + 2), "aligned"),
    ("backward", dict(df=None), "NULL df"), ("backward", dict(saved=None), "NULL saved"),
    ("backward", dict(dv_step=0), "overlap"), ("backward", dict(df_batch=16), "overlap"),
    ("backward", dict(dy=PTR + 1), "aligned"), ("backward", dict(dy=PTR, dy_step=-1), "stride")])
def test_scan_refusals_of_one_direction(lib, call, bad, word):
    from paper_2312_06126_amd import spz
    assert getattr(lib, "spz_scan_" + call)(ctypes.byref(scan_args(**bad)), None, 0, None) == spz.SPZ_EINVAL
    assert word in lib.spz_last_error(None).decode()


def test_scan_needs_its_workspace(lib):
    from paper_2312_06126_amd import spz
    a = scan_args(batch=1, steps=4096, f_batch=4096 * 16)
    for back, call in ((0, lib.spz_scan_forward), (1, lib.spz_scan_backward)):
        need = lib.spz_scan_workspace(ctypes.byref(a), back)
        assert need > 0
        assert call(ctypes.byref(a), None, need, None) == spz.SPZ_ESIZE
        assert call(ctypes.byref(a), PTR, need - 1, None) == spz.SPZ_ESIZE
        assert call(ctypes.byref(a), PTR + 4, need, None) == spz.SPZ_EINVAL
    assert lib.spz_scan_saved(None) == spz.SPZ_EINVAL and lib.spz_scan_workspace(None, 0) == spz.SPZ_EINVAL
    assert lib.spz_scan_forward(None, None, 0, None) == spz.SPZ_EINVAL


def norm_args(**kw):
    from paper_2312_06126_amd import spz
    a = spz.BlockNormArgs(rows=4, width=16, x=PTR, h=PTR, z=PTR, x_row=16, h_row=16, z_row=16, x_out=PTR, u=PTR, x_out_row=16,
                          u_row=16, dx=PTR, dh=PTR, dz=PTR, dx_row=16, dh_row=16, dz_row=16, eps=1e-6, post=1, pre=1, gate=1)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("back,bad,word", [
    (None, dict(prec=-1), "precision"), (None, dict(rows=-1), "extent"), (None, dict(width=1 << 31), "extent"),
    (None, dict(post=3), "norm"), (None, dict(pre=-1), "norm"), (None, dict(gate=7), "gate"), (None, dict(eps=0.0), "eps"),
    (None, dict(eps=float("nan")), "eps"), (None, dict(drop_p=1.5), "drop_p"), (None, dict(drop_p=float("nan")), "drop_p"),
    (None, dict(x=None), "NULL x"), (None, dict(z=None), "NULL z"), (None, dict(x=PTR + ODD), "aligned"),
    (None, dict(w_pre=PTR + ODD), "aligned"), (None, dict(h_row=-1), "stride"), (None, dict(h=None, pre=0), "neither"),
    (False, dict(x_out=None), "NULL output"), (False, dict(u=None), "NULL output"), (False, dict(u_row=15), "overlap"),
    (True, dict(dx_row=0), "overlap"), (True, dict(dz_row=3), "overlap"), (True, dict(du=PTR, du_row=-5), "stride")])
def test_block_norm_refusals(lib, back, bad, word):
    from paper_2312_06126_amd import spz
    a = norm_args(**bad)
    if back in (None, False):
        assert lib.spz_block_norm_forward(ctypes.byref(a), None) == spz.SPZ_EINVAL
        assert word in lib.spz_last_error(None).decode()
    if back in (None, True):
        assert lib.spz_block_norm_backward(ctypes.byref(a), PTR, 1 << 40, None) == spz.SPZ_EINVAL
        assert word in lib.spz_last_error(None).decode()


def test_block_norm_needs_its_workspace(lib):
    from paper_2312_06126_amd import spz
    a = norm_args()
    need = lib.spz_block_norm_workspace(ctypes.byref(a))
    assert need > 0
    assert lib.spz_block_norm_backward(ctypes.byref(a), None, need, None) == spz.SPZ_ESIZE
    assert lib.spz_block_norm_backward(ctypes.byref(a), PTR, need - 1, None) == spz.SPZ_ESIZE
    assert lib.spz_block_norm_backward(ctypes.byref(a), PTR + 8, need, None) == spz.SPZ_EINVAL


@pytest.mark.parametrize("kw", [
    dict(prec=2), dict(rows=-1), dict(width=-1), dict(x=None), dict(y=None), dict(x=PTR + 1), dict(y=PTR + 2),
    dict(x_row=-1), dict(y_row=7), dict(p=-0.1), dict(p=1.1), dict(p=float("nan"))])
def test_dropout_refusals(lib, kw):
    from paper_2312_06126_amd import spz
    d = dict(prec=0, rows=4, width=8, x=PTR, x_row=8, y=PTR, y_row=8, p=0.5, seed=1, step=2, tensor=3, stream=None)
    d.update(kw)
    assert lib.spz_dropout(*d.values()) == spz.SPZ_EINVAL
    assert b"spz_dropout" in lib.spz_last_error(None)


@pytest.mark.parametrize("kw,code", [
    (dict(prec=9), -1), (dict(rows=-1), -1), (dict(outer=1 << 31), -1), (dict(inner=131073), -1), (dict(x=None), -1),
    (dict(image=None), -1), (dict(w_scale=None), -1), (dict(y=None), -1), (dict(x=PTR + 1), -1), (dict(image=PTR + 8), -1),
    (dict(bias=PTR + 2), -1), (dict(x_row=-1), -1), (dict(y_row=31), -1), (dict(ws=None), -4), (dict(n=0), -4)])
def test_quant_refusals(lib, kw, code):
    # A shape whose rows go through the workspace.
    d = dict(prec=0, rows=512, outer=32, inner=8192, x=PTR, x_row=8192, image=PTR, w_scale=PTR, bias=None, y=PTR, y_row=32, ws=PTR,
             n=1 << 40, stream=None)
    d.update(kw)
    assert lib.spz_quant_linear(*d.values()) == code
    assert b"spz_quant_linear" in lib.spz_last_error(None)


def test_quant_rows_and_pack_refusals(lib):
    assert lib.spz_quant_rows(0, 4, 8, None, 8, PTR, 8, PTR, None) == -1
    assert lib.spz_quant_rows(0, 4, 8, PTR, 8, PTR, 7, PTR, None) == -1
    assert lib.spz_quant_rows(0, 4, 8, PTR, 8, PTR, 8, None, None) == -1
    assert lib.spz_quant_pack(4, 8, None, 8, PTR, None) == -1
    assert lib.spz_quant_pack(4, 8, PTR, -8, PTR, None) == -1
    assert lib.spz_quant_pack(4, 8, PTR, 8, PTR + 1, None) == -1
    assert lib.spz_quant_image_bytes(-1, 8) == -1
    assert lib.spz_quant_image_bytes(33, 33) == 4 * 1024


def test_empty_calls_need_no_arrays(lib):
    from paper_2312_06126_amd import spz
    a = spz.ScanArgs(batch=0, steps=5, width=7)
    assert lib.spz_scan_forward(ctypes.byref(a), None, 0, None) == 0
    assert lib.spz_scan_backward(ctypes.byref(a), None, 0, None) == 0
    assert lib.spz_scan_saved(ctypes.byref(a)) == 0
    n = spz.BlockNormArgs(rows=3, width=0, eps=1e-6, pre=1)
    assert lib.spz_block_norm_forward(ctypes.byref(n), None) == 0
    assert lib.spz_dropout(0, 0, 8, None, 8, None, 8, 0.5, 1, 2, 3, None) == 0
    assert lib.spz_quant_linear(0, 0, 8, 8, None, 8, None, None, None, None, 8, PTR, 1 << 20, None) == 0


# ----------------------------------------------------------------------------- references against differences

def directional(fn, inputs, grads, rng, rel=1e-6):
    """d/de fn(inputs + e direction) against the gradients' inner product with the direction (central
    differences with e = 1e-5: error about e^2 and 1e-16 / e)."""
    for k in grads:
        d = rng.standard_normal(inputs[k].shape)
        e = 1e-5
        up, down = dict(inputs), dict(inputs)
        up[k], down[k] = inputs[k] + e * d, inputs[k] - e * d
        diff = (fn(up) - fn(down)) / (2 * e)
        dot = float((grads[k] * d).sum())
        assert abs(diff - dot) <= rel * (1.0 + abs(dot)) * 10, (k, diff, dot)


def test_scan_reference_gradients():
    rng = np.random.default_rng(0)
    B, T, D = 3, 7, 4
    reset = rng.random((B, T)) < 0.3
    lengths = np.array([7, 0, 4])
    inp = dict(f=rng.standard_normal((B, T, D)), v=rng.standard_normal((B, T, D)), h0=rng.standard_normal((B, D)))
    wy, wh = rng.standard_normal((B, T, D)), rng.standard_normal((B, D))

    def loss(i):
        o = ref.scan(i["f"], i["v"], i["h0"], reset, lengths)
        return float((o["y"][0] * wy).sum() + (o["hT"][0] * wh).sum())

    o = ref.scan(inp["f"], inp["v"], inp["h0"], reset, lengths, wy, wh)
    directional(loss, inp, {k: o["d" + k][0] for k in inp}, rng)


@pytest.mark.parametrize("post,pre,gate", [("rms", "rms", "silu"), ("layer", "layer", "sigmoid"), ("none", "rms", "none"),
                                           ("layer", "none", "silu")])
def test_block_norm_reference_gradients(post, pre, gate):
    rng = np.random.default_rng(1)
    R, D = 4, 6
    valid = np.array([1, 0, 1, 1])
    factor = ref.drop_factor((R, D), 0.4, 99, 3, 1)
    inp = {k: rng.standard_normal((R, D)) for k in ("x", "h", "z")}
    inp.update({k: rng.standard_normal(D) for k in ("w_post", "b_post", "scale", "w_pre", "b_pre")})
    wx, wu = rng.standard_normal((R, D)), rng.standard_normal((R, D))
    opts = dict(post=post, pre=pre, gate_kind=gate, factor=factor, valid=valid, eps=1e-3)

    def loss(i):
        o = ref.block_norm(**i, **opts)
        return float((o["x_out"][0] * wx).sum() + ((o["u"][0] * wu).sum() if pre != "none" else 0.0))

    o = ref.block_norm(**inp, **opts, dx_out=wx, du=wu)
    names = [k for k in inp if not (k == "z" and gate == "none") and not (k in ("w_post", "b_post") and post == "none")
             and not (k in ("w_pre", "b_pre") and pre == "none")]
    directional(loss, inp, {k: o["d" + k][0] for k in names}, rng)


def test_dropout_words_match_the_oracle_generator():
    from oracle import philox
    seed, step, tensor = 0x1234567890ABCDEF, 41, 3
    words = ref.philox16(64, seed, step, tensor)
    full = philox.words(seed, 32, step, 5, tensor)
    assert [int(w) & 0xFFFF for w in full] == list(words[0::2])
    assert [int(w) >> 16 for w in full] == list(words[1::2])
