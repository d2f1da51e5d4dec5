"""Arrays that share elements, without a GPU: the rule against all places of small arrays, and the calls' refusals."""
import ctypes
import itertools

import numpy as np
import pytest

from .test_more_ops_abi import attention_args, head_args
from .test_ops_abi import PTR, lib  # noqa: F401


def places(at, width, n, s):
    """Every element's place."""
    i = np.array(list(itertools.product(*(range(x) for x in n)))).reshape(-1, 3) @ np.array(s)
    return (at + i[:, None] + np.arange(width)[None]).ravel()


def ask(lib, size, x, y):  # noqa: F811
    def array(at, width, n, s):
        return ctypes.c_void_p(PTR + at * size), width, (ctypes.c_int64 * 3)(*n), (ctypes.c_int64 * 3)(*s)

    f = lib.spzt_shares
    f.restype = ctypes.c_int
    f.argtypes = [ctypes.c_int32] + [ctypes.c_void_p, ctypes.c_int64, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)] * 2
    return f(size, *array(*x), *array(*y))


def strides(rng, n, width):
    """Strides of an array without overlaps, in some order of its dimensions, with gaps or without."""
    s, span = [0, 0, 0], width
    gap = rng.integers(0, 2)
    for i in rng.permutation(3):
        s[i] = int(span + gap * rng.integers(0, 4))
        span += (n[i] - 1) * s[i] if gap else span * (n[i] - 1)
    return s


@pytest.mark.parametrize("size", [2, 4])
def test_rule_of_shared_elements(lib, size):  # noqa: F811
    rng = np.random.default_rng(size)
    seen = [0, 0, 0]
    for _ in range(6000):
        n = [int(i) for i in rng.integers(1, 4, 3)]
        w = [int(i) for i in rng.integers(1, 6, 2)]
        s = strides(rng, n, max(w))
        kind = rng.integers(0, 3)          # the same strides; strides of its own; another number in one dimension
        m, t = list(n), list(s)
        if kind == 1:
            t = strides(rng, n, w[1])
        elif kind == 2:
            m[rng.integers(0, 3)] = int(rng.integers(0, 4))
        x, y = places(0, w[0], n, s), None
        at = int(rng.integers(-x.max() - 3, x.max() + 4))
        y = places(at, w[1], m, t) if all(m) else np.array([], int)
        shared = np.intersect1d(x, y).size > 0
        for a, b in (((0, w[0], n, s), (at, w[1], m, t)), ((at, w[1], m, t), (0, w[0], n, s))):
            got = ask(lib, size, a, b)
            # Never found where nothing is shared; always found where strides are the same.
            assert got <= shared, (a, b)
            if kind == 0 or (kind == 1 and x.size == np.ptp(x) + 1 and y.size == np.ptp(y) + 1):
                assert got == shared, (a, b)
                seen[kind] += shared
            seen[2] += kind == 2 and got
    assert min(seen) > 100


def test_arrays_of_nothing_share_nothing(lib):  # noqa: F811
    x = (0, 4, (2, 3, 1), (12, 4, 0))
    assert ask(lib, 4, x, x) == 1
    for y in ((0, 0, (2, 3, 1), (12, 4, 0)), (0, 4, (0, 3, 1), (12, 4, 0))):
        assert ask(lib, 4, x, y) == 0 and ask(lib, 4, y, x) == 0


def apart(args, names, sizes):
    """Each array in a place of its own."""
    for i, (n, size) in enumerate(zip(names, sizes)):
        setattr(args, n, PTR + (i << 20))
        assert size < 1 << 20
    return args


ARRAYS = ("q", "k", "v", "y", "dy", "dq", "dk", "dv", "rate", "state", "last", "dlast", "dstate")


@pytest.mark.parametrize("back,change,word", [
    (False, dict(y="q"), "y shares"), (False, dict(y="k"), "y shares"), (False, dict(y=("v", 4)), "y shares"), (False, dict(y="v", y_head=9, y_step=27, y_batch=216), "y shares"),
    (False, dict(last=("state", 512)), "last shares"),
    (True, dict(dq="dk"), "dq, dk and dv"), (True, dict(dk="dv"), "dq, dk and dv"), (True, dict(dv="dq"), "dq, dk and dv"), (True, dict(dq=("dk", -60)), "dq, dk and dv"),
    (True, dict(dq=("dk", 48 * 7)), "dq, dk and dv"), (True, dict(dq="q"), "dq, dk or dv"), (True, dict(dk="k"), "dq, dk or dv"), (True, dict(dv="v"), "dq, dk or dv"),
    (True, dict(dv="dy"), "dq, dk or dv"), (True, dict(dq="dy"), "dq, dk or dv"), (True, dict(dstate="dlast"), "dstate"), (True, dict(dstate="state"), "dstate"),
    (True, dict(dstate=("dlast", 4 * 767)), "dstate")])
def test_attention_refuses_shared_arrays(lib, back, change, word):  # noqa: F811
    a = apart(attention_args(), ARRAYS, [8192] * len(ARRAYS))
    for n, v in change.items():
        setattr(a, n, getattr(a, v) if isinstance(v, str) else getattr(a, v[0]) + v[1] if isinstance(v, tuple) else v)
    call = lib.spz_linear_attention_backward if back else lib.spz_linear_attention_forward
    assert call(ctypes.byref(a), PTR, 1 << 50, None) == -1
    assert word in lib.spz_last_error(None).decode() and "share" in lib.spz_last_error(None).decode()


@pytest.mark.parametrize("back,change", [
    (False, dict(q_out="k_out")), (False, dict(q_out="k")), (False, dict(k_out="q")), (False, dict(q_out=("q", 64))), (False, dict(k_out=("k", 4))),
    (False, dict(q_out="q", q_out_row=64)), (False, dict(k_out=("q_out", 4 * 16))), (True, dict(dq="dk")), (True, dict(dq="dk_out")), (True, dict(dk="dq_out")),
    (True, dict(dq="k")), (True, dict(dk="q")), (True, dict(dq=("dq_out", 4))), (True, dict(dk=("dq", 4 * 32)))])
def test_head_norm_refuses_shared_arrays(lib, back, change):  # noqa: F811
    a = apart(head_args(), ("q", "k", "q_out", "k_out", "dq_out", "dk_out", "dq", "dk"), [4096] * 8)
    for n, v in change.items():
        setattr(a, n, getattr(a, v) if isinstance(v, str) else getattr(a, v[0]) + v[1] if isinstance(v, tuple) else v)
    call = (lambda: lib.spz_head_norm_backward(ctypes.byref(a), PTR, 1 << 50, None)) if back else (lambda: lib.spz_head_norm_forward(ctypes.byref(a), None))
    assert call() == -1
    assert "share" in lib.spz_last_error(None).decode()
