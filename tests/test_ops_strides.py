"""Strides of the scan's outputs that no address space holds are refused before any arithmetic on them wraps (no GPU)."""
import ctypes

import pytest

from .test_ops_abi import lib, scan_args  # noqa: F401


@pytest.mark.parametrize("call,names", [("forward", ["y"]), ("backward", ["df", "dv"])])
@pytest.mark.parametrize("batch,steps,outer,inner", [(2, (1 << 22) + 1, 1 << 41, 1 << 41), (2, (1 << 30) + 1, 1 << 41, 1 << 34),
                                                     (2, (1 << 22) + 1, (1 << 42) - 1, (1 << 41) + 7)])
def test_output_strides_whose_span_wraps(lib, call, names, batch, steps, outer, inner):  # noqa: F811
    """(steps - 1) * inner passes 2^63: rows of the two sequences would overlap modulo 2^64 only."""
    from paper_2312_06126_amd import spz
    for name in names:
        for a, b in (("_batch", "_step"), ("_step", "_batch")):
            sizes = dict(batch=batch, steps=steps) if a == "_batch" else dict(batch=steps, steps=batch)
            args = scan_args(width=1, **sizes, **{k + s: 0 for k in ("f", "v") for s in ("_batch", "_step")})
            for other in ("y", "df", "dv"):   # the ones not under test: rows side by side
                setattr(args, other + "_batch", sizes["steps"])
                setattr(args, other + "_step", 1)
            setattr(args, name + a, outer)
            setattr(args, name + b, inner)
            assert getattr(lib, "spz_scan_" + call)(ctypes.byref(args), (1 << 20), 1 << 60, None) == spz.SPZ_EINVAL
            assert "overlap" in lib.spz_last_error(None).decode()
