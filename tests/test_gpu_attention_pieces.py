"""Linear attention whose time is cut into pieces, with values that are not finite inside: they reach what the recurrence has them
reach, all of it, and nothing else."""
import numpy as np
import pytest

from .helpers import log
from .test_gpu_attention import inputs, ref_of, run
from .test_gpu_ops import PRECS, check, torch_

pytestmark = pytest.mark.gpu

SHAPES = [(2, 400, 2, 24, 40), (1, 700, 1, 96, 100), (1, 900, 2, 130, 64), (1, 640, 1, 64, 64)]


def assert_in_pieces(shape, prec):
    """Only calls in pieces need a workspace."""
    from paper_2312_06126_amd import ops
    assert min(ops._attention_sizes(*shape, {"fp32": 0, "bf16": 1}[prec])) > 0


def spoiled(x):
    """Rows [steps] of the first sequence and head of which some element is not finite."""
    return ~torch_().isfinite(x[0, :, 0].float()).all(-1)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_values_that_are_not_finite_inside_a_piece(shape, prec):
    """In the middle of a piece, on its first step and on its last one; the next episode starts in the same piece, on the first step of
    a later one, inside one; the one that holds the value starts before it, in the same piece or in another, or on the value's step."""
    torch = torch_()
    assert_in_pieces(shape, prec)
    T = shape[1]
    t, _, _ = inputs(np.random.default_rng(sum(shape)), *shape, prec, False, False)
    for bad, before, behind in ((200, 195, 210), (200, 70, 320), (192, 128, 256), (192, 192, 350), (191, 3, 192), (255, 250, 256), (200, 100, 201), (130, 65, T - 1)):
        reset = np.zeros((shape[0], T), np.uint8)
        reset[:, [before, behind]] = 1
        want = ref_of(t, reset, None, prec)
        rest = np.ones(T, bool)
        rest[before:behind] = False
        for name, value in (("k", float("inf")), ("v", float("nan")), ("dy", float("-inf")), ("q", float("nan"))):
            log("not finite in pieces %s %s %s at %d, starts %d and %d" % (shape, prec, name, bad, before, behind))
            u = dict(t, **{name: t[name].clone()})
            u[name][0, bad, 0, 1] = value
            got = run(u, reset)
            check("last", got["last"], want["last"], "fp32")
            check("dstate", got["dstate"], want["dstate"], "fp32")
            fore, aft = rest.copy(), rest.copy()
            if name in "kv":                       # the state from the value on
                fore[before:bad] = True
                aft[:] = True
                aft[bad] = False
            else:                                  # the gradient to it up to the value, and its own step
                aft[bad + 1:behind] = True
                fore[:] = True
                fore[bad] = False
            for part, rows in (("y", fore), ("dq", fore), ("dk", aft), ("dv", aft)):
                check(part, got[part][:, rows], tuple(x[:, rows] for x in want[part]), prec)
            hit = np.zeros(T, bool)
            hit[bad:behind] = name in "kv"
            hit[before:bad + 1] |= name not in "kv"
            hit = torch.from_numpy(hit).cuda()
            if name in "kv":
                assert torch.equal(spoiled(got["y"]), hit) and torch.equal(spoiled(got["dq"]), hit)
            else:
                assert torch.equal(spoiled(got["dk"]), hit) and torch.equal(spoiled(got["dv"]), hit)


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_states_that_are_not_finite_stay(shape, value, prec):
    """However far the state has decayed: no factor makes a number of them (the first head's factor over a chunk is below float32's numbers)."""
    torch = torch_()
    assert_in_pieces(shape, prec)
    t, _, _ = inputs(np.random.default_rng(1), *shape, prec, False, False)
    t["rate"][0] = 3.0
    u = dict(t, state=t["state"].clone(), dlast=t["dlast"].clone())
    u["state"][0, 0], u["dlast"][0, 0] = value, value
    got = run(u)
    for part in ("y", "dq", "dk", "dv"):
        assert spoiled(got[part]).all(), part
    for part in ("last", "dstate"):
        assert not torch.isfinite(got[part][0, 0]).any(), part
    x = ref_of(t, None, None, prec)
    for part in ("y", "dq", "dk", "dv"):
        check(part, got[part][1:], tuple(z[1:] for z in x[part]), prec)
        check(part, got[part][:, :, 1:], tuple(z[:, :, 1:] for z in x[part]), prec)
