"""Calls of the recurrent block's operators with more work than one dispatch takes (2^32 work-items): the
results are those of calls on parts, or of the one row that every row repeats."""
import numpy as np
import pytest

from .helpers import log
from .test_gpu_ops import gpu, torch_

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    """Up to some hundred gigabytes a test: given back before the next one."""
    yield
    torch_().cuda.empty_cache()


def all_equal(rows, row, step=1 << 24):
    """Every row of `rows` is `row`, a part at a time."""
    return all(bool((rows[i:i + step] == row).all()) for i in range(0, len(rows), step))


def test_scan_of_many_states():
    """2^32 channels of odd width, one thread each, forward and backward."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(51)
    B, D = (1 << 22) + 1, 1025
    one = {k: gpu(rng.standard_normal((1, 1, D)), "bf16") for k in ("f", "v", "dy")}
    t = {k: x.expand(B, 1, D) for k, x in one.items()}
    log("scan %d x 1 x %d" % (B, D))
    y, hT, saved = ops.scan(t["f"], t["v"], save=True)
    y1, hT1, saved1 = ops.scan(one["f"], one["v"], save=True)
    assert all_equal(y[:, 0], y1[0, 0], 1 << 20) and all_equal(hT, hT1[0], 1 << 20)
    del y, hT
    got, want = ops.scan_backward(t["f"], t["v"], t["dy"], saved), ops.scan_backward(one["f"], one["v"], one["dy"], saved1)
    for g, w in zip(got, want):
        assert all_equal(g.reshape(B, D), w.reshape(D), 1 << 20)
