"""Calls of the recurrent block's operators with more work than one dispatch takes (2^32 work-items): the
results are those of calls on parts, or of the one row that every row repeats."""
import numpy as np
import pytest

from .helpers import log
from .test_gpu_ops import gpu, host, torch_

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


def philox_tail(first, count, step, tensor, seed):
    """Dropout's 16-bit words of elements first .. first + count - 1 (multiples of 8)."""
    from oracle import philox
    u = np.uint64
    blk = np.arange(first // 8, (first + count) // 8, dtype=np.uint64)
    w = np.stack(philox.block(blk, u(step), u(5) + ((blk >> u(32)) << u(8)), u(tensor), u(seed), u(0)), 1)
    return np.stack([w & u(0xFFFF), w >> u(16)], 2).reshape(-1)


def test_block_norm_of_many_rows():
    """2^28 rows, 16 of them a workgroup; dropout counts elements over all rows."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    R, D = (1 << 28) + 24, 2
    log("block_norm %d x %d" % (R, D))
    x = torch.empty((R, D), dtype=torch.bfloat16, device="cuda").uniform_(-1, 1)
    x_out, u = ops.block_norm(x, x, pre="layer")
    for part in (slice(0, 1 << 20), slice(R // 2, R // 2 + 4099), slice((1 << 28) - 4096, R)):
        a, b = ops.block_norm(x[part], x[part], pre="layer")
        assert torch.equal(x_out[part], a) and torch.equal(u[part], b)
    del x_out, u
    zero, one = (torch.full((1, D), c, dtype=torch.bfloat16, device="cuda").expand(R, D) for c in (0.0, 1.0))
    x_out, _ = ops.block_norm(zero, one, post="none", pre="none", drop=(0.25, 11, 12, 13))
    n = 4096
    assert np.array_equal(host(x_out[-n // D:]).reshape(-1) != 0, philox_tail(R * D - n, n, 12, 13, 11) >= 16384)


def test_block_norm_of_many_rows_of_a_wave():
    """2^26 rows of a wave each."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    R, D = (1 << 26) + 5, 264
    log("block_norm %d x %d" % (R, D))
    x = gpu(np.random.default_rng(52).standard_normal((1, D)), "bf16")
    _, u = ops.block_norm(x.expand(R, D))
    assert all_equal(u, ops.block_norm(x)[1][0], 1 << 22)


def test_block_norm_gradients_of_many_columns():
    """The vectors' gradients of more columns than one dispatch sums. Sums of small integers are exact."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    R, D = 2, (1 << 25) + 7
    log("block_norm backward %d x %d" % (R, D))
    x = torch.empty((R, D), dtype=torch.bfloat16, device="cuda").uniform_(-1, 1)
    du = torch.randint(-4, 5, (R, D), device="cuda").bfloat16()
    zero = torch.zeros(D, device="cuda")
    g = ops.block_norm_backward(None, du, x, b_pre=zero)
    assert torch.equal(g["db_pre"], du.float().sum(0))


def test_dropout_of_many_elements():
    """2^35 elements, in place: the words of the last ones are those of their 64-bit index."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    R, D, n = (1 << 15) + 1, 1 << 20, 4096
    log("dropout %d x %d" % (R, D))
    x = torch.ones((R, D), dtype=torch.bfloat16, device="cuda")
    ops.dropout(x, 0.25, 11, 12, 13, out=x)
    assert np.array_equal(host(x[-1, -n:]) != 0, philox_tail(R * D - n, n, 12, 13, 11) >= 16384)
    assert np.array_equal(host(x[0, :n]) != 0, philox_tail(0, n, 12, 13, 11) >= 16384)


def test_dropout_of_many_elements_of_rows_apart():
    from paper_2312_06126_amd import ops
    torch = torch_()
    R, D, n = (1 << 15) + 1, 1 << 20, 4096
    log("dropout %d x %d, rows apart" % (R, D))
    x = torch.ones((1, D), dtype=torch.bfloat16, device="cuda").expand(R, D)
    y = ops.dropout(x, 0.25, 11, 12, 13)
    assert np.array_equal(host(y[-1, -n:]) != 0, philox_tail(R * D - n, n, 12, 13, 11) >= 16384)


def test_quant_rows_of_many_rows():
    """2^26 rows, a wave each."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    R, D = (1 << 26) + 5, 3
    log("quant_rows %d x %d" % (R, D))
    x = torch.empty((R, D), dtype=torch.bfloat16, device="cuda").uniform_(-1, 1)
    q, s = ops.quant_rows(x)
    for part in (slice(0, R // 2), slice(R // 2, R)):
        a, b = ops.quant_rows(x[part])
        assert torch.equal(q[part], a) and torch.equal(s[part], b)


def test_quant_pack_of_a_large_image():
    """An image of more than 4 GiB: the images of parts of the channels, one after the other."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    N, K = (1 << 15) + 40, 131072
    log("quant_pack %d x %d" % (N, K))
    q = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda")
    s = torch.ones(N, device="cuda")
    image = ops.quant_pack(q, s).image
    for n0, n1 in ((0, 1 << 14), (1 << 14, N)):
        part = ops.quant_pack(q[n0:n1], s[n0:n1]).image
        assert torch.equal(image[n0 * K:n0 * K + part.numel()], part)


@pytest.mark.parametrize("R,K,N", [((1 << 30) + 70, 8, 1), ((1 << 28) + 70, 2056, 1), ((1 << 26) + 70, 0, 2)])
def test_quant_linear_of_many_rows(R, K, N):
    """64 or 32 rows a workgroup in LDS, and a wave a row where there are no inputs."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(53)
    log("quant_linear %d x %d x %d" % (R, K, N))
    x = gpu(rng.standard_normal((1, K)), "bf16")
    w = ops.quant_pack(torch.from_numpy(rng.integers(-127, 128, (N, K)).astype(np.int8)).cuda(), torch.ones(N, device="cuda"))
    bias = gpu(rng.standard_normal(N))
    y = ops.quant_linear(x.expand(R, K), w, bias=bias)
    assert all_equal(y, ops.quant_linear(x, w, bias=bias)[0])


def test_quant_linear_of_many_tiles():
    """The simple form's 32 x 32 tiles, a wave each, without inputs: 2^26 of them leave the bias everywhere."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    R, N = (1 << 21) + 33, 1 << 15
    log("quant_linear %d x 0 x %d" % (R, N))
    bias = gpu(np.random.default_rng(54).standard_normal(N))
    w = ops.quant_pack(torch.zeros((N, 0), dtype=torch.int8, device="cuda"), torch.ones(N, device="cuda"))
    y = ops.quant_linear(torch.empty((R, 0), dtype=torch.bfloat16, device="cuda"), w, bias=bias)
    assert all_equal(y, bias.bfloat16(), 1 << 16)
