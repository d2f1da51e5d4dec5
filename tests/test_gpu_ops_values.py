"""Values of the recurrent block's operators where float32 has to be used with care: sigmoids far from
zero, and the state behind sequences that end before the last step."""
import numpy as np
import pytest

from . import ops_reference as ref
from .helpers import log
from .test_gpu_ops import gpu, host, torch_

pytestmark = pytest.mark.gpu


def sigmoid_arguments():
    rng = np.random.default_rng(41)
    x = np.concatenate([np.linspace(-80, 80, 4001), rng.uniform(-80, 80, 4000), rng.standard_normal(186), [0.0, -0.0, 1e-30, -1e-30, 0.5]])
    return x.astype(np.float32)   # 8192 of them


def relative(name, got, want, units):
    off = np.abs(got - want) / np.abs(want)
    log("%s: at most %.2f of %g units" % (name, off.max() / ref.U, units))
    assert (off <= units * ref.U).all(), (name, off.max() / ref.U, units)


# In units of 2^-24. e = exp(-|x|): the hardware's 2^t (1 ulp: 2) and a product by fma (1): 3. The larger of a = sigmoid(x) and 1 - a
# is 1 / (1 + e): at most half of e's 3, 1 of the sum, 2 of the reciprocal (1 ulp). The other one is e / (1 + e): 3 / (1 + e) of
# e, 1 + 2 of the quotient, 1 of the product: less than 7. 1 - a may be 2 more, for ways whose e and 1 + e are off
# on the same side; a product of both is 7 + 9 + 1.
A, B, AB = 7, 9, 17


def test_sigmoids_of_the_scan():
    """a, 1 - a and both gradients of single steps, each to a few units of its own size over |f| <= 80."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    f = sigmoid_arguments().reshape(8, 1, -1)
    a, b = ref.sigmoid(f.astype(np.float64))
    one, zero = torch.ones(f.shape, device="cuda"), torch.zeros(f.shape, device="cuda")
    keep, hT, saved = ops.scan(gpu(f), zero, one[:, 0].contiguous(), save=True)
    relative("a", host(keep), a, A)
    relative("1 - a", host(ops.scan(gpu(f), one)[0]), b, B)
    df, dv, dh0 = ops.scan_backward(gpu(f), zero, one, saved)
    relative("df", host(df), a * b, AB)
    relative("dv", host(dv), b, B)
    relative("dh0", host(dh0), a[:, 0], A)


@pytest.mark.parametrize("width", [64, 16392])
def test_sigmoids_of_the_gates(width):
    """Gates and their slopes the same, in rows that stay in registers and in rows read again."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rows = 2 * 8192 // width if width < 8192 else 1
    z = np.resize(sigmoid_arguments(), (rows, width))
    s, t = ref.sigmoid(z.astype(np.float64))
    one, zero = torch.ones(z.shape, device="cuda"), torch.zeros(z.shape, device="cuda")
    for gate in ("sigmoid", "silu"):
        x_out, _ = ops.block_norm(zero, one, gpu(z), post="none", pre="none", gate=gate)
        dz = ops.block_norm_backward(one, None, zero, one, gpu(z), post="none", pre="none", gate=gate)["dz"]
        if gate == "sigmoid":
            relative("gate", host(x_out), s, A)
            relative("slope", host(dz), s * t, AB)
        else:
            # z s is one rounding more; the slope s (1 + z t) is a sum of s and z s t, which may cancel.
            some = z != 0
            relative("silu", host(x_out)[some], (z * s)[some], A + 1)
            off = np.abs(host(dz) - s * (1.0 + z * t))
            assert (off <= ((A + 1) * s + (A + B + 2) * s * t * np.abs(z)) * ref.U * 1.01).all()


@pytest.mark.parametrize("B,T,D", [(2, 6000, 40), (1, 3001, 7), (3, 300, 24), (200, 40, 513)])
def test_last_state_is_that_of_the_last_step(B, T, D):
    """hT and y's last row are one number, whichever way the sequence is walked and wherever it ends."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    rng = np.random.default_rng(42)
    f, v, h0 = gpu(rng.standard_normal((B, T, D)) * 2 + 1), gpu(rng.standard_normal((B, T, D))), gpu(rng.standard_normal((B, D)))
    for n in (0, 1, T // 3, T - 1, T):
        y, hT = ops.scan(f, v, h0, lengths=torch.full((B,), n, dtype=torch.int32, device="cuda"))
        assert torch.equal(hT, y[:, n - 1] if n else h0), n


@pytest.mark.parametrize("kind", ["normal", "relu"])
def test_quant_of_bfloat16_like_torch(kind):
    """bfloat16 rows, where ties are common: scales, integers and products are those of the same formula in torch."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(43)
    x = torch.randn((100000, 200), generator=gen, device="cuda").bfloat16()
    if kind == "relu":
        x = torch.relu(x)
    q, s = ops.quant_rows(x)
    scale = x.float().abs().amax(1) / 127.0
    want = torch.round(x.float() / scale[:, None])
    assert torch.equal(s, scale) and torch.equal(q.float(), want)
    w = ops.quant_pack(torch.eye(200, dtype=torch.int8, device="cuda"), torch.ones(200, device="cuda"))
    assert torch.equal(ops.quant_linear(x, w), (want * scale[:, None]).bfloat16())


@pytest.mark.parametrize("B,T,D", [(2, 0, 4), (0, 3, 4), (2, 3, 0), (0, 0, 0)])
def test_scan_without_elements(B, T, D):
    """No steps leave the state and its gradient as they are; no sequences or channels leave nothing."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    f, state = torch.ones((B, T, D), device="cuda"), torch.randn((B, D), device="cuda")
    y, hT, saved = ops.scan(f, f, state, save=True)
    df, dv, dh0 = ops.scan_backward(f, f, y, saved, dhT=state)
    assert y.shape == df.shape == dv.shape == (B, T, D)
    assert hT.shape == dh0.shape == (B, D)
    if T == 0:
        assert torch.equal(hT, state) and torch.equal(dh0, state)
    x = torch.ones((B * T, D), device="cuda")
    x_out, u = ops.block_norm(x, x)
    assert x_out.shape == u.shape == ops.dropout(x, 0.5, 1, 2).shape == x.shape
    g = ops.block_norm_backward(x_out, u, x, x, w_post=torch.ones(D, device="cuda"))
    assert g["dh"].shape == x.shape and g["dw_post"].shape == (D,) and not g["dw_post"].any()
    q, s = ops.quant_rows(x)
    assert q.shape == x.shape and not s.any()
    w = ops.quant_pack(torch.ones((3, D), dtype=torch.int8, device="cuda"), torch.ones(3, device="cuda"))
    assert ops.quant_linear(x, w).shape == (B * T, 3) and not ops.quant_linear(x, w).any() or D
