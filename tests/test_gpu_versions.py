"""Tensors that a call writes are marked as written: what autograd saved of them before is not used with the new values."""
import pytest

from .test_gpu_ops import torch_

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_between_a_product_with_a_copy_and_its_gradient(bits):
    """A step raises the versions of the parameters and copies that it writes, and of no others."""
    from paper_2312_06126_amd import ops
    torch = torch_()
    params = [torch.ones((16, 16), device="cuda") for _ in range(3)]
    copies = [torch.ones((16, 16), device="cuda", dtype=torch.bfloat16), None, torch.ones((16, 16), device="cuda", dtype=torch.bfloat16)]
    opt = ops.AdamW(params, bits=bits, copies=copies)
    grads = [torch.ones((16, 16), device="cuda") for _ in range(3)]
    x = torch.ones((4, 16), device="cuda", dtype=torch.bfloat16, requires_grad=True)
    for given, written in ((grads, (True, True)), ([grads[0], grads[1], None], (True, False)), ([None, grads[1], None], (False, False)),
                           ([grads[0], grads[1].bfloat16(), grads[2]], (True, True))):
        before = [t._version for t in (*params, copies[0], copies[2])]
        outs = [(x @ c).sum() for c in (copies[0], copies[2])]
        opt.step(given, step=1, lr=1e-2)
        after = [t._version for t in (*params, copies[0], copies[2])]
        assert [b > a for a, b in zip(before, after)] == [g is not None for g in given] + [given[0] is not None, given[2] is not None]
        for out, changed in zip(outs, written):
            if changed:
                with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                    out.backward()
            else:
                out.backward()
