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


def test_outputs_that_a_caller_gives():
    """Each tensor that a caller gives to be written has its version raised, its operands have not; what is saved of it is refused."""
    from paper_2312_06126_amd import ops
    torch = torch_()

    def ones(*shape, dtype=torch.float32):
        return torch.ones(shape, device="cuda", dtype=dtype)

    f, v, h = ones(2, 5, 16), ones(2, 5, 16), ones(2, 16)
    q, k, w, s = ones(2, 5, 3, 16), ones(2, 5, 3, 16), ones(2, 5, 3, 8), ones(2, 3, 16, 8)
    a, b, x = ones(6, 4, 16), ones(6, 2, 16), ones(6, 16)
    weights = ops.quant_pack(*ops.quant_rows(ones(8, 16)))
    saved = ops.scan(f, v, h, save=True)[2]
    calls = [lambda o: ops.scan(f, v, h, out=o[0], hT=o[1]), lambda o: ops.scan(f, v, o[0], hT=o[0]), lambda o: ops.scan_backward(f, v, f, saved, out=o),
             lambda o: ops.dropout(x, 0.5, 1, 2, out=o[0]), lambda o: ops.dropout(o[0], 0.5, 1, 2, out=o[0]), lambda o: ops.quant_linear(x, weights, out=o[0]),
             lambda o: ops.head_norm(a, b, out=o), lambda o: ops.head_norm(a, out=(o[0], None)), lambda o: ops.head_norm(*o, out=o),
             lambda o: ops.head_norm_backward(a, b, a, b, out=o), lambda o: ops.linear_attention(q, k, w, out=o[0], last=o[1]),
             lambda o: ops.linear_attention(q, k, w, state=o[0], last=o[0]), lambda o: ops.linear_attention_backward(q, k, w, w, state=s, out=o)]
    outs = [(ones(2, 5, 16), ones(2, 16)), (ones(2, 16),), (ones(2, 5, 16), ones(2, 5, 16)), (ones(6, 16),), (ones(6, 16),), (ones(6, 8),),
            (ones(6, 4, 16), ones(6, 2, 16)), (ones(6, 4, 16),), (ones(6, 4, 16), ones(6, 2, 16)), (ones(6, 4, 16), ones(6, 2, 16)),
            (ones(2, 5, 3, 8), ones(2, 3, 16, 8)), (ones(2, 3, 16, 8),), (ones(2, 5, 3, 16), ones(2, 5, 3, 16), ones(2, 5, 3, 8))]
    assert len(calls) == len(outs)
    side = torch.cuda.Stream()
    for call, given in zip(calls, outs):
        kept = (f, v, h, q, k, w, s, a, b, x, saved, weights.image, weights.scale)
        before = [t._version for t in kept]
        for stream in (None, side):
            leaf = ones(*given[0].shape).requires_grad_()
            product = (leaf * given[0]).sum()
            versions = [t._version for t in given]
            with torch.cuda.stream(stream):
                call(given)
            torch.cuda.synchronize()
            assert all(t._version > n for t, n in zip(given, versions))
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                product.backward()
        assert [t._version for t in kept] == before
