"""Operators of the linear-attention block on arrays in each other's place: what is taken gives the same bits, the rest is refused."""
import numpy as np
import pytest

from .helpers import log
from .test_gpu_attention import inputs, run
from .test_gpu_head_norm import inputs as head_inputs
from .test_gpu_ops import PRECS, torch_

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("shape", [(3, 1, 2, 40, 64), (2, 4, 2, 24, 130), (3, 50, 2, 64, 200), (2, 150, 2, 33, 5), (2, 400, 1, 24, 130)], ids=str)
def test_attention_writes_y_in_the_place_of_v(shape, prec):
    from paper_2312_06126_amd import ops
    torch = torch_()
    log("y in the place of v %s %s" % (shape, prec))
    t, reset, lengths = inputs(np.random.default_rng(sum(shape)), *shape, prec)
    a = dict(rate=t["rate"], state=t["state"], reset=torch.from_numpy(reset).cuda(), lengths=torch.from_numpy(lengths).cuda())
    y, last = ops.linear_attention(t["q"], t["k"], t["v"], **a)
    v = t["v"].clone()
    got, end = ops.linear_attention(t["q"], t["k"], v, out=v, **a)
    assert got is v and torch.equal(v, y) and torch.equal(end, last)


@pytest.mark.parametrize("prec", PRECS)
def test_attention_gradients_into_parts_of_a_head(prec):
    """dq, dk and dv that follow each other within each head of one array, as do q, k and v."""
    torch = torch_()
    B, T, H, K, V = 2, 70, 3, 24, 40
    t, reset, lengths = inputs(np.random.default_rng(1), B, T, H, K, V, prec)
    want = run(t, reset, lengths)
    at, parts = 0, {}
    both = torch.full((2, B, T, H, 2 * K + 2 * V), 7.0, dtype=t["q"].dtype, device="cuda")
    for n, w in (("q", K), ("k", K), ("v", V), ("dy", V)):
        parts[n] = both[0, ..., at:at + w].copy_(t[n])
        parts["d" + n] = both[1, ..., at:at + w]
        at += w
    got = run(dict(t, **{n: parts[n] for n in ("q", "k", "v", "dy")}), reset, lengths, outs=(parts["ddy"], parts["dq"], parts["dk"], parts["dv"]))
    assert all(torch.equal(got[n], want[n]) for n in want)
    assert got["dk"] is parts["dk"] and torch.equal(parts["dv"], want["dv"])


def test_attention_refuses_outputs_that_share_elements():
    from paper_2312_06126_amd import ops
    from paper_2312_06126_amd.spz import SPZ_EINVAL, SpzError
    torch = torch_()
    t, _, _ = inputs(np.random.default_rng(2), 2, 9, 3, 16, 16, "fp32", False, False)
    q, k, v, dy, state = (t[n] for n in ("q", "k", "v", "dy", "state"))
    x, y, z = (torch.empty_like(q) for _ in range(3))
    wide = torch.empty((2, 10, 3, 16), device="cuda")
    states = torch.zeros(2 * 3 * 16 * 16 + 4, device="cuda")

    def back(*out):
        return lambda: ops.linear_attention_backward(q, k, v, dy, out=out)

    for call in (back(x, x, y), back(x, y, x), back(y, x, x), back(wide[:, 1:], wide[:, :-1], x), back(q, x, y), back(x, y, dy), back(x, v, y),
                 lambda: ops.linear_attention(q, k, v, out=q), lambda: ops.linear_attention(q, k, v, out=k),
                 lambda: ops.linear_attention(q, k, wide[:, 1:], out=wide[:, :-1]),
                 lambda: ops.linear_attention(q, k, v, state=states[4:].view(2, 3, 16, 16), last=states[:-4].view(2, 3, 16, 16))):
        with pytest.raises(SpzError) as e:
            call()
        assert e.value.code == SPZ_EINVAL and "share" in str(e.value)
    back(x, y, z)()


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("dim", [64, 39, 200])
def test_head_norm_gradients_in_the_place_of_operands(dim, prec):
    from paper_2312_06126_amd import ops
    from paper_2312_06126_amd.spz import SPZ_EINVAL, SpzError
    torch = torch_()
    t = head_inputs(np.random.default_rng(dim), 50, 3, 3, dim, prec)
    a = dict(w_q=t["w_q"], w_k=t["w_k"], norm="layer", positions=torch.arange(50, dtype=torch.int32, device="cuda"), freqs=ops.rotation_freqs(dim // 2 * 2))
    want = ops.head_norm_backward(t["dq"], t["dk"], t["q"], t["k"], **a)
    q, k = t["q"].clone(), t["k"].clone()
    got = ops.head_norm_backward(t["dq"], t["dk"], q, k, out=(q, k), **a)
    assert all(got[n] is None or torch.equal(got[n], want[n]) for n in want)
    # Heads of queries and of keys in one array: the parts of a row.
    one = torch.empty((50, 6, dim), dtype=q.dtype, device="cuda")
    yq, yk = ops.head_norm(t["q"], t["k"], out=(one[:, :3], one[:, 3:]), **a)
    want = ops.head_norm(t["q"], t["k"], **a)
    assert torch.equal(yq, want[0]) and torch.equal(yk, want[1])
    x, q, k = torch.empty_like(q), t["q"], t["k"]
    for call in (lambda: ops.head_norm(q, k, out=(x, x), **a), lambda: ops.head_norm(q, k, out=(k, q), **a), lambda: ops.head_norm(q, k, out=(x, q), **a),
                 lambda: ops.head_norm(q, k, out=(one[:, :3], one[:, 2:5]), **a), lambda: ops.head_norm_backward(t["dq"], t["dk"], q, k, out=(x, x), **a),
                 lambda: ops.head_norm_backward(t["dq"], t["dk"], q, k, out=(t["dk"], x), **a)):
        with pytest.raises(SpzError) as e:
            call()
        assert e.value.code == SPZ_EINVAL and "share" in str(e.value)
