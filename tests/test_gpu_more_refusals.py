"""What head_norm, linear_attention and their backward calls refuse on torch tensors."""
import pytest

from .test_gpu_ops import torch_

pytestmark = pytest.mark.gpu


def inputs():
    torch = torch_()
    q = torch.ones((6, 4, 16), device="cuda")
    w = torch.ones(16, device="cuda")
    heads = dict(q=q, k=q[:, :2].clone(), w_q=w, b_q=w.clone(), w_k=w.clone(), b_k=w.clone(), positions=torch.arange(6, dtype=torch.int32, device="cuda"),
                 freqs=torch.ones(8, dtype=torch.float64, device="cuda"), valid=torch.ones(6, dtype=torch.uint8, device="cuda"))
    x = torch.ones((2, 5, 3, 16), device="cuda")
    v = torch.ones((2, 5, 3, 8), device="cuda")
    attention = dict(q=x, k=x.clone(), v=v, rate=torch.ones(3, device="cuda"), state=torch.ones((2, 3, 16, 8), device="cuda"),
                     reset=torch.zeros((2, 5), dtype=torch.uint8, device="cuda"), lengths=torch.full((2,), 5, dtype=torch.int32, device="cuda"))
    return heads, attention


def calls(heads, attention, change):
    """Each call with one floating operand replaced by what change(operand) gives."""
    from paper_2312_06126_amd import ops
    for n in ("q", "k", "w_q", "b_q", "w_k", "b_k"):
        a = dict(heads, **{n: change(heads[n])})
        yield lambda: ops.head_norm(**a)
        yield lambda: ops.head_norm_backward(heads["q"], heads["k"], **a)
    yield lambda: ops.head_norm_backward(change(heads["q"]), heads["k"], **heads)
    yield lambda: ops.head_norm_backward(heads["q"], change(heads["k"]), **heads)
    for n in ("q", "k", "v", "rate", "state"):
        a = dict(attention, **{n: change(attention[n])})
        yield lambda: ops.linear_attention(**a)
        yield lambda: ops.linear_attention_backward(dy=attention["v"], **a)
    yield lambda: ops.linear_attention_backward(dy=change(attention["v"]), **attention)
    yield lambda: ops.linear_attention_backward(dy=attention["v"], dlast=change(attention["state"]), **attention)


def test_tensors_that_require_a_gradient():
    from paper_2312_06126_amd.spz import SPZ_EINVAL, SpzError
    torch = torch_()
    heads, attention = inputs()

    def leaf(x):
        return x.clone().requires_grad_()

    for call in calls(heads, attention, leaf):
        with pytest.raises(SpzError) as e:
            call()
        assert e.value.code == SPZ_EINVAL and "gradient" in str(e.value)
    with torch.no_grad():
        for call in calls(heads, attention, leaf):
            call()


def test_types_devices_and_shapes():
    from paper_2312_06126_amd.spz import SPZ_EINVAL, SpzError
    heads, attention = inputs()
    for change in (lambda x: x.cpu(), lambda x: x.half(), lambda x: x.double(), lambda x: x[..., :-1], lambda x: 1.0, lambda x: [1.0]):
        for call in calls(heads, attention, change):
            with pytest.raises(SpzError) as e:
                call()
            assert e.value.code == SPZ_EINVAL


def test_other_arguments():
    from paper_2312_06126_amd import ops
    from paper_2312_06126_amd.spz import SPZ_EINVAL, SpzError
    torch = torch_()
    heads, attention = inputs()
    q, x, v, state = heads["q"], attention["q"], attention["v"], attention["state"]

    def head(**kw):
        return lambda: ops.head_norm(**dict(heads, **kw))

    def attend(**kw):
        return lambda: ops.linear_attention(**dict(attention, **kw))

    def back(**kw):
        return lambda: ops.linear_attention_backward(dy=v, **dict(attention, **kw))

    wide = torch.ones((2, 5, 3, 300), device="cuda")
    for call in (head(norm="l2"), head(pairs="odd"), head(eps=0.0), head(eps="a"), head(eps=float("nan")), head(positions=None), head(freqs=None),
                 head(positions=heads["positions"].long()), head(positions=heads["positions"][:5]), head(freqs=heads["freqs"].float()),
                 head(freqs=torch.ones(9, dtype=torch.float64, device="cuda")), head(freqs=1.0), head(valid=heads["valid"].float()), head(valid=[1] * 6),
                 head(out=q), head(out=(q, None)), head(out=(q, heads["k"].bfloat16())), head(out=(q[:, :1], heads["k"])), head(q=q[0]), head(k=heads["k"][0]),
                 head(q=q.transpose(1, 2).contiguous().transpose(1, 2)), lambda: ops.head_norm_backward(q, heads["k"], q),
                 lambda: ops.head_norm(torch.ones((2, 2, 1025), device="cuda")), lambda: ops.head_norm(q, out=(torch.ones((6, 1, 16), device="cuda").expand(6, 4, 16), None)),
                 attend(k=None), attend(v=None), attend(scale="a"), attend(scale=float("nan")), attend(lengths=[5, 5]), attend(lengths=attention["lengths"].long()),
                 attend(reset=attention["reset"].float()), attend(reset=attention["reset"][:1]), attend(last=state[:1]), attend(out=x), attend(out=v.bfloat16()),
                 attend(q=wide, k=wide, state=None), attend(state=state.transpose(2, 3).contiguous().transpose(2, 3)), attend(rate=attention["rate"].double()),
                 attend(out=v[:, :1].expand(2, 5, 3, 8)), back(out=v), back(out=(x, x)), back(out=(x, x.clone(), None)), back(out=(x, x.clone(), x)),
                 back(scale=float("inf")), lambda: ops.linear_attention_backward(dy=x, **attention)):
        with pytest.raises(SpzError) as e:
            call()
        assert e.value.code == SPZ_EINVAL
