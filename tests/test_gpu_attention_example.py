"""The example that runs head norms, linear attention, block norms and AdamW together: its gradients against torch's
differentiation of the same network in float64, and its samplers' single steps against the whole sequence."""
import math

import pytest

from .helpers import log
from .test_gpu_ops import torch_

pytestmark = pytest.mark.gpu


def network(p, rate, freqs, obs, reset, lengths, heads, wide):
    """The example's outputs [batch, steps, CUE] from its formulas, step by step, in the type of p; and the live steps."""
    torch = torch_()
    B, T, _ = obs.shape

    def norm(x):
        return x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()

    x = obs @ p["w_in"]
    q, k, v, z = (norm(x) * p["w_first"] @ p["w"] + p["b"]).chunk(4, -1)
    q, k, v = (t.unflatten(-1, (heads, wide)) for t in (q, k, v))
    q, k = norm(q) * p["w_q"], norm(k) * p["w_k"]
    state = torch.zeros((B, heads, wide, wide), dtype=x.dtype, device=x.device)
    position = torch.zeros(B, dtype=x.dtype, device=x.device)
    ys = []
    for t in range(T):
        cut = reset[:, t]
        position = torch.where(cut, 0.0, position)
        angle = position[:, None, None] * freqs
        turn = torch.polar(torch.ones_like(angle), angle)

        def turned(a):
            r = torch.complex(a[..., :wide // 2], a[..., wide // 2:]) * turn
            return torch.cat([r.real, r.imag], -1)

        state = torch.where(cut[:, None, None, None], 0.0, state * torch.exp(-rate)[:, None, None])
        state = state + turned(k[:, t])[..., None] * v[:, t][..., None, :]
        ys.append((turned(q[:, t])[..., None] * state).sum(-2) / math.sqrt(wide))
        position = position + 1
    h = (norm(torch.stack(ys, 1)) * p["w_y"]).flatten(2)
    out = norm(x + p["scale"] * (z * torch.sigmoid(z)) * h) * p["w_pre"] @ p["w_out"]
    return out, torch.arange(T, device=x.device)[None] < lengths[:, None]


def block_and_batch(steps=40, batch=6):
    from examples import attention_policy as example
    torch = torch_()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    block = example.Block(gen)
    for n in ("b", "w_first", "scale", "w_pre", "w_q", "w_k", "w_y"):      # not the ones that they start as
        block.p[n].add_(0.2 * torch.randn(block.p[n].shape, generator=gen, device="cuda"))
    return example, block, example.rollouts(batch, steps, gen)


def exact(example, block, batch):
    p = {n: t.double().requires_grad_() for n, t in block.p.items()}
    obs, reset, lengths, target = batch
    out, live = network(p, block.rate.double(), block.freqs, obs.double(), reset, lengths, example.HEADS, example.WIDE)
    return p, out, live


def test_gradients_against_differentiation_in_float64():
    """Float32 throughout: each gradient within 2^-24 times the square root of the operations behind an element (some 10^5
    to 10^6 in a chain of six products and norms), times a norm's amplification of ten: 1e-4 of the gradient's norm."""
    torch = torch_()
    example, block, batch = block_and_batch()
    loss, grads = block.gradients(batch)
    p, out, live = exact(example, block, batch)
    want = torch.where(live[..., None], out - batch[3].double(), 0.0).pow(2).sum() / live.sum()
    assert abs(loss.item() - want.item()) < 1e-4 * want.item()
    for n, g in zip(p, torch.autograd.grad(want, list(p.values()))):
        off = (grads[n].double() - g).norm() / g.norm()
        log("%s: %.2e" % (n, off.item()))
        assert off < 1e-4, (n, off.item())


def test_samplers_steps_are_the_sequence():
    torch = torch_()
    example, block, batch = block_and_batch()
    obs, reset = batch[:2]
    act = block.sampler(obs.shape[0])
    got = torch.stack([act(obs[:, t].contiguous(), reset[:, t].contiguous()) for t in range(obs.shape[1])], 1)
    with torch.no_grad():
        _, want, _ = exact(example, block, (obs, reset, torch.full_like(batch[2], obs.shape[1]), batch[3]))
    assert (got.double() - want).norm() < 1e-4 * want.norm()


def test_a_step_changes_the_weights_as_adamw_does():
    """The first step from zero moments: lr times the sign of the gradient and the decay, but for gradients near eps."""
    torch = torch_()
    _, block, batch = block_and_batch()
    before = {n: t.clone() for n, t in block.p.items()}
    _, grads = block.gradients(batch)
    block.step(batch, 1)
    for n, t in block.p.items():
        g = grads[n]
        decay = 0.01 if t.dim() == 2 else 0.0
        want = before[n] - 2e-3 * (g / (g.abs() + 1e-8) + decay * before[n])
        assert torch.allclose(t, want, rtol=1e-6, atol=1e-7), n


def test_example_runs():
    from examples import attention_policy
    first, last, served = attention_policy.run(steps=5, batch=8, length=20, samplers=3, log=log)
    assert all(math.isfinite(x) for x in (first, last, served))
