"""A policy with a memory: a recurrent residual block trained on replayed sequences, then run step by
step for many samplers with 8-bit weights.

The task needs a history: each episode shows a cue in its first observation only, and the network's output
at every later step is to be that cue. Sequences are drawn as a learner would replay them: windows of
different lengths, with episode starts inside.

    python examples/history_policy.py [--steps 300]

The framework computes the recurrence, norms, gate, dropout and their gradients, and the products of the
samplers' steps; the projections' products in training and Adam are torch's.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2312_06126_amd import ops  # noqa: E402

OBS, CUE, WIDTH = 17, 6, 256   # observation columns (the cue in the last of them), width of the block
DROP = 0.05
SEED = 1


def rollouts(batch, steps, gen):
    """Observations [batch, steps, OBS], episode starts, lengths and the cue of every step's episode."""
    obs = torch.randn((batch, steps, OBS), generator=gen, device="cuda")
    reset = torch.rand((batch, steps), generator=gen, device="cuda") < 0.03
    reset[:, 0] = True
    cues = torch.randn((batch, steps, CUE), generator=gen, device="cuda")
    start = torch.where(reset, torch.arange(steps, device="cuda"), 0).cummax(1).values
    target = torch.gather(cues, 1, start[..., None].expand(-1, -1, CUE))
    obs[..., OBS - CUE:] = torch.where(reset[..., None], target, torch.zeros_like(target))
    lengths = torch.randint(steps // 2, steps + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
    return obs, reset, lengths, target


class Block:
    """x = drop(obs W_in); u = norm(x); f, v, z = u W + b; y = scan(f, v); x' = x + r drop(silu(z) norm(y));
    out = norm(x') W_out."""

    def __init__(self, gen):
        def weight(n_in, n_out):
            return (torch.rand((n_in, n_out), generator=gen, device="cuda") * 2 - 1) * (3.0 / n_in) ** 0.5

        ones = torch.ones(WIDTH, device="cuda")
        self.p = dict(w_in=weight(OBS, WIDTH), w=weight(WIDTH, 3 * WIDTH), b=torch.zeros(3 * WIDTH, device="cuda"),
                      w_out=weight(WIDTH, CUE), w_first=ones.clone(), w_post=ones.clone(), scale=ones.clone(), w_pre=ones.clone())
        self.p["b"][:WIDTH] = torch.linspace(0.0, 6.0, WIDTH, device="cuda")   # gates that remember for 2 to 400 steps
        self.adam = torch.optim.Adam(list(self.p.values()), lr=2e-3)

    def step(self, batch, count):
        """One update step on a batch of sequences; returns its loss."""
        p, D = self.p, WIDTH
        obs, reset, lengths, target = batch
        B, T, _ = obs.shape
        valid = (torch.arange(T, device="cuda")[None] < lengths[:, None]).reshape(-1)
        flat = obs.reshape(B * T, OBS)
        drop_in, drop_block = (DROP, SEED, count, 0), (DROP, SEED, count, 1)
        joint = dict(w_post=p["w_post"], scale=p["scale"], w_pre=p["w_pre"], gate="silu", drop=drop_block, valid=valid)

        x = ops.dropout(flat @ p["w_in"], *drop_in)
        _, u = ops.block_norm(x, w_pre=p["w_first"], valid=valid)
        proj = u @ p["w"] + p["b"]
        f, v, z = (proj[:, i * D:(i + 1) * D] for i in range(3))
        f3, v3 = (t.unflatten(0, (B, T)) for t in (f, v))
        y, _, saved = ops.scan(f3, v3, reset=reset, lengths=lengths, save=True)
        y2 = y.reshape(B * T, D)
        _, u2 = ops.block_norm(x, y2, z, **joint)
        out = u2 @ p["w_out"]
        error = torch.where(valid[:, None], out - target.reshape(B * T, CUE), 0.0)
        n = valid.sum()
        loss = (error * error).sum() / n

        dout = 2.0 * error / n
        du2 = dout @ p["w_out"].t()
        g = ops.block_norm_backward(None, du2, x, y2, z, **joint)
        dproj = torch.empty_like(proj)
        df, dv = (dproj[:, i * D:(i + 1) * D].unflatten(0, (B, T)) for i in range(2))
        ops.scan_backward(f3, v3, g["dh"].unflatten(0, (B, T)), saved, reset=reset, lengths=lengths, out=(df, dv))
        dproj[:, 2 * D:] = g["dz"]
        du = dproj @ p["w"].t()
        g1 = ops.block_norm_backward(None, du, x, w_pre=p["w_first"], valid=valid)
        dx = ops.dropout(g["dx"] + g1["dx"], *drop_in)
        grads = dict(w_in=flat.t() @ dx, w=u.t() @ dproj, b=dproj.sum(0), w_out=u2.t() @ dout, w_first=g1["dw_pre"],
                     w_post=g["dw_post"], scale=g["dscale"], w_pre=g["dw_pre"])
        for k, t in p.items():
            t.grad = grads[k]
        self.adam.step()
        return loss

    def sampler(self, n):
        """step(obs [n, OBS], reset [n]) -> out [n, CUE] of n samplers, with 8-bit weights."""
        p, D = self.p, WIDTH
        packed = {k: ops.quant_pack(*ops.quant_rows(p[k].t().contiguous())) for k in ("w_in", "w", "w_out")}
        state = torch.zeros((n, D), device="cuda")

        def step(obs, reset):
            x = ops.quant_linear(obs, packed["w_in"])
            _, u = ops.block_norm(x, w_pre=p["w_first"])
            proj = ops.quant_linear(u, packed["w"], bias=p["b"])
            f, v, z = (proj[:, i * D:(i + 1) * D] for i in range(3))
            y, _ = ops.scan(f[:, None], v[:, None], state, reset=reset[:, None], hT=state)
            _, u2 = ops.block_norm(x, y[:, 0], z, w_post=p["w_post"], scale=p["scale"], w_pre=p["w_pre"], gate="silu")
            return ops.quant_linear(u2, packed["w_out"])

        return step


def run(steps=300, batch=64, length=50, samplers=16, log=print):
    """Trains, then runs the samplers; returns (first loss, last losses' mean, samplers' mean square error)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(SEED)
    block = Block(gen)
    losses = []
    for i in range(steps):
        losses.append(block.step(rollouts(batch, length, gen), i))
        if i % 50 == 0 or i == steps - 1:
            log("step %d: loss %.4f" % (i, losses[-1].item()))
    act = block.sampler(samplers)
    obs, reset, _, target = rollouts(samplers, 200, gen)
    out = torch.stack([act(obs[:, t].contiguous(), reset[:, t].contiguous()) for t in range(obs.shape[1])], 1)
    served = ((out - target) ** 2).sum(-1).mean().item()
    log("%d samplers, %d steps, 8-bit weights: mean square error %.4f" % (samplers, obs.shape[1], served))
    return losses[0].item(), torch.stack(losses[-20:]).mean().item(), served


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=300)
    run(ap.parse_args().steps)
