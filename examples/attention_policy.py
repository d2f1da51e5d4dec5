"""A policy that looks things up in its history: a linear-attention block trained on replayed sequences with an 8-bit
AdamW, then run step by step for many samplers.

The task needs a history: each episode shows a cue in its first observation only, and the network's output at every later
step is to be that cue. Sequences are drawn as a learner would replay them: windows of different lengths, with episode
starts inside.

    python examples/attention_policy.py [--steps 300]

The framework computes the norms, the rotation, the attention, their gradients and the optimizer's step; the products with
the weights are torch's.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.history_policy import CUE, OBS, rollouts  # noqa: E402
from paper_2312_06126_amd import ops  # noqa: E402

HEADS, WIDE = 4, 32            # heads and their width
WIDTH = HEADS * WIDE
SEED = 2


class Block:
    """x = obs W_in; u = norm(x); q, k, v, z = u W + b; q, k = turned norms of their heads; y = attention(q, k, v);
    x' = x + r silu(z) heads' norm(y); out = norm(x') W_out."""

    def __init__(self, gen, bits=8):
        def weight(n_in, n_out):
            return (torch.rand((n_in, n_out), generator=gen, device="cuda") * 2 - 1) * (3.0 / n_in) ** 0.5

        ones = torch.ones(WIDTH, device="cuda")
        head = torch.ones(WIDE, device="cuda")
        self.p = dict(w_in=weight(OBS, WIDTH), w=weight(WIDTH, 4 * WIDTH), b=torch.zeros(4 * WIDTH, device="cuda"), w_out=weight(WIDTH, CUE), w_first=ones.clone(),
                      scale=ones.clone(), w_pre=ones.clone(), w_q=head.clone(), w_k=head.clone(), w_y=head.clone())
        self.p["b"][:2 * WIDTH] = 1.0            # queries and keys that meet whatever the observation
        # Heads that remember for 4 to 500 steps, and angles for positions within an episode.
        self.rate = 1.0 / torch.tensor([4.0 * 5.0 ** i for i in range(HEADS)], device="cuda")
        self.freqs = ops.rotation_freqs(WIDE)
        self.adam = ops.AdamW(list(self.p.values()), bits=bits, weight_decay=[0.01 if t.dim() == 2 else 0.0 for t in self.p.values()])

    def parts(self, proj):
        """q, k, v [rows, heads, width] and z [rows, width] of a projection."""
        q, k, v = (proj[:, i * WIDTH:(i + 1) * WIDTH].unflatten(1, (HEADS, WIDE)) for i in range(3))
        return q, k, v, proj[:, 3 * WIDTH:]

    def gradients(self, batch):
        """Loss and gradients of a batch of sequences."""
        p = self.p
        obs, reset, lengths, target = batch
        B, T, _ = obs.shape
        step = torch.arange(T, device="cuda")
        valid = (step[None] < lengths[:, None]).reshape(-1)
        start = torch.where(reset, step, 0).cummax(1).values
        turn = dict(w_q=p["w_q"], w_k=p["w_k"], positions=(step - start).reshape(-1).to(torch.int32), freqs=self.freqs, valid=valid)
        masks = dict(reset=reset, lengths=lengths)
        joint = dict(scale=p["scale"], w_pre=p["w_pre"], post="none", gate="silu", valid=valid)
        flat = obs.reshape(B * T, OBS)

        x = flat @ p["w_in"]
        _, u = ops.block_norm(x, w_pre=p["w_first"], valid=valid)
        proj = u @ p["w"] + p["b"]
        q, k, v, z = self.parts(proj)
        tq, tk = (t.unflatten(0, (B, T)) for t in ops.head_norm(q, k, **turn))
        y, _ = ops.linear_attention(tq, tk, v.unflatten(0, (B, T)), self.rate, **masks)
        y = y.flatten(0, 1)
        h, _ = ops.head_norm(y, w_q=p["w_y"], valid=valid)
        _, u2 = ops.block_norm(x, h.flatten(1), z, **joint)
        out = u2 @ p["w_out"]
        error = torch.where(valid[:, None], out - target.reshape(B * T, CUE), 0.0)
        n = valid.sum()
        loss = (error * error).sum() / n

        dout = 2.0 * error / n
        g = ops.block_norm_backward(None, dout @ p["w_out"].t(), x, h.flatten(1), z, **joint)
        gy = ops.head_norm_backward(g["dh"].unflatten(1, (HEADS, WIDE)), None, y, w_q=p["w_y"], valid=valid)
        dproj = torch.empty_like(proj)
        dq, dk, dv, dz = self.parts(dproj)
        dtq, dtk, _, _ = ops.linear_attention_backward(tq, tk, v.unflatten(0, (B, T)), gy["dq"].unflatten(0, (B, T)), self.rate,
                                                       out=(torch.empty_like(tq), torch.empty_like(tk), dv.unflatten(0, (B, T))), **masks)
        gt = ops.head_norm_backward(dtq.flatten(0, 1), dtk.flatten(0, 1), q, k, out=(dq, dk), **turn)
        dz.copy_(g["dz"])
        g1 = ops.block_norm_backward(None, dproj @ p["w"].t(), x, w_pre=p["w_first"], valid=valid)
        dx = g["dx"] + g1["dx"]
        return loss, dict(w_in=flat.t() @ dx, w=u.t() @ dproj, b=dproj.sum(0), w_out=u2.t() @ dout, w_first=g1["dw_pre"], scale=g["dscale"],
                          w_pre=g["dw_pre"], w_q=gt["dw_q"], w_k=gt["dw_k"], w_y=gy["dw_q"])

    def step(self, batch, count):
        """One update step, the count-th from 1, on a batch of sequences; returns its loss."""
        loss, grads = self.gradients(batch)
        self.adam.step([grads[name] for name in self.p], step=count, lr=2e-3)
        return loss

    def sampler(self, n):
        """step(obs [n, OBS], reset [n]) -> out [n, CUE] of n samplers, whose states are kept here."""
        p = self.p
        state = torch.zeros((n, HEADS, WIDE, WIDE), device="cuda")
        position = torch.zeros(n, dtype=torch.int32, device="cuda")

        def step(obs, reset):
            position.mul_(~reset)
            x = obs @ p["w_in"]
            _, u = ops.block_norm(x, w_pre=p["w_first"])
            q, k, v, z = self.parts(u @ p["w"] + p["b"])
            q, k = ops.head_norm(q, k, w_q=p["w_q"], w_k=p["w_k"], positions=position, freqs=self.freqs)
            y, _ = ops.linear_attention(q[:, None], k[:, None], v[:, None], self.rate, state, reset=reset[:, None], last=state)
            h, _ = ops.head_norm(y[:, 0], w_q=p["w_y"])
            _, u2 = ops.block_norm(x, h.flatten(1), z, scale=p["scale"], w_pre=p["w_pre"], post="none", gate="silu")
            position.add_(1)
            return u2 @ p["w_out"]

        return step


def run(steps=300, batch=64, length=50, samplers=16, log=print):
    """Trains, then runs the samplers; returns (first loss, last losses' mean, samplers' mean square error)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(SEED)
    block = Block(gen)
    losses = []
    for i in range(steps):
        losses.append(block.step(rollouts(batch, length, gen), i + 1))
        if i % 50 == 0 or i == steps - 1:
            log("step %d: loss %.4f" % (i, losses[-1].item()))
    act = block.sampler(samplers)
    obs, reset, _, target = rollouts(samplers, 200, gen)
    out = torch.stack([act(obs[:, t].contiguous(), reset[:, t].contiguous()) for t in range(obs.shape[1])], 1)
    served = ((out - target) ** 2).sum(-1).mean().item()
    log("%d samplers, %d steps: mean square error %.4f" % (samplers, obs.shape[1], served))
    return losses[0].item(), torch.stack(losses[-20:]).mean().item(), served


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=300)
    run(ap.parse_args().steps)
