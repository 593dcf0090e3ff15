"""A pipeline stage of feed-forward blocks under one-step-delayed training.

The stage holds a few blocks, x <- x + FFN(RMSNorm(x)). Each step runs its microbatches
as an asynchronous pipeline does: a microbatch's forward, then the backward of the one
that entered ``depth`` forwards earlier, all at the stale weights; what waits for its
backward is kept in 8 bits. Gradients are added up over the microbatches in the fp32 buffers
that delayed Muon (matrices) and delayed AdamW (norm weights) read, which clip from one norm
over both. The stage learns to imitate a fixed random stage of the same shape.

    python examples/ffn_stage.py [--dim 512 --hidden 1536 --steps 60]
"""
from __future__ import annotations

import argparse
import os
import sys
from collections import deque

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_30634_gb300 import dpo, ffn, muon  # noqa: E402


class Stage:
    """``blocks`` feed-forward blocks, their delayed optimizers, and the microbatches in
    flight. Matrix i of block b is number 3 b + i in ``muon`` (gate, up, down)."""

    def __init__(self, dim, hidden, blocks, *, tokens, device="cuda", seed=0, lr=2e-3):
        gen = torch.Generator(device=device).manual_seed(seed)
        shapes = [(hidden, dim), (hidden, dim), (dim, hidden)] * blocks
        start = [torch.randn(s, generator=gen, device=device) * s[1] ** -0.5 for s in shapes]
        self.blocks, self.dim, self.hidden = blocks, dim, hidden
        self.muon = muon.DelayedMuon(shapes, ef=True, lr=lr, max_grad_norm=1.0, device=device,
                                     grad_dtype=dpo.DPO_F32, x0=start, weight_decay=0.0)
        self.adamw = dpo.DelayedAdamW([dim] * blocks, ef=True, lr=lr, max_grad_norm=1.0,
                                      stash_dtype=dpo.DPO_BF16, grad_dtype=dpo.DPO_F32,
                                      device=device, weight_decay=0.0,
                                      x0=[torch.ones(dim, device=device)] * blocks)
        self.sqnorm = torch.zeros(1, dtype=torch.float64, device=device)
        self.muon.set_clip_source(self.sqnorm)
        self.adamw.set_clip_source(self.sqnorm)

    def weights(self, b):
        return [self.muon.stale(3 * b + i) for i in range(3)]

    def forward(self, x):
        """(the stream leaving the stage, what its backward needs)."""
        saved, stream, branch = [], None, x
        for b in range(self.blocks):
            n = ffn.add_rms_norm(branch, self.adamw.stale(b), residual=stream, save8=True)
            branch, kept = ffn.gated_ffn(n.y, *self.weights(b))
            stream = n.h
            saved.append((n.x8, n.rstd, kept))
        return stream + branch, saved

    def backward(self, grad, saved, accumulate):
        """Gradients of the weights; returns the gradient of the stage's input."""
        for b in reversed(range(self.blocks)):
            x8, rstd, kept = saved[b]
            w = self.adamw.stale(b)
            dy = ffn.gated_ffn_backward(grad, kept, *self.weights(b),
                                        *(self.muon.grads(3 * b + i) for i in range(3)),
                                        x8=x8, gain=w, accumulate=accumulate)
            grad, _ = ffn.add_rms_norm_backward(dy, w, rstd, x8=x8, dh=grad,
                                                dweight=self.adamw.grads(b), accumulate=accumulate)
        return grad

    def step(self, batch, target, depth):
        """One optimizer step over the microbatches of ``batch``; the mean loss."""
        waiting, losses = deque(), []
        count = 0

        def retire():
            nonlocal count
            grad, saved = waiting.popleft()
            self.backward(grad, saved, accumulate=count > 0)
            count += 1

        for x, y in zip(batch, target):
            out, saved = self.forward(x)
            diff = out.float() - y.float()
            losses.append(diff.square().mean())
            grad = (diff * (2.0 / (diff.numel() * len(batch)))).bfloat16()
            waiting.append((grad, saved))
            if len(waiting) > depth:
                retire()
        while waiting:
            retire()
        dpo.global_sqnorm([self.adamw, self.muon], self.sqnorm)
        self.adamw.step()
        self.muon.step()
        return torch.stack(losses).mean()

    def close(self):
        self.muon.close()
        self.adamw.close()


def train(dim=512, hidden=1536, blocks=2, tokens=1024, microbatches=4, depth=2, steps=60, seed=0,
          log=print):
    """Losses of every step, and the bytes that a microbatch in flight keeps."""
    teacher = Stage(dim, hidden, blocks, tokens=tokens, seed=seed + 1)
    stage = Stage(dim, hidden, blocks, tokens=tokens, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 2)
    losses = []
    for k in range(steps):
        batch = [torch.randn(tokens, dim, generator=gen, device="cuda").bfloat16()
                 for _ in range(microbatches)]
        target = [teacher.forward(x)[0] for x in batch]
        losses.append(stage.step(batch, target, depth))
        if log and k % 10 == 0:
            log(f"step {k:4d}  loss {losses[-1].item():.5f}")
    _, saved = stage.forward(batch[0])
    kept = sum(x8.nbytes + 4 * rstd.numel() + pair.nbytes for x8, rstd, pair in saved)
    plain = blocks * tokens * (2 * (dim + 2 * hidden) + 4)
    assert ffn.status() == 0
    losses = torch.stack(losses).tolist()
    if log:
        log(f"kept per microbatch: {kept} bytes, {plain} in bf16")
    teacher.close()
    stage.close()
    return losses, kept, plain


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("dim", 512), ("hidden", 1536), ("blocks", 2), ("tokens", 1024),
                        ("microbatches", 4), ("depth", 2), ("steps", 60)):
        ap.add_argument(f"--{name}", type=int, default=value)
    train(**vars(ap.parse_args()))
