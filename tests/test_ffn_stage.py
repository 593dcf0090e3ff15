"""examples/ffn_stage.py: the feed-forward operators with the delayed optimizers."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location(
        "ffn_stage", os.path.join(ROOT, "examples", "ffn_stage.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_the_stage_learns_from_8_bit_activations(cuda_device):
    losses, kept, plain = example().train(dim=264, hidden=712, tokens=300, steps=40, log=None)
    assert all(l == l and l < 1e3 for l in losses)
    means = [sum(losses[i:i + 5]) for i in range(0, 40, 5)]   # it falls all the way
    assert all(b < a for a, b in zip(means, means[1:])), means
    assert kept < 0.53 * plain


def test_stage_gradients_against_autograd(cuda_device):
    """Two blocks' gradients from 8-bit activations against torch's in fp32: the 8-bit
    forms are a few per cent off an element, independently, which sums over the tokens
    and columns average; a wrong term would be of the gradient's own size."""
    mod = example()
    stage = mod.Stage(256, 640, 2, tokens=500)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(500, 256, generator=g, device="cuda").bfloat16()
    up = (torch.randn(500, 256, generator=g, device="cuda") * 1e-2).bfloat16()
    out, saved = stage.forward(x)
    dx = stage.backward(up, saved, accumulate=False)
    ws = [stage.muon.stale(i).float().requires_grad_() for i in range(6)]
    ns = [stage.adamw.stale(i).float().requires_grad_() for i in range(2)]
    xin = x.float().requires_grad_()
    s = xin
    for b in range(2):
        n = s * torch.rsqrt(s.square().mean(1, keepdim=True) + 1e-5) * ns[b]
        s = s + (torch.nn.functional.silu(n @ ws[3 * b].t()) * (n @ ws[3 * b + 1].t())) @ ws[3 * b + 2].t()
    s.backward(up.float())
    rel = lambda a, b: ((a.float() - b).norm() / b.norm()).item()
    assert rel(out, s.detach()) < 1e-2
    assert rel(dx, xin.grad) < 5e-2
    for i in range(6):
        assert rel(stage.muon.grads(i), ws[i].grad) < 5e-2, i
    for i in range(2):
        assert rel(stage.adamw.grads(i), ns[i].grad) < 5e-2, i
    stage.close()
