"""The feed-forward block at sizes that take its products' other forms: tiles 64 columns
wide, K split over clusters where all end inside a tile, dx apart from the weights'
gradients, lists of tiles of several rounds, and the streaming form with K split and ragged
rows. Bars as in test_ffn_gpu.py.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import ffn as ref
from paper_2606_30634_gb300 import ffn
from test_ffn_gpu import RND, check_backward, check_forward, ffn_case, np64, randn

pytestmark = pytest.mark.gpu

SIZES = [(9, 264, 4104), (20, 512, 4096), (33, 136, 2056), (64, 768, 2048), (70, 1032, 264),
         (128, 520, 1560), (200, 776, 2072), (384, 264, 1032), (500, 768, 2048), (900, 136, 4360)]


@pytest.mark.parametrize("t,d,f", SIZES)
@pytest.mark.parametrize("kind,keep,x8", [("silu", "8bit", True), ("gelu", "bf16", False)])
def test_forms(t, d, f, kind, keep, x8):
    g, x, *w = ffn_case(t, d, f, seed=21)
    out, kept = ffn.gated_ffn(x, *w, activation=kind, keep=keep)
    check_forward(x, w, kind, out, kept)
    dout = randn(g, t, d, scale=1e-2)
    X, arg = np64(x), dict(x=x)
    if x8:
        p, gain = ffn.pack8(x), 1 + randn(g, d, scale=0.2)
        X = ref.decode(p.codes.cpu().numpy(), p.scales.cpu().numpy()) * np64(gain)
        arg = dict(x8=p, gain=gain)
    runs = []
    for _ in range(2):
        dw = [torch.empty(v.shape, device=v.device) for v in w]
        runs.append([ffn.gated_ffn_backward(dout, kept, *w, *dw, **arg), *dw])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    check_backward(dout, X, kept, w, runs[0], rnd=RND["f32"])
    dw = [torch.zeros(v.shape, device=v.device) for v in w]
    assert torch.equal(ffn.gated_ffn_backward(dout, kept, *w, *dw, accumulate=True, **arg),
                       runs[0][0])
    assert all(torch.equal(a, b) for a, b in zip(dw, runs[0][1:]))
    assert ffn.status() == 0


@pytest.mark.parametrize("t", [1, 5, 8])
@pytest.mark.parametrize("d,f", [(2056, 4104), (8, 4104), (4104, 8), (1000, 16392)])
def test_few_tokens(t, d, f):
    _, x, *w = ffn_case(t, d, f, seed=22)
    out, kept = ffn.gated_ffn(x, *w, keep="bf16")
    check_forward(x, w, "silu", out, kept)
    assert torch.equal(out, ffn.gated_ffn(x, *w, keep="none")[0])


@pytest.mark.parametrize("t", [20, 130])
@pytest.mark.parametrize("keep", ["8bit", "bf16"])
def test_non_finite_tokens_stay_in_their_rows(t, keep):
    d, f = 264, 4104
    g, x, *w = ffn_case(t, d, f, seed=23)
    dout = randn(g, t, d, scale=1e-2)
    bad = x.clone()
    bad[3, 5], bad[t - 1, 7] = float("nan"), float("inf")
    rows = np.ones(t, bool)
    rows[[3, t - 1]] = False
    res = []
    for v in (x, bad):
        out, kept = ffn.gated_ffn(v, *w, keep=keep)
        dw = [torch.empty(u.shape, device=u.device) for u in w]
        res.append((out, ffn.gated_ffn_backward(dout, kept, *w, *dw, x=v)))
    keep_rows = torch.from_numpy(rows).to(x.device)
    for a, b in zip(*res):
        assert torch.equal(a[keep_rows], b[keep_rows])
        assert not torch.isfinite(b[~keep_rows]).all(dim=1).any()
    assert ffn.status() == 0
