"""The block's products with K split over clusters, in every epilogue: the gate with its
8-bit scales over the lanes of a row, the gate's backward, and several tiles to a cluster.
Bars as in test_ffn_gpu.py; the sizes are in ffn_forms.py.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from ffn_forms import DOWN, DX, GATE, ROUNDS, SPLIT, WHOLE, forms, rounds
from paper_2606_30634_gb300 import dpo, ffn
from test_ffn_gpu import check_backward, check_forward, ffn_case, np64, randn

pytestmark = pytest.mark.gpu


def takes(size, keep, products, several=False):
    """The products are split on this device, whatever its number of clusters."""
    got = forms(size, keep, None)
    for p in products:
        if p == DX or (keep == "bf16" and size[0] <= 8 and p in (GATE, DOWN)):
            continue
        assert got[p].kind == dpo.DPO_FFN_SPLIT, (size, p)
        assert not several or rounds(got[p]) > 1


def step(x, w, dout, kind, keep, dtype=torch.bfloat16):
    out, kept = ffn.gated_ffn(x, *w, activation=kind, keep=keep)
    dw = [torch.empty(v.shape, dtype=dtype, device=v.device) for v in w]
    return out, kept, [ffn.gated_ffn_backward(dout, kept, *w, *dw, x=x), *dw]


def flat(kept):
    return [t for p in kept[:2] for t in (p if isinstance(p, tuple) else [p])]


@pytest.mark.parametrize("size", SPLIT)
@pytest.mark.parametrize("kind,keep", [("silu", "8bit"), ("gelu", "8bit"), ("gelu", "bf16"),
                                       ("silu", "bf16")])
def test_split(size, kind, keep):
    takes(size, keep, SPLIT[size])
    t, d, f = size
    g, x, *w = ffn_case(t, d, f, seed=41, pitch=8)
    dout = randn(g, t, d, scale=1e-2)
    out, kept, grads = step(x, w, dout, kind, keep)
    check_forward(x, w, kind, out, kept)
    check_backward(dout, np64(x), kept, w, grads)
    again = step(x, w, dout, kind, keep)
    for a, b in zip([out, *flat(kept), *grads], [again[0], *flat(again[1]), *again[2]]):
        assert torch.equal(a, b)
    assert ffn.status() == 0


@pytest.mark.parametrize("size", ROUNDS)
def test_several_tiles_to_a_cluster(size):
    takes(size, "8bit", ROUNDS[size], several=True)
    t, d, f = size
    g, x, *w = ffn_case(t, d, f, seed=42)
    dout = randn(g, t, d, scale=1e-2)
    out, kept, grads = step(x, w, dout, "silu", "8bit")
    check_forward(x, w, "silu", out, kept)
    check_backward(dout, np64(x), kept, w, grads)
    again = step(x, w, dout, "silu", "8bit")
    for a, b in zip([out, *flat(kept), *grads], [again[0], *flat(again[1]), *again[2]]):
        assert torch.equal(a, b)
    assert ffn.status() == 0


@pytest.mark.parametrize("size", WHOLE)
@pytest.mark.parametrize("keep", ["8bit", "bf16"])
def test_one_share_of_k(size, keep):
    takes(size, keep, WHOLE[size])
    _, x, *w = ffn_case(*size, seed=43)
    out, kept = ffn.gated_ffn(x, *w, keep=keep)
    check_forward(x, w, "silu", out, kept)
    assert ffn.status() == 0


@pytest.mark.parametrize("size", [(39, 2560, 528), (261, 1448, 392), (69, 1416, 8), (19, 1808, 976)])
@pytest.mark.parametrize("keep", ["8bit", "bf16"])
def test_non_finite_tokens_stay_in_their_rows(size, keep):
    takes(size, keep, SPLIT[size])
    t, d, f = size
    g, x, *w = ffn_case(t, d, f, seed=44)
    dout = randn(g, t, d, scale=1e-2)
    bad = x.clone()
    bad[3, 5], bad[t - 1, d - 1] = float("nan"), float("inf")
    rows = torch.ones(t, dtype=torch.bool, device=x.device)
    rows[3] = rows[t - 1] = False
    (out, kept, grads), (bout, bkept, bgrads) = (step(v, w, dout, "silu", keep) for v in (x, bad))
    for a, b in zip([out, grads[0], *flat(kept)], [bout, bgrads[0], *flat(bkept)]):
        assert torch.equal(a[rows], b[rows])
    assert not torch.isfinite(bout[~rows]).any() and not torch.isfinite(bgrads[0][~rows]).all(1).any()
    if keep == "8bit":
        for p in bkept[:2]:
            assert torch.isnan(ffn.unpack8(p)[3]).all()
            assert not torch.isfinite(ffn.unpack8(p)[t - 1]).any()
    assert ffn.status() == 0


@pytest.mark.parametrize("size", [(39, 2560, 528), (572, 2056, 456), (135, 1408, 256)])
def test_a_group_with_an_infinity_keeps_its_finite_scale(size):
    """One gate column overflows to infinity: its code is NaN, and its group's scale is that
    of the other 31 columns. The 8-bit values of the other columns are those without it."""
    takes(size, "8bit", SPLIT[size])
    t, d, f = size
    g, x, wg, wu, wd = ffn_case(t, d, f, seed=45)
    x[:, 0] = 1.0                     # a column of x that no weight reads but one
    wg[:, 0] = wu[:, 0] = 0
    _, clean = ffn.gated_ffn(x, wg, wu, wd)
    big = wg.clone()
    col = f - 5
    big[col] = 0
    big[col, 0] = float("inf")        # inf for every token, with no NaN beside it
    _, kept = ffn.gated_ffn(x, big, wu, wd)
    zero = wg.clone()
    zero[col] = 0
    _, want = ffn.gated_ffn(x, zero, wu, wd)
    others = torch.arange(f, device=x.device) != col
    assert torch.equal(kept.gate.scales, want.gate.scales)
    assert torch.equal(kept.gate.codes[:, others], want.gate.codes[:, others])
    assert torch.isnan(ffn.unpack8(kept.gate)[:, col]).all()
    assert torch.equal(kept.up.codes, clean.up.codes)
