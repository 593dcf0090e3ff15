"""The gate's backward where the gate is far outside the activation's curve: act' is 1 or 0
there, whatever the square of the gate overflows to. Bars as in test_ffn_gpu.py; the
evaluation's 2^-18 is of act' and its terms, which are at most 1 + 10 where the curve bends
(|G| <= 10) and nothing beyond.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import ffn as ref
from paper_2606_30634_gb300 import ffn
from test_ffn_gpu import B, DEV, U, ffn_case, np64, randn, within

pytestmark = pytest.mark.gpu

LARGE = [1e9, -1e9, 1e18, -1e18, 1e19, -1e19, 1e20, -1e20, 3e38, -3e38, 12.0, -12.0]


@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("t,d,f", [(40, 64, 72), (355, 1704, 104), (2600, 136, 264)])
def test_large_gates(kind, t, d, f):
    g, x, *w = ffn_case(t, d, f, seed=31)
    G, up = randn(g, t, f), randn(g, t, f)
    at = torch.arange(len(LARGE), device=DEV)
    G[3 * at, 5 * at] = torch.tensor(LARGE, device=DEV).bfloat16()
    dout = randn(g, t, d, scale=1e-2)
    dw = [torch.empty_like(v) for v in w]
    ffn.gated_ffn_backward(dout, ffn.Kept(G, up, kind, "bf16"), *w, *dw, x=x)
    DO, X, G, up, WG, WU, WD = (np64(v) for v in (dout, x, G, up, *w))
    with np.errstate(over="ignore"):   # exp of -G in the logistic function
        _, dwg, _, _, dg, _, _ = ref.ffn_backward(DO, X, G, up, WG, WU, WD, kind)
        slope = ref.act(G, kind)[1]
    assert np.all(np.isfinite(dg))
    da, eda = np.abs(DO @ WD), 2 * U * d * (np.abs(DO) @ np.abs(WD))
    ev = 2.0 ** -18 * (1 + np.minimum(np.abs(G), 10))
    edg = np.abs(up * slope) * eda + (da + eda) * np.abs(up) * ev + B * np.abs(dg)
    bar = edg.T @ np.abs(X) + 2 * U * t * (np.abs(dg).T @ np.abs(X))
    within(dw[0], dwg, bar + (B + 4 * U) * (np.abs(dwg) + bar) + 1e-30, "dw_gate")
    assert ffn.status() == 0
