"""The feed-forward calls of include/dpo.h with outputs left out and with the pitches and
addresses that the tensor calls never give them. Expected are the full call's results, bit
for bit where the same kernel forms run, else the bars of test_ffn_gpu.py.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from ffn_forms import DOWN, DX, forms
from oracle import ffn as ref
from paper_2606_30634_gb300 import dpo, ffn
from test_ffn_gpu import (DEV, DT, RND, U, check_backward, ffn_case, gen, norm_case, np64,
                          randn, within)

pytestmark = pytest.mark.gpu

TYPE = {torch.float32: dpo.DPO_F32, torch.bfloat16: dpo.DPO_BF16}


def p(t):
    return None if t is None else t.data_ptr()


def packed(codes, scales):
    return dpo.dpo_packed8(p(codes), p(scales), codes.stride(0), scales.stride(0))


def norm(x, w, r=None, h=None, y=None, rstd=None, x8=None):
    a = dpo.dpo_rmsnorm_args(
        x=p(x), residual=p(r), weight=p(w), h=p(h), y=p(y), rstd=p(rstd), rows=x.shape[0], cols=x.shape[1],
        ld_x=x.stride(0), ld_residual=r.stride(0) if r is not None else 0, ld_h=x.shape[1],
        ld_y=x.shape[1], eps=1e-5, dtype=TYPE[x.dtype], weight_dtype=TYPE[w.dtype])
    if x8 is not None:
        a.x8 = packed(*x8)
    dpo.dpo_rmsnorm(a)


@pytest.mark.parametrize("rows,cols", [(5, 768), (700, 64), (9, 777)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_with_outputs_left_out(rows, cols, dtype):
    _, x, r, w = norm_case(rows, cols, dtype, "f32", True)
    o = ffn.add_rms_norm(x, w, r, eps=1e-5, save8=True)
    for left_out in ("h", "y", "x8", "hy"):
        h, y = torch.empty_like(x), torch.empty_like(x)
        rstd = torch.empty(rows, device=DEV)
        codes, scales = torch.empty_like(o.x8.codes), torch.empty_like(o.x8.scales)
        norm(x, w, r, None if "h" in left_out else h, None if "y" in left_out else y, rstd,
             None if left_out == "x8" else (codes, scales))
        assert torch.equal(rstd, o.rstd)
        assert "h" in left_out or torch.equal(h, o.h)
        assert "y" in left_out or torch.equal(y, o.y)
        assert left_out == "x8" or (torch.equal(codes, o.x8.codes) and torch.equal(scales, o.x8.scales))


def norm_back(dy, w, rstd, h=None, x8=None, dh=None, dx=None, dw=None):
    rows, cols = dy.shape
    ws = torch.empty(max(1, dpo.dpo_rmsnorm_workspace(rows, cols)), dtype=torch.uint8, device=DEV)
    a = dpo.dpo_rmsnorm_backward_args(
        dy=p(dy), h=p(h), rstd=p(rstd), weight=p(w), dh=p(dh), dx=p(dx), dweight=p(dw), rows=rows,
        cols=cols, ld_dy=dy.stride(0), ld_h=h.stride(0) if h is not None else 0,
        ld_dh=dh.stride(0) if dh is not None else 0, ld_dx=cols, dtype=TYPE[dy.dtype],
        weight_dtype=TYPE[w.dtype], dweight_dtype=dpo.DPO_F32, workspace=p(ws),
        workspace_bytes=ws.numel() if dw is not None else 0)
    if dw is None:
        a.workspace = None
    if x8 is not None:
        a.x8 = packed(*x8)
    dpo.dpo_rmsnorm_backward(a)


@pytest.mark.parametrize("rows,cols", [(5, 768), (700, 64), (9, 777), (3, 8200)])
@pytest.mark.parametrize("kept", ["h", "x8"])
def test_norm_backward_with_outputs_left_out(rows, cols, kept):
    g, x, _, w = norm_case(rows, cols, "bf16", "bf16", False)
    o = ffn.add_rms_norm(x, w, eps=1e-5, save8=True)
    dy, dh = randn(g, rows, cols, scale=1e-2), randn(g, rows, cols)
    arg = dict(h=o.h) if kept == "h" else dict(x8=o.x8)
    wdx, wdw = ffn.add_rms_norm_backward(dy, w, o.rstd, dh=dh, **arg)
    dx, dw = torch.empty_like(dy), torch.empty(cols, device=DEV)
    norm_back(dy, w, o.rstd, dh=dh, dx=dx, **arg)
    norm_back(dy, w, o.rstd, dh=dh, dw=dw, **arg)
    assert torch.equal(dx, wdx) and torch.equal(dw, wdw)
    norm_back(dy, w, o.rstd, dh=dh, **arg)   # nothing wanted, nothing launched


def backward(dout, kept, w, dw, x=None, x8=None, gain=None, dx=None, accumulate=False):
    (t, d), f = dout.shape, w[0].shape[0]
    ws = torch.empty(dpo.dpo_ffn_workspace(t, d, f, x is None)[1], dtype=torch.uint8, device=DEV)
    a = dpo.dpo_ffn_backward_args(
        dout=p(dout), x=p(x), gain=p(gain), w_gate=p(w[0]), w_up=p(w[1]), w_down=p(w[2]), dx=p(dx),
        dw_gate=p(dw[0]), dw_up=p(dw[1]), dw_down=p(dw[2]), tokens=t, dim=d, hidden=f,
        ld_dout=dout.stride(0), ld_x=x.stride(0) if x is not None else 0, ld_dx=d,
        act=ffn.ACTIVATIONS[kept.activation], keep=ffn.KEEP[kept.keep], grad_dtype=TYPE[dw[0].dtype],
        gain_dtype=TYPE[gain.dtype] if gain is not None else 0, accumulate=accumulate, workspace=p(ws),
        workspace_bytes=ws.numel())
    if x8 is not None:
        a.x8 = packed(*x8)
    if kept.keep == "bf16":
        a.gate, a.up = p(kept.gate), p(kept.up)
    else:
        a.gate8, a.up8 = packed(*kept.gate), packed(*kept.up)
    dpo.dpo_ffn_backward(a)


# dx in the list, and in a launch of its own
@pytest.mark.parametrize("t,d,f,alone", [(70, 1032, 264, False), (300, 200, 328, False),
                                         (20, 512, 4096, True), (2600, 136, 264, False)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_block_backward_without_dx(t, d, f, alone, dtype):
    assert (forms((t, d, f), "8bit", None)[DX].kind != dpo.DPO_FFN_NO_LAUNCH) == alone
    g, x, *w = ffn_case(t, d, f, seed=61)
    _, kept = ffn.gated_ffn(x, *w)
    dout = randn(g, t, d, scale=1e-2)
    dw = [torch.empty(v.shape, dtype=dtype, device=DEV) for v in w]
    backward(dout, kept, w, dw, x=x)
    full = [torch.empty_like(v) for v in dw]
    dx = ffn.gated_ffn_backward(dout, kept, *w, *full, x=x)
    check_backward(dout, np64(x), kept, w, [dx, *dw], rnd=RND["f32" if dtype is torch.float32 else "bf16"])
    assert ffn.status() == 0


def test_8_bit_rows_without_a_gain_at_any_address():
    """x8 from rows that begin at odd addresses, 33 codes and 3 scales further apart than
    they need to be; no gain."""
    t, d, f = 301, 200, 328
    g, x, *w = ffn_case(t, d, f, seed=62)
    _, kept = ffn.gated_ffn(x, *w)
    dout, q = randn(g, t, d, scale=1e-2), ffn.pack8(x)
    codes = torch.zeros(t, d + 33, dtype=torch.uint8, device=DEV)[:, 5:5 + d]
    scales = torch.zeros(t, q.scales.shape[1] + 3, dtype=torch.uint8, device=DEV)[:, 1:1 + q.scales.shape[1]]
    codes.copy_(q.codes)
    scales.copy_(q.scales)
    res = []
    for x8 in (q, (codes, scales)):
        dw = [torch.empty_like(v) for v in w]
        dx = torch.empty_like(dout)
        backward(dout, kept, w, dw, x8=x8, dx=dx)
        res.append([dx, *dw])
    assert all(torch.equal(a, b) for a, b in zip(*res))
    assert torch.equal(ffn.unpack8(ffn.Packed8(codes, scales)), ffn.unpack8(q))
    check_backward(dout, np64(ffn.unpack8(q)), kept, w, res[0])


@pytest.mark.parametrize("t,d,f", [(300, 200, 384), (2600, 136, 256), (19, 1808, 1024), (39, 2560, 512)])
@pytest.mark.parametrize("shift,pad", [(0, 0), (1, 1), (2, 2), (4, 6), (0, 4)])
def test_kept_codes_of_any_pitch_and_scales_at_any_address(t, d, f, shift, pad):
    """hidden a multiple of 128, where codes are read in 32-byte pieces and scales in fours
    if their addresses allow it: with padded codes and scale rows that begin anywhere."""
    g, x, *w = ffn_case(t, d, f, seed=63)
    dout = randn(g, t, d, scale=1e-2)
    want, kept = ffn.gated_ffn(x, *w)
    ng = f // 32
    mine = []
    for _ in range(2):
        codes = torch.zeros(t, f + 16 * pad, dtype=torch.uint8, device=DEV)[:, :f]
        scales = torch.zeros(t * (ng + pad) + shift, dtype=torch.uint8, device=DEV)
        mine.append((codes, scales[shift:].view(t, ng + pad)[:, :ng]))
    out = torch.empty_like(want)
    ws = torch.empty(dpo.dpo_ffn_workspace(t, d, f)[0], dtype=torch.uint8, device=DEV)
    dpo.dpo_ffn_forward(dpo.dpo_ffn_args(
        x=p(x), w_gate=p(w[0]), w_up=p(w[1]), w_down=p(w[2]), out=p(out), gate8=packed(*mine[0]),
        up8=packed(*mine[1]), tokens=t, dim=d, hidden=f, ld_x=d, ld_out=d, act=dpo.DPO_ACT_SILU,
        keep=dpo.DPO_KEEP_8BIT, workspace=p(ws), workspace_bytes=ws.numel()))
    assert torch.equal(out, want)
    for (c, s), k in zip(mine, (kept.gate, kept.up)):
        assert torch.equal(c, k.codes) and torch.equal(s, k.scales)
    res = []
    for k in (kept, ffn.Kept(ffn.Packed8(*mine[0]), ffn.Packed8(*mine[1]), "silu", "8bit")):
        dw = [torch.empty_like(v) for v in w]
        res.append([ffn.gated_ffn_backward(dout, k, *w, *dw, x=x), *dw])
    assert all(torch.equal(a, b) for a, b in zip(*res))
    assert ffn.status() == 0


def test_pitched_outputs_of_the_split_products():
    """out and dx with a pitch, written by the split form's own stores, nothing beside them."""
    t, d, f = 20, 512, 4096
    got = forms((t, d, f), "8bit", None)
    assert got[DOWN].kind == got[DX].kind == dpo.DPO_FFN_SPLIT
    g, x, *w = ffn_case(t, d, f, seed=64)
    dout = randn(g, t, d, scale=1e-2)
    want, kept = ffn.gated_ffn(x, *w)
    wide = [torch.full((t, d + 24), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    out, dx = (v[:, 8:8 + d] for v in wide)
    ffn.gated_ffn(x, *w, out=out)
    dw = [torch.empty_like(v) for v in w]
    wdx = ffn.gated_ffn_backward(dout, kept, *w, *dw, x=x)
    ffn.gated_ffn_backward(dout, kept, *w, *dw, x=x, dx=dx)
    assert torch.equal(out, want) and torch.equal(dx, wdx)
    for v in wide:
        assert (v[:, :8] == 7).all() and (v[:, 8 + d:] == 7).all()


@pytest.mark.parametrize("cols,pitch,at", [(96, 128, 0), (96, 99, 1), (1027, 1030, 2), (4096, 4100, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_8_bit_rows_at_any_address(cols, pitch, at, dtype):
    wide = torch.randn(37, pitch, generator=gen(cols), device=DEV).to(dtype)
    x = wide[:, at:at + cols]
    q = ffn.pack8(x)
    want = ffn.pack8(x.contiguous())
    assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)
    out = torch.full((37, pitch), 7.0, dtype=dtype, device=DEV)
    assert torch.equal(ffn.unpack8(q, out=out[:, at:at + cols]), ffn.unpack8(q, dtype=dtype))
    assert (out[:, :at] == 7).all() and (out[:, at + cols:] == 7).all()


@pytest.mark.parametrize("cols,at", [(767, 1), (768, 1), (1024, 2), (4096, 3)])
@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_norm_at_any_address(cols, at, dtype, wdtype):
    rows, g = 33, gen(cols + at)
    part = lambda s=1.0: randn(g, rows, cols + 5, scale=s, dtype=DT[dtype])[:, at:at + cols]
    x, r, dy, dh = part(), part(0.5), part(1e-2), part()
    w = (1 + randn(g, cols + 5, scale=0.2, dtype=DT[wdtype]))[at:at + cols]
    o = ffn.add_rms_norm(x, w, r, eps=1e-5, save8=True)
    y, s, rstd, _ = ref.rms_norm(np64(x), np64(w), float(np.float32(1e-5)), np64(r))
    within(o.rstd, rstd, 32 * U * rstd, "rstd")
    within(o.y, y, (RND[dtype] + 32 * U) * np.abs(y) + 1e-38, "y")
    within(o.h, s, (RND[dtype] + 2 * U) * np.abs(s), "h")
    n = np64(o.h) * np64(o.rstd)[:, None]
    d8 = ref.decode(o.x8.codes.cpu().numpy(), o.x8.scales.cpu().numpy())
    h = torch.empty(rows, cols + 5, dtype=DT[dtype], device=DEV)[:, at:at + cols].copy_(o.h)
    for arg, v in ((dict(h=h), n), (dict(x8=o.x8), d8)):
        dx, dw = ffn.add_rms_norm_backward(dy, w, o.rstd, dh=dh, **arg)
        wdx, wdw = ref.rms_norm_backward(np64(dy), np64(w), np64(o.rstd), v, np64(dh))
        gr = np.abs(np64(dy) * np64(w))
        mag = (np64(o.rstd)[:, None] * (gr + np.abs(v) * (gr * np.abs(v)).mean(1, keepdims=True)) +
               np.abs(np64(dh)))
        within(dx, wdx, RND[dtype] * np.abs(wdx) + 64 * U * mag + 1e-38, "dx")
        within(dw, wdw, (rows + 64) * U * np.abs(np64(dy) * v).sum(0) + 1e-38, "dweight")
