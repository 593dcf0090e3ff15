"""The loops of the persistent kernels: rows that a CTA of the norm's backward takes one
after another, spans that a warp of the 8-bit kernels walks. Bars as in
test_ffn_gpu.py.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import ffn as ref
from paper_2606_30634_gb300 import ffn
from test_ffn_gpu import DEV, DT, RND, U, ffn_case, gen, norm_case, np64, randn, within

pytestmark = pytest.mark.gpu

# Six row sets or more to a CTA of 152 SMs, and a ragged last one: 16 warps an SM, a row of 1
# to 16 warps; in 16-byte pieces (the ring; fp32 above 4096 and all above 8192 columns from
# registers), in pieces of two and of one element.
LOOPS = [(17001, 64), (15001, 768), (7003, 777), (4003, 2048), (4003, 2050), (2003, 4096), (1003, 8192),
         (1003, 8200), (1003, 8198), (1003, 8199)]


def back_shape(rows, cols, sms):
    """(row sets, CTAs) of the norm's backward."""
    warps = 1
    while warps * 32 * (16 if cols <= 8192 else 32) < cols:
        warps *= 2
    cta = max(warps, 8)
    sets = -(-rows // (cta // warps))
    return sets, min(sets, sms * (16 // cta))


@pytest.mark.parametrize("rows,cols", LOOPS)
@pytest.mark.parametrize("dtype,wdtype", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("kept", ["h", "x8"])
def test_norm_backward_over_many_rows(rows, cols, dtype, wdtype, kept):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    sets, ctas = back_shape(rows, cols, sms)
    assert sets > 5 * ctas and sets % ctas != 0
    g, h, dh, w = norm_case(rows, cols, dtype, wdtype, True, seed=51)
    dy = randn(g, rows, cols, scale=1e-2, dtype=DT[dtype])
    rstd = (1 / torch.sqrt(h.double().square().mean(1) + 1e-5)).float()
    if kept == "h":
        arg, n = dict(h=h), np64(h) * np64(rstd)[:, None]
    else:
        p = ffn.pack8(h.float() * rstd[:, None])
        arg, n = dict(x8=p), ref.decode(p.codes.cpu().numpy(), p.scales.cpu().numpy())
    dx, dw = ffn.add_rms_norm_backward(dy, w, rstd, dh=dh, **arg)
    again = ffn.add_rms_norm_backward(dy, w, rstd, dh=dh, **arg)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
    wdx, wdw = ref.rms_norm_backward(np64(dy), np64(w), np64(rstd), n, np64(dh))
    gr = np.abs(np64(dy) * np64(w))
    mag = (np64(rstd)[:, None] * (gr + np.abs(n) * (gr * np.abs(n)).mean(1, keepdims=True)) +
           np.abs(np64(dh)))
    within(dx, wdx, RND[dtype] * np.abs(wdx) + 64 * U * mag + 1e-38, "dx")
    within(dw, wdw, (rows + 64) * U * np.abs(np64(dy) * n).sum(0) + 1e-38, "dweight")


def plain_encode(x):
    """Codes and scale bytes by elementary operations, all exact but the rounding to E4M3."""
    rows, cols = x.shape
    groups = torch.nn.functional.pad(x.float(), (0, -cols % 32)).view(rows, -1, 32)
    m, e = torch.frexp(groups.abs().amax(-1))
    e = torch.where(m > 0, torch.where(m > 0.875, e - 8, e - 9).clamp(min=-126), -126)
    q = torch.ldexp(groups, -e[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return q.view(rows, -1)[:, :cols], (e + 127).to(torch.uint8)


def spans(rows, cols, elems):
    return rows * -(-cols // elems)


# More spans than the 4 x 152 CTAs of packing (32 warps an SM) or the 64 x 152 of widening
# hold, with a number of spans to a row that does not divide them: pieces of 8 (4) elements
# in spans of 1024, of two in 512, of one in 256.
@pytest.mark.parametrize("dtype,rows,cols,pitch,elems", [
    ("bf16", 3001, 4104, 4104, 1024), ("f32", 3001, 4100, 4100, 1024), ("bf16", 3001, 2050, 2050, 512),
    ("f32", 3001, 1555, 1555, 256), ("bf16", 16001, 1555, 1555, 256), ("f32", 16001, 1553, 1555, 256),
    ("bf16", 27001, 4104, 4112, 1024)])
def test_pack_and_unpack_over_many_spans(dtype, rows, cols, pitch, elems):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    n = spans(rows, cols, elems)
    assert n > sms * 4 * 8 and sms * 4 * 8 % -(-cols // elems) != 0
    if rows > 10000:
        assert n > sms * 64 * 8
    x = torch.randn(rows, pitch, generator=gen(rows + cols), device=DEV).to(DT[dtype])[:, :cols]
    p = ffn.pack8(x)
    q, s = plain_encode(x)
    assert torch.equal(p.codes, q) and torch.equal(p.scales, s)
    want = torch.ldexp(q.view(torch.float8_e4m3fn).float(),
                       s.int().repeat_interleave(32, 1)[:, :cols] - 127)
    assert torch.equal(ffn.unpack8(p, dtype=DT[dtype]), want.to(DT[dtype]))   # exact in both


@pytest.mark.parametrize("t,d,f", [(40000, 1032, 72), (27001, 2056, 24)])
def test_8_bit_rows_of_many_tokens_in_the_backward(t, d, f):
    """The rows are widened beside the gate's backward, several spans to a warp: the same
    gradients as from the widened rows."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert spans(t, d, 1024) > sms * 64 * 8
    g, x, *w = ffn_case(t, d, f, seed=52)
    _, kept = ffn.gated_ffn(x, *w)
    p, dout = ffn.pack8(x), randn(g, t, d, scale=1e-2)
    res = []
    for arg in (dict(x8=p), dict(x=ffn.unpack8(p))):
        dw = [torch.empty_like(v) for v in w]
        res.append([ffn.gated_ffn_backward(dout, kept, *w, *dw, **arg), *dw])
    assert all(torch.equal(a, b) for a, b in zip(*res))
    assert ffn.status() == 0
