"""What the feed-forward calls take and give as tensors: shapes, strides, addresses,
streams, and what was kept after it has been away. The numbers are those of the same
call on plain tensors, bit for bit, which test_ffn_gpu.py compares with the definitions.
"""
from __future__ import annotations

import pytest
import torch

from paper_2606_30634_gb300 import ffn
from test_ffn_gpu import DEV, ffn_case, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(7,), (4, 33), (2, 3, 40), (2, 1, 3, 64), (0, 5, 64)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_pack8_keeps_the_shape(shape, dtype):
    x = randn(gen(1), *shape, dtype=dtype)
    p = ffn.pack8(x)
    assert p.shape == p.codes.shape == x.shape
    assert p.scales.shape == (*shape[:-1], -(-shape[-1] // 32))
    flat = ffn.pack8(x.reshape(-1, shape[-1]))
    assert torch.equal(p.codes.view(flat.codes.shape), flat.codes)
    assert torch.equal(p.scales.view(flat.scales.shape), flat.scales)
    back = ffn.unpack8(p)
    assert back.shape == x.shape and torch.equal(back.view(flat.codes.shape), ffn.unpack8(flat))


def test_the_norms_8_bit_rows_keep_the_shape():
    g = gen(2)
    x, w, dy = randn(g, 2, 5, 72), 1 + randn(g, 72, scale=0.1), randn(g, 2, 5, 72)
    o = ffn.add_rms_norm(x, w, save8=True)
    assert o.y.shape == o.x8.shape == ffn.unpack8(o.x8).shape == x.shape
    flat = ffn.add_rms_norm(x.view(10, 72), w, save8=True)
    assert torch.equal(o.x8.codes.view(10, 72), flat.x8.codes)
    dx, dw = ffn.add_rms_norm_backward(dy, w, o.rstd, x8=o.x8)
    dx2, dw2 = ffn.add_rms_norm_backward(dy.view(10, 72), w, o.rstd, x8=flat.x8)
    assert dx.shape == x.shape and torch.equal(dx.view(10, 72), dx2) and torch.equal(dw, dw2)


def away(p):
    """A Packed8 moved to the host and back: contiguous, without the pitch it had."""
    return ffn.Packed8(p.codes.cpu().to(DEV), p.scales.cpu().to(DEV))


@pytest.mark.parametrize("t,d,f", [(1, 64, 72), (7, 328, 136), (300, 200, 328), (1001, 520, 1560),
                                   (23, 2400, 1096)])
def test_what_was_kept_may_have_been_on_the_host(t, d, f):
    g, x, *w = ffn_case(t, d, f)
    _, kept = ffn.gated_ffn(x, *w)
    back = ffn.Kept(away(kept.gate), away(kept.up), kept.activation, kept.keep)
    assert t == 1 or f % 32 == 0 or back.gate.codes.stride() != kept.gate.codes.stride()
    dout = randn(g, t, d, scale=1e-2)
    res = []
    for k in (kept, back):
        dw = [torch.empty_like(v) for v in w]
        res.append([ffn.gated_ffn_backward(dout, k, *w, *dw, x=x), *dw])
    assert all(torch.equal(a, b) for a, b in zip(*res))
    assert ffn.status() == 0
