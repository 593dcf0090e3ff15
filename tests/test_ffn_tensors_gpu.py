"""What the feed-forward calls take and give as tensors: shapes, strides, addresses,
streams, and what was kept after it has been away. The numbers are those of the same
call on plain tensors, bit for bit, which test_ffn_gpu.py compares with the definitions.
"""
from __future__ import annotations

import threading

import pytest
import torch

from paper_2606_30634_gb300 import dpo, ffn, muon
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


def beside(g, rows, cols):
    """A random matrix and an empty one in the columns to its right, in one buffer."""
    buf = randn(g, rows, 2 * cols)
    return buf[:, :cols], buf[:, cols:], buf


@pytest.mark.parametrize("t,d,f", [(5, 64, 72), (40, 264, 520), (300, 200, 328), (2600, 136, 264),
                                   (23, 2056, 1096)])
@pytest.mark.parametrize("side", [0, 1])
def test_outputs_beside_inputs(t, d, f, side):
    """out and dx in the columns beside x and dout: nothing but their own columns changes."""
    g, _, *w = ffn_case(t, d, f)
    x, out, buf = beside(g, t, d)
    dout, dx, dbuf = beside(g, t, d)
    if side:
        x, out, dout, dx = out, x, dx, dout
    x0, dout0 = x.clone(), dout.clone()
    want, kept = ffn.gated_ffn(x0, *w, keep="bf16")
    dw = [torch.empty_like(v) for v in w]
    wdx = ffn.gated_ffn_backward(dout0, kept, *w, *dw, x=x0)
    got, _ = ffn.gated_ffn(x, *w, keep="bf16", out=out)
    gdx = ffn.gated_ffn_backward(dout, kept, *w, *dw, x=x, dx=dx)
    assert got is out and gdx is dx
    assert torch.equal(out, want) and torch.equal(dx, wdx)
    assert torch.equal(x, x0) and torch.equal(dout, dout0)
    assert ffn.status() == 0


@pytest.mark.parametrize("rows,cols", [(1, 64), (7, 72), (300, 1000), (2003, 33)])
def test_norm_outputs_beside_its_inputs(rows, cols):
    g = gen(rows)
    x, y, _ = beside(g, rows, cols)
    r, h, _ = beside(g, rows, cols)
    dy, dx, _ = beside(g, rows, cols)
    w = 1 + randn(g, cols, scale=0.1)
    x0, r0, dy0 = x.clone(), r.clone(), dy.clone()
    want = ffn.add_rms_norm(x0, w, r0)
    rstd = torch.empty_like(want.rstd)
    p, ld = (lambda v: v.data_ptr()), 2 * cols
    dpo.dpo_rmsnorm(dpo.dpo_rmsnorm_args(
        x=p(x), residual=p(r), weight=p(w), h=p(h), y=p(y), rstd=p(rstd), rows=rows, cols=cols,
        ld_x=ld, ld_residual=ld, ld_h=ld, ld_y=ld, eps=1e-5, dtype=dpo.DPO_BF16,
        weight_dtype=dpo.DPO_BF16))
    wdx, _ = ffn.add_rms_norm_backward(dy0, w, rstd, h=want.h)
    dpo.dpo_rmsnorm_backward(dpo.dpo_rmsnorm_backward_args(
        dy=p(dy), h=p(h), rstd=p(rstd), weight=p(w), dx=p(dx), rows=rows, cols=cols, ld_dy=ld,
        ld_h=ld, ld_dx=ld, dtype=dpo.DPO_BF16, weight_dtype=dpo.DPO_BF16))
    for a, b in ((y, want.y), (h, want.h), (rstd, want.rstd), (dx, wdx), (x, x0), (r, r0), (dy, dy0)):
        assert torch.equal(a, b)


def test_weights_of_an_optimizer(cuda_device):
    """The stale weights of both optimizers: in bf16 they are what the block takes; the fp32
    ones of a default DelayedAdamW are refused with what to do, and are fine in the norm."""
    t, d, f = 9, 64, 72
    g, x, *w = ffn_case(t, d, f)
    want, _ = ffn.gated_ffn(x, *w)
    shapes = [v.shape for v in w]
    start = [v.float().flatten() for v in w]
    sets = [dpo.DelayedAdamW([v.numel() for v in w], stash_dtype=dpo.DPO_BF16, x0=start),
            muon.DelayedMuon([tuple(s) for s in shapes], x0=[v.float() for v in w]),
            dpo.DelayedAdamW([v.numel() for v in w] + [d], x0=start + [torch.ones(d, device=DEV)])]
    try:
        for o in sets[:2]:
            stale = [o.stale(i).view(s) for i, s in enumerate(shapes)]
            out, kept = ffn.gated_ffn(x, *stale)
            assert torch.equal(out, want)
        wide = [sets[2].stale(i).view(s) for i, s in enumerate(shapes)]
        with pytest.raises(TypeError, match="stash_dtype=DPO_BF16"):
            ffn.gated_ffn(x, *wide)
        dw = [torch.empty_like(v) for v in w]
        for k in range(3):
            with pytest.raises(TypeError, match=("w_gate", "w_up", "w_down")[k] + ".*stash_dtype"):
                ffn.gated_ffn_backward(x, kept, *w[:k], wide[k], *w[k + 1:], *dw, x=x)
        o = ffn.add_rms_norm(x, sets[2].stale(3))
        assert torch.equal(o.y, ffn.add_rms_norm(x, torch.ones(d, device=DEV)).y)
    finally:
        for o in sets:
            o.close()


def test_threads_and_streams_at_once():
    """Four host threads, each with a stream and sizes of its own, step at once; each gets what
    it gets alone, and an error of one is not another's."""
    sizes = [(5, 264, 520), (77, 136, 264), (900, 520, 1560), (20, 512, 4096)]
    jobs = []
    for i, (t, d, f) in enumerate(sizes):
        g, x, *w = ffn_case(t, d, f, seed=70 + i)
        jobs.append((x, w, 1 + randn(g, d, scale=0.1), randn(g, t, d, scale=1e-2)))

    def step(x, w, wn, dout):
        n = ffn.add_rms_norm(x, wn, x, save8=True)
        out, kept = ffn.gated_ffn(n.y, *w)
        dw = [torch.empty_like(v) for v in w]
        dy = ffn.gated_ffn_backward(dout, kept, *w, *dw, x8=n.x8, gain=wn)
        dx, dwn = ffn.add_rms_norm_backward(dy, wn, n.rstd, x8=n.x8, dh=dout)
        return [out, dx, dwn, *dw]

    want = [step(*j) for j in jobs]
    torch.cuda.synchronize()
    got, wrong = [None] * len(jobs), []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for k in range(20):
                    got[i] = step(*jobs[i])
                    with pytest.raises(dpo.DpoError, match="dpo_ffn_forward: out"):
                        ffn.gated_ffn(jobs[i][0], *jobs[i][1], out=jobs[i][0])
            stream.synchronize()
        except BaseException as e:
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong
    for a, b in zip(want, got):
        assert all(torch.equal(u, v) for u, v in zip(a, b))
    assert ffn.status() == 0
