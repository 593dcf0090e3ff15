"""The feed-forward operators on the GPU against their 64-bit definitions
(oracle/ffn.py).

Where the bars come from. u = 2^-24 is fp32's half step and b = 2^-8 bf16's (relative).
- 8 bits: the codes and scales of given values are exact.
- Norm: a row's sum of squares is 32 fused steps per thread and a tree of at most ten
  more, so rstd is off by at most about 21 u + 3 u, and each product after it one u:
  32 u for fp32 outputs, b (1 + 2^-7) + 32 u for bf16 ones, of the magnitudes that
  enter the output.
- Products of K terms: fp32 accumulation, at worst (truncating) K 2u of the sum of the
  terms' magnitudes; a bf16 result adds b of itself. Errors of an operand pass through
  |operand| products, the gate's through |act'| <= 1.13 and its evaluation 2^-18.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import ffn as ref
from paper_2606_30634_gb300 import dpo, ffn

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8 * (1 + 2.0 ** -7)
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
RND = {"f32": 0.0, "bf16": B}
DEV = "cuda"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)


def np64(t):
    return t.detach().double().cpu().numpy()


def within(got, want, bar, what):
    got, bar = np64(got) if isinstance(got, torch.Tensor) else got, np.asarray(bar)
    assert got.shape == want.shape, what
    assert np.all(np.isfinite(got)), what
    over = np.abs(got - want) - bar
    assert np.all(over <= 0), f"{what}: {np.max(over):.3e} over its bar at {np.argmax(over)}"


# ---------------------------------------------------------------- 8 bits ----

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pitch", [
    (1, 1, 1), (3, 31, 31), (2, 32, 32), (5, 33, 40), (7, 100, 100), (4, 777, 777), (9, 1026, 1026),
    (6, 1024, 1032), (3, 4097, 4097), (300, 1555, 1555), (64, 4096, 4096), (1, 20000, 20000)])
def test_pack8_is_exact(dtype, rows, cols, pitch):
    g = gen(rows * 7919 + cols)
    full = torch.randn(rows, pitch, generator=g, device=DEV)
    full *= torch.exp2(torch.randint(-30, 30, (rows, pitch), generator=g, device=DEV).float())
    x = full.to(DT[dtype])[:, :cols]
    p = ffn.pack8(x)
    q, s = ref.encode(np64(x))
    assert np.array_equal(p.scales.cpu().numpy(), s)
    assert np.array_equal(p.codes.cpu().numpy(), q)
    want = ref.decode(q, s)
    assert np.array_equal(np64(ffn.unpack8(p)), want)          # bf16 holds them
    assert np.array_equal(np64(ffn.unpack8(p, dtype=torch.float32)), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pack8_special_values(dtype):
    x = torch.zeros(8, 64, device=DEV)
    x[0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 3.0])
    x[1] = float("nan")
    x[2, 5] = 1e-38
    x[3, :3] = torch.tensor([3e38, -3.3e38, 1.0])
    x[4, 40] = 448.0
    x[5, 40] = 449.0
    x[6, :2] = torch.tensor([1e-40, -1e-45])
    x[7, 33] = -0.0
    x = x.to(DT[dtype])
    p = ffn.pack8(x)
    q, s = ref.encode(np64(x))
    assert np.array_equal(p.scales.cpu().numpy(), s)
    got = ffn.unpack8(p, dtype=torch.float32).cpu().numpy()
    with np.errstate(over="ignore"):   # -3.3e38's code stands for -2^128: fp32's infinity
        want = ref.decode(q, s).astype(np.float32)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(got[0, :3]).all() and got[0, 3] == 3.0 and np.isnan(got[1]).all()


# ------------------------------------------------------------------ norm ----

NORM_SIZES = [(1, 1), (2, 8), (3, 33), (1, 4096), (5, 768), (9, 777), (4, 1025), (130, 2048),
              (3, 4098), (2, 8200), (2, 16384), (700, 64)]


def norm_case(rows, cols, dtype, wdtype, residual, seed=0):
    g = gen(seed + rows * 31 + cols)
    x = randn(g, rows, cols, dtype=DT[dtype])
    x[:, ::17] *= 20
    r = randn(g, rows, cols, scale=0.5, dtype=DT[dtype]) if residual else None
    w = 1 + randn(g, cols, scale=0.2, dtype=DT[wdtype])
    return g, x, r, w


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm(rows, cols, dtype, wdtype, residual):
    _, x, r, w = norm_case(rows, cols, dtype, wdtype, residual)
    if rows > 2:
        x[1] = 0                                  # an empty row
        if r is not None:
            r[1] = 0
    o = ffn.add_rms_norm(x, w, r, eps=1e-5, save8=True)
    y, s, rstd, n = ref.rms_norm(np64(x), np64(w), float(np.float32(1e-5)),
                                 None if r is None else np64(r))
    within(o.rstd, rstd, 32 * U * rstd, "rstd")
    within(o.y, y, (RND[dtype] + 32 * U) * np.abs(y) + 1e-38, "y")
    if residual:
        within(o.h, s, (RND[dtype] + 2 * U) * np.abs(s), "h")
    else:
        assert o.h is x
    # each 8-bit value within half a step of the row's own, whose fp32 form is 32 u off
    unit = np.exp2(np.repeat(o.x8.scales.cpu().numpy().astype(float) - 127, 32, 1)[:, :cols])
    d = ref.decode(o.x8.codes.cpu().numpy(), o.x8.scales.cpu().numpy())
    within(d, n, (2.0 ** -4 + 64 * U) * np.abs(n) + unit * 2.0 ** -10, "x8")
    want = ref.scale_bytes(n).astype(int)
    assert np.max(np.abs(o.x8.scales.cpu().numpy().astype(int) - want)) <= 1
    assert np.mean(o.x8.scales.cpu().numpy() != want) <= 0.01 or want.size < 200


@pytest.mark.parametrize("dtype,wdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("kept", ["h", "x8"])
def test_norm_backward(rows, cols, dtype, wdtype, kept):
    g, h, dh, w = norm_case(rows, cols, dtype, wdtype, rows % 2 == 1, seed=5)
    dy = randn(g, rows, cols, scale=1e-2, dtype=DT[dtype])
    if rows > 2:
        dy[2] = 0
    rstd = (1 / torch.sqrt(h.double().square().mean(1) + 1e-5)).float()
    if kept == "h":
        arg, n = dict(h=h), np64(h) * np64(rstd)[:, None]
    else:
        p = ffn.pack8(h.float() * rstd[:, None])
        arg, n = dict(x8=p), ref.decode(p.codes.cpu().numpy(), p.scales.cpu().numpy())
    dx, dw = ffn.add_rms_norm_backward(dy, w, rstd, dh=dh, **arg)
    wdx, wdw = ref.rms_norm_backward(np64(dy), np64(w), np64(rstd), n,
                                     None if dh is None else np64(dh))
    gr = np.abs(np64(dy) * np64(w))
    mag = np64(rstd)[:, None] * (gr + np.abs(n) * (gr * np.abs(n)).mean(1, keepdims=True))
    if dh is not None:
        mag = mag + np.abs(np64(dh))
    within(dx, wdx, RND[dtype] * np.abs(wdx) + 64 * U * mag + 1e-38, "dx")
    # a thread adds its rows in turn, then at most 40 more sums of partial rows
    within(dw, wdw, (rows + 64) * U * np.abs(np64(dy) * n).sum(0) + 1e-38, "dweight")
    acc = randn(g, cols, dtype=DT[wdtype])
    old = np64(acc)
    _, same = ffn.add_rms_norm_backward(dy, w, rstd, dh=dh, dweight=acc, accumulate=True, **arg)
    assert same is acc
    bar = (rows + 66) * U * (np.abs(np64(dy) * n).sum(0) + np.abs(old))
    within(acc, old + wdw, bar + RND[wdtype] * np.abs(old + wdw) + 1e-38, "accumulated dweight")


def test_norm_gradient_by_differences():
    """The fp32 kernels against each other: the backward is the forward's directional
    derivative. Step 2^-6 along a unit direction: truncation h^2 / 6 of the third
    derivative and rounding 32 u |y . dy| / h, both under 1e-3 of the derivative."""
    g = gen(11)
    x, w, dy = (torch.randn(s, generator=g, device=DEV) for s in ((4, 96), (96,), (4, 96)))
    v = torch.randn(4, 96, generator=g, device=DEV)
    h = 2.0 ** -6
    f = lambda z: (ffn.add_rms_norm(z, w).y.double() * dy.double()).sum().item()
    d = (f(x + h * v) - f(x - h * v)) / (2 * h)
    o = ffn.add_rms_norm(x, w)
    dx, _ = ffn.add_rms_norm_backward(dy, w, o.rstd, h=o.h)
    want = (dx.double() * v.double()).sum().item()
    assert abs(d - want) <= 5e-3 * max(1.0, abs(want)), (d, want)


# ------------------------------------------------------------------- ffn ----

def mags(*ts):
    return [np.abs(t) for t in ts]


def ffn_case(t, d, f, seed=0, pitch=0):
    g = gen(seed + t + 3 * d + 7 * f)
    x = randn(g, t, d + pitch)[:, :d]
    wg, wu, wd = randn(g, f, d, scale=d ** -0.5), randn(g, f, d, scale=d ** -0.5), randn(
        g, d, f, scale=f ** -0.5)
    return g, x, wg, wu, wd


def check_forward(x, w, kind, out, kept):
    X, WG, WU, WD = (np64(t) for t in (x, *w))
    out64, G, Uu, A = ref.ffn(X, WG, WU, WD, kind)
    aX, aWG, aWU, aWD = mags(X, WG, WU, WD)
    ek = 2 * U * X.shape[1]
    eg, eu = ek * (aX @ aWG.T), ek * (aX @ aWU.T)
    ea = 1.13 * eg * np.abs(Uu) + np.abs(ref.act(G, kind)[0]) * eu + (B + 2.0 ** -18) * np.abs(A)
    bar = ea @ aWD.T + 2 * U * A.shape[1] * (np.abs(A) @ aWD.T)
    within(out, out64, bar + B * (np.abs(out64) + bar) + 1e-30, "out")
    if kept is None:
        return
    for got, want, e in ((kept.gate, G, eg), (kept.up, Uu, eu)):
        if kept.keep == "bf16":
            within(got, want, e + B * (np.abs(want) + e), "kept")
        else:
            s = got.scales.cpu().numpy()
            v = ref.decode(got.codes.cpu().numpy(), s)
            unit = np.exp2(np.repeat(s.astype(float) - 127, 32, 1)[:, :want.shape[1]])
            within(v, want, (2.0 ** -4 + 2.0 ** -20) * (np.abs(want) + e) + e + unit * 2.0 ** -10,
                   "kept")
            assert np.max(np.abs(s.astype(int) - ref.scale_bytes(want).astype(int))) <= 1


def kept64(p, keep):
    return np64(p) if keep == "bf16" else ref.decode(p.codes.cpu().numpy(), p.scales.cpu().numpy())


def check_backward(dout, X, kept, w, got, old=None, rnd=B):
    """got: dx, dw_gate, dw_up, dw_down; X the block's input in 64 bits; old: what the
    weights' gradients were added to."""
    kind = kept.activation
    G, Uu = kept64(kept.gate, kept.keep), kept64(kept.up, kept.keep)
    DO, WG, WU, WD = (np64(t) for t in (dout, *w))
    dx, dwg, dwu, dwd, dg, du, a = ref.ffn_backward(DO, X, G, Uu, WG, WU, WD, kind)
    aDO, aX, aWG, aWU, aWD = mags(DO, X, WG, WU, WD)
    act, slope = ref.act(G, kind)
    da = np.abs(DO @ WD)
    eda = 2 * U * DO.shape[1] * (aDO @ aWD)
    ev = 2.0 ** -18 * (1 + np.abs(G))
    edg = np.abs(Uu * slope) * eda + (da + eda) * np.abs(Uu) * ev + B * np.abs(dg)
    edu = np.abs(act) * eda + (da + eda) * ev + B * np.abs(du)
    ea = np.abs(Uu) * ev + B * np.abs(a)
    t, f = G.shape
    bars = [edg @ aWG + edu @ aWU + 2 * U * 2 * f * (np.abs(dg) @ aWG + np.abs(du) @ aWU),
            edg.T @ aX + 2 * U * t * (np.abs(dg).T @ aX), edu.T @ aX + 2 * U * t * (np.abs(du).T @ aX),
            aDO.T @ ea + 2 * U * t * (aDO.T @ np.abs(a))]
    old = old or [0.0] * 3
    for name, g, want, bar, o in zip(("dx", "dw_gate", "dw_up", "dw_down"), got, (dx, dwg, dwu, dwd),
                                     bars, [0.0] + old):
        want = want + o
        r = B if name == "dx" else rnd
        within(g, want, bar + (r + 4 * U) * (np.abs(want) + bar) + 1e-30, name)


SIZES = [(1, 8, 8), (3, 64, 72), (7, 328, 136), (13, 328, 136), (25, 72, 520), (64, 264, 1000), (129, 136, 264), (300, 200, 328), (257, 512, 384), (40, 1032, 2072),
         (1001, 520, 1560)]


@pytest.mark.parametrize("t,d,f", SIZES)
@pytest.mark.parametrize("kind,keep", [("silu", "8bit"), ("gelu", "8bit"), ("silu", "bf16"),
                                       ("gelu", "none")])
def test_ffn_forward(t, d, f, kind, keep):
    _, x, *w = ffn_case(t, d, f, pitch=8 if t % 2 else 0)
    out, kept = ffn.gated_ffn(x, *w, activation=kind, keep=keep)
    check_forward(x, w, kind, out, kept)
    assert (kept is None) == (keep == "none")
    assert ffn.status() == 0


@pytest.mark.parametrize("t,d,f", SIZES)
@pytest.mark.parametrize("kind,keep,x8,grad", [
    ("silu", "8bit", True, "bf16"), ("gelu", "8bit", False, "f32"), ("silu", "bf16", False, "bf16"),
    ("gelu", "bf16", True, "f32")])
def test_ffn_backward(t, d, f, kind, keep, x8, grad):
    g, x, *w = ffn_case(t, d, f, seed=3)
    _, kept = ffn.gated_ffn(x, *w, activation=kind, keep=keep)
    dout = randn(g, t, d + 8, scale=1e-2)[:, :d]
    dw = [randn(g, *s.shape, scale=1e-2, dtype=DT[grad]) for s in w]
    X = np64(x)
    arg = dict(x=x)
    if x8:
        p, gain = ffn.pack8(x), 1 + randn(g, d, scale=0.2, dtype=DT[grad])
        arg = dict(x8=p, gain=gain)
        X = ref.decode(p.codes.cpu().numpy(), p.scales.cpu().numpy()) * np64(gain)
    first = [v.clone() for v in dw]
    dx = ffn.gated_ffn_backward(dout, kept, *w, *first, **arg)
    check_backward(dout, X, kept, w, [dx, *first], rnd=RND[grad])
    old = [np64(v) for v in dw]
    dx2 = ffn.gated_ffn_backward(dout, kept, *w, *dw, accumulate=True, **arg)
    assert torch.equal(dx, dx2)
    check_backward(dout, X, kept, w, [dx2, *dw], old, rnd=RND[grad])
    assert ffn.status() == 0


def test_ffn_by_cta_pairs():
    """Enough tiles that every launch goes to the pairs (more than four rounds of
    single CTAs), with ragged edges in every dimension; twice, bit for bit."""
    t, d, f = 2600, 1048, 4136
    g, x, *w = ffn_case(t, d, f, seed=9)
    p, gain = ffn.pack8(x), 1 + randn(g, d, scale=0.2)
    dout = randn(g, t, d, scale=1e-2)
    runs = []
    for _ in range(2):
        out, kept = ffn.gated_ffn(x, *w)
        dw = [torch.empty_like(v) for v in w]
        runs.append([out, ffn.gated_ffn_backward(dout, kept, *w, *dw, x8=p, gain=gain), *dw,
                     kept.gate.codes, kept.up.scales])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    check_forward(x, w, "silu", runs[0][0], kept)
    X = ref.decode(p.codes.cpu().numpy(), p.scales.cpu().numpy()) * np64(gain)
    check_backward(dout, X, kept, w, runs[0][1:5])
    assert ffn.status() == 0


@pytest.mark.parametrize("keep", ["8bit", "bf16"])
def test_ffn_by_cta_pairs_in_whole_chunks(keep):
    """hidden a multiple of 128: what is kept is read in aligned 32-byte pieces."""
    t, d, f = 2500, 520, 4096
    g, x, *w = ffn_case(t, d, f, seed=2)
    dout = randn(g, t, d, scale=1e-2)
    out, kept = ffn.gated_ffn(x, *w, activation="gelu", keep=keep)
    dw = [torch.zeros_like(v) for v in w]
    dx = ffn.gated_ffn_backward(dout, kept, *w, *dw, x=x)
    check_forward(x, w, "gelu", out, kept)
    check_backward(dout, np64(x), kept, w, [dx, *dw])
    assert ffn.status() == 0


def test_ffn_non_finite_tokens_stay_in_their_rows():
    _, x, *w = ffn_case(200, 136, 264)
    clean, _ = ffn.gated_ffn(x, *w)
    x = x.clone()
    x[7, 3], x[150, 9] = float("nan"), float("inf")
    out, kept = ffn.gated_ffn(x, *w)
    bad = torch.tensor([7, 150], device=DEV)
    keep = torch.ones(200, dtype=torch.bool, device=DEV)
    keep[bad] = False
    assert torch.equal(out[keep], clean[keep]) and not torch.isfinite(out[bad]).any()
    assert torch.isnan(ffn.unpack8(kept.gate)[bad]).all()


def test_empty_calls():
    g, x, *w = ffn_case(4, 64, 72)
    e = x[:0]
    out, kept = ffn.gated_ffn(e, *w)
    dw = [torch.ones_like(v) for v in w]
    dx = ffn.gated_ffn_backward(e, kept, *w, *dw, x=e, accumulate=True)
    assert out.shape == dx.shape == (0, 64) and all((v == 1).all() for v in dw)
    ffn.gated_ffn_backward(e, kept, *w, *dw, x=e)
    assert all((v == 0).all() for v in dw)
    o = ffn.add_rms_norm(e, w[0][0], save8=True)
    _, dwn = ffn.add_rms_norm_backward(e, w[0][0], o.rstd, x8=o.x8)
    assert (dwn == 0).all() and ffn.unpack8(ffn.pack8(e)).shape == (0, 64)


def test_offsets_past_32_bits():
    """Rows 2^32 elements apart (norm, 8 bits) and 2^26 apart over 130 rows (ffn)."""
    big = torch.zeros((1 << 33) + 4096, dtype=torch.bfloat16, device=DEV)
    x = big.as_strided((3, 4096), (1 << 32, 1))
    x.copy_(randn(gen(1), 3, 4096))
    w = 1 + randn(gen(2), 4096, scale=0.1)
    a, b = ffn.add_rms_norm(x, w, save8=True), ffn.add_rms_norm(x.contiguous(), w, save8=True)
    assert torch.equal(a.y, b.y) and torch.equal(a.x8.codes, b.x8.codes)
    assert torch.equal(ffn.pack8(x).codes, ffn.pack8(x.contiguous()).codes)
    da, _ = ffn.add_rms_norm_backward(x, w, a.rstd, h=x)
    db, _ = ffn.add_rms_norm_backward(x.contiguous(), w, a.rstd, h=x.contiguous())
    assert torch.equal(da, db)
    _, y, *ws = ffn_case(130, 64, 72)
    z = big.as_strided((128, 64), (1 << 26, 1))
    z.copy_(y[:128])
    assert torch.equal(ffn.gated_ffn(z, *ws)[0], ffn.gated_ffn(y[:128], *ws)[0])


def test_other_streams_and_graphs():
    g, x, *w = ffn_case(77, 136, 264)
    dout = randn(g, 77, 136, scale=1e-2)
    wn = 1 + randn(g, 136, scale=0.1)

    def step(stream=None):
        n = ffn.add_rms_norm(x, wn, x, save8=True, stream=stream)
        out, kept = ffn.gated_ffn(n.y, *w, stream=stream)
        dw = [torch.empty_like(v) for v in w]
        dy = ffn.gated_ffn_backward(dout, kept, *w, *dw, x8=n.x8, gain=wn, stream=stream)
        dx, dwn = ffn.add_rms_norm_backward(dy, wn, n.rstd, x8=n.x8, dh=dout, stream=stream)
        return [out, dx, dwn, *dw]

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = step()
    for v in cap:
        v.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, cap))


def test_refusals_of_tensors():
    g, x, wg, wu, wd = ffn_case(4, 64, 72)
    with pytest.raises(ValueError):
        ffn.gated_ffn(x.cpu(), wg, wu, wd)
    with pytest.raises(ValueError):
        ffn.gated_ffn(x.t(), wg, wu, wd)
    with pytest.raises(TypeError):
        ffn.gated_ffn(x.float(), wg, wu, wd)
    with pytest.raises(ValueError):
        ffn.gated_ffn(x, wg, wu[:8], wd)
    with pytest.raises(ValueError):
        ffn.gated_ffn(x, wg, wu, wd, activation="relu")
    with pytest.raises(dpo.DpoError) as e:
        ffn.gated_ffn(x[:, :60].contiguous(), wg[:, :60].contiguous(), wu[:, :60].contiguous(),
                      wd[:60].contiguous())
    assert e.value.code == dpo.DPO_EINVAL
    out, kept = ffn.gated_ffn(x, wg, wu, wd)
    dw = [torch.empty_like(v) for v in (wg, wu, wd)]
    with pytest.raises(ValueError):
        ffn.gated_ffn_backward(out, kept, wg, wu, wd, *dw)
    with pytest.raises(ValueError):
        ffn.gated_ffn_backward(out, None, wg, wu, wd, *dw, x=x)
    with pytest.raises(dpo.DpoError):
        ffn.gated_ffn_backward(out, kept, wg, wu, wd, dw[0], dw[0], dw[2], x=x)
    with pytest.raises(TypeError):
        ffn.pack8(x.half())
    with pytest.raises(ValueError):
        ffn.add_rms_norm(x, wg[0][:32])
    with pytest.raises(ValueError):
        ffn.add_rms_norm_backward(x, wg[0], torch.ones(4, device=DEV))
    with pytest.raises(ValueError):
        ffn.add_rms_norm_backward(x, wg[0], torch.ones(4, device=DEV), h=x, accumulate=True)
