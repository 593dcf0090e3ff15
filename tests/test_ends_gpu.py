"""The operators of a pipeline's ends on the GPU against their 64-bit definitions
(oracle/ends.py).

Where the bars come from. u = 2^-24 is fp32's half step and b = 2^-8 bf16's (relative).
- Embedding: one product in fp32, then the output's rounding. Its gradient: n terms, one u of
  the sum of their magnitudes each, two products.
- Dropout: the mask is exact; a product with a rounded factor, a sum.
- A row's distribution: z, its maximum m and d = z - m carry u (|z| + |m| + |d|); e^d by
  ex2.approx (2^-22) of d log2(e), another 1.5 u |d|. A thread adds n of them one after the
  other, u each, and 64 more joining threads and warps; a maximum that rises multiplies the sum
  by another exponential (2^-22), in random order about log(n) times, 16 are allowed for.
- The gradient: the errors of z - m - log S pass into p, whose exponential has 2^-20 (bf16
  results) or 2^-22; then a handful of u.
- Products of K terms: fp32 accumulation, at worst (truncating, 16 terms at a time, two steps
  each) K/4 u of the sum of the terms' magnitudes. G is rounded to bf16 for its products, and what is
  kept for it may be rounded to 2^-11.
"""
from __future__ import annotations

import math
import threading

import numpy as np
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from oracle import ends as ref
from paper_2606_30634_gb300 import dpo, ends, ffn
from test_ffn_gpu import B, DEV, DT, RND, U, gen, np64, randn, within

pytestmark = pytest.mark.gpu

TINY = 1e-38
f32 = np.float32


def ids_of(g, shape, vocab, padding=True):
    """Some ids common, some padding of each kind."""
    u = torch.rand(shape, generator=g, device=DEV)
    ids = (u ** 3 * vocab).long().clamp(max=vocab - 1)
    if padding:
        r = torch.rand(shape, generator=g, device=DEV)
        for cut, value in ((0.03, -1), (0.06, -100), (0.09, vocab), (0.11, 2 ** 40), (0.12, -2 ** 63)):
            ids = torch.where((r >= cut - 0.03) & (r < cut), value, ids)
    return ids


# ------------------------------------------------------------- embedding ----

EMBED = [(1, 1, 1), (1, 10, 4096), (7, 5, 8), (3, 100, 33), (257, 50, 520), (1000, 5003, 777),
         (33, 70, 2050), (5, 7, 9000), (2048, 300, 256)]


@pytest.mark.parametrize("tokens,vocab,dim", EMBED)
@pytest.mark.parametrize("td", ["f32", "bf16"])
@pytest.mark.parametrize("od", ["f32", "bf16"])
def test_embed(tokens, vocab, dim, td, od):
    g = gen(tokens + dim)
    table, ids = randn(g, vocab, dim, dtype=DT[td]), ids_of(g, (tokens,), vocab)
    out = ends.embed(ids, table, scale=1.7, dtype=DT[od])
    want = ref.embed(ids.cpu().numpy(), np64(table), float(f32(1.7)))
    assert out.dtype is DT[od] and out.shape == (tokens, dim)
    within(out, want, (RND[od] + 2 * U) * np.abs(want) + TINY, "out")
    same = ends.embed(ids, table)
    assert same.dtype is DT[td]
    within(same, ref.embed(ids.cpu().numpy(), np64(table)), 0.0, "unscaled rows")


def check_embed_backward(dy, ids, vocab, scale, gd, **kw):
    dim = dy.shape[-1]
    want, mag, count = ref.embed_backward(np64(dy), ids.cpu().numpy(), vocab, float(f32(scale)))
    dtable = torch.full((vocab, dim), 7.0, dtype=DT[gd], device=DEV)
    got = ends.embed_backward(dy, ids, dtable, scale=scale, **kw)
    assert got is dtable
    bar = (count[:, None] + 3) * U * mag
    within(dtable, want, bar + RND[gd] * np.abs(want) + TINY, "dtable")
    assert torch.equal(dtable[torch.from_numpy(count == 0).to(DEV)],
                       torch.zeros(int((count == 0).sum()), dim, dtype=DT[gd], device=DEV))
    old = randn(gen(3), vocab, dim, dtype=DT[gd])
    acc = old.clone()
    ends.embed_backward(dy, ids, acc, scale=scale, accumulate=True, **kw)
    total = want + np64(old)
    within(acc, total, bar + 2 * U * (mag + np.abs(np64(old))) + RND[gd] * np.abs(total) + TINY, "added")
    absent = torch.from_numpy(count == 0).to(DEV)
    assert torch.equal(acc[absent], old[absent])
    return dtable


@pytest.mark.parametrize("tokens,vocab,dim", EMBED + [(9000, 300, 24), (40000, 5000, 8), (20000, 70000, 5)])
@pytest.mark.parametrize("dd", ["f32", "bf16"])
@pytest.mark.parametrize("gd", ["f32", "bf16"])
def test_embed_backward(tokens, vocab, dim, dd, gd):
    g = gen(tokens + dim)
    dy, ids = randn(g, tokens, dim, dtype=DT[dd]), ids_of(g, (tokens,), vocab)
    first = check_embed_backward(dy, ids, vocab, 0.3, gd)
    again = ends.embed_backward(dy, ids, torch.empty_like(first), scale=0.3)
    assert torch.equal(first, again)   # its order is fixed


@pytest.mark.parametrize("tokens", [1, 31, 32, 33, 500, 8192, 8193, 65536])
@pytest.mark.parametrize("kind", ["one id", "all different", "padding", "two runs", "descending"])
def test_embed_backward_of_runs(tokens, kind):
    """Runs that begin and end at, before and behind the ends of chunks and of the sort's CTAs."""
    n, dim = torch.arange(tokens, device=DEV), 12
    ids = {"one id": torch.full_like(n, 3), "all different": (n * 7919) % 65537, "padding": torch.full_like(n, -1),
           "two runs": (n >= tokens // 2 - 1).long() * 5 + 1, "descending": tokens - 1 - n}[kind]
    dy = randn(gen(tokens), tokens, dim, dtype=torch.float32)
    check_embed_backward(dy, ids, 65537 if kind in ("all different", "descending") else 9, 1.0, "f32")


def test_embed_backward_of_more_than_a_span():
    """131100 tokens in three spans: an fp32 buffer within the bar of one sum, a bf16 one rounded
    twice more (its old value and the sum each pass a rounding of at most the row's magnitude)."""
    g = gen(4)
    tokens, vocab, dim = 2 * ends.DPO_EMBED_SPAN + 28, 61, 8
    dy, ids = randn(g, tokens, dim), ids_of(g, (tokens,), vocab)
    check_embed_backward(dy, ids, vocab, 1.0, "f32")
    want, mag, count = ref.embed_backward(np64(dy), ids.cpu().numpy(), vocab)
    got = ends.embed_backward(dy, ids, torch.empty(vocab, dim, dtype=torch.bfloat16, device=DEV))
    within(got, want, (count[:, None] + 9) * U * mag + 3 * B * mag, "bf16")


@pytest.mark.parametrize("dim,pitch,shift", [(64, 72, 0), (64, 65, 0), (64, 66, 2), (40, 48, 8), (33, 37, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_embed_pitches_and_addresses(dim, pitch, shift, dtype):
    g = gen(dim + pitch + shift)
    vocab, dt = 50, DT[dtype]
    table = randn(g, vocab, pitch + shift, dtype=dt)[:, shift:shift + dim]
    ids = ids_of(g, (3, 41), vocab)
    buf = torch.full((3, 41, pitch + shift), 5.0, dtype=dt, device=DEV)
    out = buf[..., shift:shift + dim]
    assert ends.embed(ids, table, out=out) is out
    assert torch.equal(out, ends.embed(ids, table.contiguous()))
    assert (buf[..., :shift] == 5).all() and (buf[..., shift + dim:] == 5).all()
    dy = randn(g, 3, 41, pitch + shift, dtype=dt)[..., shift:shift + dim]
    grads = torch.full((vocab, pitch + shift), 5.0, dtype=dt, device=DEV)
    d = grads[:, shift:shift + dim]
    ends.embed_backward(dy, ids, d)
    assert torch.equal(d, ends.embed_backward(dy.contiguous(), ids, torch.empty(vocab, dim, dtype=dt, device=DEV)))
    assert (grads[:, :shift] == 5).all() and (grads[:, shift + dim:] == 5).all()


def test_ids_of_a_batch():
    """Slices of a batch of tokens, int32 ids, a single id."""
    g = gen(5)
    tokens = ids_of(g, (6, 30), 100)
    table = randn(g, 100, 16)
    for ids in (tokens[:, :-1], tokens[:, 1:], tokens[2], tokens[::2, 3:9], tokens[:, 4:5], tokens[3, 7]):
        small = torch.where((ids < 0) | (ids >= 100), -1, ids)
        want = ends.embed(ids.contiguous(), table)
        assert want.shape == ids.shape + (16,)
        assert torch.equal(ends.embed(ids, table), want)
        assert torch.equal(ends.embed(small.int(), table), want)
        dy = randn(g, *ids.shape, 16)
        d = [ends.embed_backward(dy, i, torch.empty(100, 16, device=DEV)) for i in (ids, ids.contiguous(), small.int())]
        assert torch.equal(d[0], d[1]) and torch.equal(d[0], d[2])
    with pytest.raises(ValueError):
        ends.embed(tokens.t(), table)
    with pytest.raises(TypeError):
        ends.embed(tokens.float(), table)
    with pytest.raises(ValueError):
        ends.embed(tokens.cpu(), table)
    with pytest.raises(ValueError):
        ends.embed_backward(randn(g, 5, 30, 16), tokens, torch.empty(100, 16, device=DEV))


def test_no_tokens():
    table = randn(gen(1), 10, 16)
    none = torch.empty(0, dtype=torch.long, device=DEV)
    assert ends.embed(none, table).shape == (0, 16)
    d = torch.ones(10, 16, device=DEV)
    ends.embed_backward(table[:0], none, d, accumulate=True)
    assert (d == 1).all()
    wide = torch.ones(10, 24, device=DEV)
    ends.embed_backward(table[:0], none, wide[:, :16])
    assert (wide[:, :16] == 0).all() and (wide[:, 16:] == 1).all()


def test_embed_takes_infinities_as_they_are():
    table = torch.zeros(3, 8, device=DEV)
    table[0], table[1] = math.inf, math.nan
    out = ends.embed(torch.tensor([0, 1, -1, 2], device=DEV), table, scale=0.5)
    assert (out[0] == math.inf).all() and out[1].isnan().all() and (out[2:] == 0).all()
    dy = torch.full((2, 8), math.nan, device=DEV)
    d = ends.embed_backward(dy, torch.tensor([-1, 7], device=DEV), torch.empty(3, 8, device=DEV))
    assert (d == 0).all()   # padding's gradient is not looked at


@pytest.mark.parametrize("tokens", [1, 200, 8192])
@pytest.mark.parametrize("vocab", [2 ** 18 - 1, 2 ** 18, 300001])
def test_embed_backward_of_large_vocabularies(tokens, vocab):
    """Ids on both sides of what the comparing sort packs beside a token's number."""
    g = gen(tokens + vocab)
    ids = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
    ids[-1] = vocab - 1
    if tokens > 1:
        ids[0], ids[1] = vocab - 1, vocab
    check_embed_backward(randn(g, tokens, 2), ids, vocab, 1.0, "f32")


@pytest.mark.parametrize("dim,pitch", [(8, 8), (33, 33), (40, 50), (2100, 2100), (5, 5000)])
@pytest.mark.parametrize("gd", ["f32", "bf16"])
def test_embed_gradient_is_cleared_to_its_edges(dim, pitch, gd):
    """Rows that begin and end anywhere: all of dtable is zero where no id is, nothing beside it."""
    for shift in (0, 1, 3):
        buf = torch.full((70, pitch + 4), 5.0, dtype=DT[gd], device=DEV)
        d = buf[:, shift:shift + dim]
        ends.embed_backward(randn(gen(1), 2, dim), torch.tensor([-1, 100], device=DEV), d)
        assert (d == 0).all() and (buf[:, :shift] == 5).all() and (buf[:, shift + dim:] == 5).all()


# --------------------------------------------------------------- dropout ----

@pytest.mark.parametrize("rows,cols,pitch", [(1, 1, 1), (3, 7, 7), (2, 8, 8), (5, 33, 40), (4, 100, 101), (64, 256, 256),
                                             (17, 130, 132), (1, 3000, 3000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999])
def test_dropout(rows, cols, pitch, dtype, p):
    g, seed, site = gen(rows + cols), 0xFEDCBA9876543210, 0xFFFFFFFE
    x, r = (randn(g, rows, pitch, dtype=DT[dtype])[:, :cols] for _ in range(2))
    mask, share = ref.kept_mask(rows, cols, p, seed, site)
    want = ref.dropout(np64(x), np64(r), mask, share)
    kept = ref.dropout(np64(x), None, mask, share)
    y = ends.dropout_add(x, r, p, seed, site=site)
    within(y, want, 3 * U * np.abs(kept) + (RND[dtype] + U) * np.abs(want) + TINY, "y")
    dx = ends.dropout_backward(x, p, seed - 2 ** 64, site=site)   # 64 bits of the seed count
    within(dx, kept, (RND[dtype] + 3 * U) * np.abs(kept) + TINY, "dx")
    assert torch.equal(dx != 0, torch.from_numpy(mask).to(DEV) & (x != 0))
    # the seed on the device, in the place of an input, from a tensor of other strides
    source = torch.tensor([seed - 2 ** 64], device=DEV)
    for out in (x.clone(), r.clone()):
        a, b = (out, r) if torch.equal(out, x) else (x, out)
        assert torch.equal(ends.dropout_add(a, b, p, source, site=site, out=out), y)


def test_dropout_masks_do_not_depend_on_types_or_strides():
    """A row's draws are its own: the mask is that of any other tensor of the shape."""
    x = torch.ones(300, 777, device=DEV)
    want = ends.dropout_add(x, None, 0.3, 7, site=2) != 0
    assert abs(want.float().mean().item() - 0.7) < 6 * (0.21 / want.numel()) ** 0.5
    for y in (torch.ones(300, 800, device=DEV)[:, 9:786], x.bfloat16(), x.view(3, 100, 777)):
        assert torch.equal((ends.dropout_add(y, None, 0.3, 7, site=2) != 0).view(300, 777), want)
    assert torch.equal(ends.dropout_add(x[:100, :40], None, 0.3, 7, site=2) != 0, want[:100, :40])


@pytest.mark.parametrize("rows,cols", [(9, 255), (9, 257), (5, 1001), (5, 1002), (3, 4100), (1000, 12), (2, 70001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout_of_odd_rows(rows, cols, dtype):
    """Rows that a warp's span, a draw or an access does not divide."""
    g = gen(rows + cols)
    x, r = (randn(g, rows, cols, dtype=DT[dtype]) for _ in range(2))
    mask, share = ref.kept_mask(rows, cols, 0.3, 99, 4)
    kept, want = ref.dropout(np64(x), None, mask, share), ref.dropout(np64(x), np64(r), mask, share)
    within(ends.dropout_add(x, r, 0.3, 99, site=4), want, 3 * U * np.abs(kept) + (RND[dtype] + U) * np.abs(want) + TINY,
           "y")
    within(ends.dropout_backward(x, 0.3, 99, site=4, out=x), kept, (RND[dtype] + 3 * U) * np.abs(kept) + TINY, "dx")


def test_dropped_elements_do_not_read_as_numbers():
    x = torch.full((64, 64), math.nan, device=DEV)
    r = torch.ones(64, 64, device=DEV)
    mask, _ = ref.kept_mask(64, 64, 0.4, 5, 0)
    y = ends.dropout_add(x, r, 0.4, 5)
    assert torch.equal(y.isnan().cpu(), torch.from_numpy(mask)) and (y[~y.isnan()] == 1).all()


def test_dropout_gradient_by_differences():
    """Linear in x, so differences of a step of one are the gradient up to rounding."""
    g = gen(8)
    x, dy = (torch.randn(5, 40, generator=g, device=DEV) for _ in range(2))
    f = lambda v: (ends.dropout_add(v, x, 0.2, 3, site=1).double() * dy.double()).sum().item()
    v = torch.randn(5, 40, generator=g, device=DEV)
    want = (ends.dropout_backward(dy, 0.2, 3, site=1).double() * v.double()).sum().item()
    assert abs(f(x + v) - f(x) - want) <= 40 * 200 * U * 4


def test_captured_dropout_draws_anew():
    seed = torch.tensor([11], device=DEV)
    x = torch.ones(100, 64, device=DEV)
    ends.dropout_add(x, None, 0.5, seed)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ends.dropout_add(x, None, 0.5, seed)
    for s in (12, 13):
        seed.fill_(s)
        graph.replay()
        assert torch.equal(y, ends.dropout_add(x, None, 0.5, s))


@pytest.mark.parametrize("kw", [dict(p=1.0), dict(p=-1.0), dict(p=math.nan)])
def test_dropout_refusals(kw):
    x = torch.ones(4, 8, device=DEV)
    with pytest.raises(dpo.DpoError):
        ends.dropout_add(x, None, kw["p"], 1)
    for bad in (1.5, "1", torch.tensor([1.0], device=DEV), torch.tensor([1, 2], device=DEV)):
        with pytest.raises(TypeError):
            ends.dropout_add(x, None, 0.1, bad)
    for site in (-1, 2 ** 32):
        with pytest.raises(ValueError):
            ends.dropout_add(x, None, 0.1, 1, site=site)


# ------------------------------------------------------ log probabilities ----

def scaled(logits, scale):
    """z as the kernels form it, and in 64 bits but for what is infinite in fp32."""
    with np.errstate(over="ignore"):
        z = np64(logits).astype(f32) * f32(scale)
    return z, np.where(np.isinf(z), z, np64(logits) * float(f32(scale)))


def bars_of(z, ids, vocab, zerr=0.0):
    """Bars of logp, the entropy, and of the log probabilities of all ids (elementwise)."""
    logs, p, h = ref.distribution(z)
    with np.errstate(invalid="ignore"):
        m = z.max(1, keepdims=True)
        # of all numbers, those whose p is 0 in 64 bits too: z - m is rounded, u of its size,
        # before log S is taken from it, u of the result (-4e16 of logits of 1e38 and a scale of
        # 1e-20: 5e9)
        d = np.where(np.isfinite(z), z - m, 0.0)
        az = np.where(np.isfinite(z), np.abs(z), 0.0)
    dz = U * (az + np.abs(m) + np.abs(d)) + zerr
    eps = dz + 1.5 * U * np.abs(d) + 2.0 ** -22
    n = max(64, vocab // 512 + 32)
    tot = (p * eps).sum(1) + (n + 64) * U + 16 * 2.0 ** -22
    logsum = np.abs(h) + (p * np.abs(d)).sum(1)
    each = dz + tot[:, None] + 3 * U * (logsum[:, None] + np.where(np.isfinite(logs), np.abs(logs), 0.0))
    ent = tot + (p * np.abs(d) * (eps + tot[:, None])).sum(1) + (p * dz).sum(1) + 4 * U * (logsum + np.abs(h))
    r = np.arange(len(ids))
    real = (ids >= 0) & (ids < vocab)
    return np.where(real, each[r, np.where(real, ids, 0)], 0.0), ent, each


def logits_case(rows, vocab, dtype, seed=0, spread=3.0, pitch=0, masked=True):
    g = gen(seed + rows * 31 + vocab)
    z = torch.randn(rows, vocab + pitch, generator=g, device=DEV) * spread
    if masked and vocab > 4:
        z[:, vocab - vocab // 5:vocab] = -math.inf
    ids = ids_of(g, (rows,), vocab)
    return g, z.to(DT[dtype])[:, :vocab], ids


LOGITS = [(1, 1), (1, 2), (3, 7), (5, 33), (2, 513), (17, 1000), (1, 5003), (4, 32000), (1, 128256), (200, 2050),
          (700, 129), (3, 50257)]


def check_logprobs(x, ids, scale, top):
    vocab = x.shape[1]
    z32, z = scaled(x, scale)
    o = ends.token_logprobs(x, ids, scale=scale, top=top)
    i = ids.cpu().numpy()
    logp, h = ref.logprobs(z, i)
    bl, bh, each = bars_of(z, i, vocab)
    finite = np.isfinite(logp)
    got = np64(o.logp)
    assert np.array_equal(got[~finite], logp[~finite], equal_nan=True)   # a masked id, no distribution
    within(got[finite], logp[finite], bl[finite], "logp")
    assert (got[(i < 0) | (i >= vocab)] == 0).all()
    got, some = np64(o.entropy), ~np.isnan(h)
    assert np.isnan(got[~some]).all()
    within(got[some], h[some], bh[some], "entropy")
    if top:
        want = ref.top(z32, top)
        assert np.array_equal(o.top_ids.cpu().numpy(), want)
        logs = ref.distribution(z)[0]
        wl = np.take_along_axis(logs, want, 1)
        gl, f = np64(o.top_logp), np.isfinite(wl)
        assert np.array_equal(gl[~f], wl[~f], equal_nan=True)
        within(gl[f], wl[f], np.take_along_axis(each, want, 1)[f], "top logp")
    else:
        assert o.top_logp is None and o.top_ids is None
    return o, z, i, (bl, bh, each)


@pytest.mark.parametrize("rows,vocab", LOGITS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale,top", [(1.0, 0), (0.7, 1), (1.3, 5), (1.0, 32)])
def test_token_logprobs(rows, vocab, dtype, scale, top):
    _, x, ids = logits_case(rows, vocab, dtype)
    check_logprobs(x, ids, scale, min(top, vocab))


@pytest.mark.parametrize("rows,vocab", LOGITS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale,entropy", [(1.0, False), (0.7, True)])
def test_token_logprobs_backward(rows, vocab, dtype, scale, entropy):
    g, x, ids = logits_case(rows, vocab, dtype)
    o, z, i, (bl, bh, each) = check_logprobs(x, ids, scale, 0)
    a = torch.randn(rows, generator=g, device=DEV)
    b = torch.randn(rows, generator=g, device=DEV) if entropy else None
    if rows > 2:
        a[1] = 0
        if entropy:
            b[1] = 0
    d = ends.token_logprobs_backward(a, x, ids, o, dentropy=b)
    assert d.dtype is x.dtype
    s = float(f32(scale))
    want = s * ref.logits_gradient(z, i, np64(a), None if b is None else np64(b))
    logs, p, h = ref.distribution(z)
    lp = np.where(p > 0, logs, 0.0)
    pe = p * (each + 1.5 * U * np.abs(lp) + (2.0 ** -20 if dtype == "bf16" else 2.0 ** -22))
    av = np.where((i >= 0) & (i < vocab), np.abs(np64(a)), 0.0)[:, None]
    bv = (np.abs(np64(b)) if entropy else np.zeros(rows))[:, None]
    one = np.zeros_like(p)
    real = (i >= 0) & (i < vocab)
    one[np.arange(rows)[real], i[real]] = 1
    hb = (each + bh[:, None] + 2 * U * (np.abs(lp) + np.abs(h[:, None])))
    bar = s * (av * (pe + 4 * U * (p + one)) + bv * (pe * np.abs(lp + h[:, None]) + p * hb +
                                                      4 * U * p * np.abs(lp + h[:, None])))
    within(d, want, bar + (RND[dtype] + 2 * U) * np.abs(want) + TINY, "dlogits")
    if rows > 2:
        assert (d[1] == 0).all()
    masked = torch.isinf(x)
    masked[torch.arange(rows, device=DEV)[ids.clamp(0, vocab - 1) == ids], ids[ids.clamp(0, vocab - 1) == ids]] = False
    assert (d[masked] == 0).all()
    y = x.clone()
    assert ends.token_logprobs_backward(a, y, ids, o, dentropy=b, dlogits=y) is y and torch.equal(y, d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pitch,shift", [(0, 1), (1, 0), (3, 2), (8, 8), (5, 3)])
def test_logits_pitches_and_addresses(dtype, pitch, shift):
    """Rows that begin anywhere give what the same rows give alone, but for the order of sums."""
    g, x, ids = logits_case(9, 1003, dtype, pitch=pitch)
    x[:, :] = x
    full = torch.zeros(9, 1003 + pitch + shift, dtype=DT[dtype], device=DEV)
    v = full[:, shift:shift + 1003]
    v.copy_(x)
    full[:, shift + 1003:] = math.nan     # nothing beside the rows is read
    full[:, :shift] = math.nan
    o, *_ = check_logprobs(v, ids, 1.0, 5)
    a = torch.randn(9, generator=g, device=DEV)
    want = ends.token_logprobs_backward(a, v, ids, o)
    buf = torch.full((9, 1003 + 7), 5.0, dtype=DT[dtype], device=DEV)
    for out in (buf[:, 3:1006], buf[:, 2:1005]):
        assert torch.equal(ends.token_logprobs_backward(a, v, ids, o, dlogits=out), want)
    assert (buf[:, :2] == 5).all() and (buf[:, 1006:] == 5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 40, 3000])
def test_rows_of_odd_values(dtype, vocab):
    """Rows that a mask empties, of the type's lowest value, with infinities and NaN, of equal
    values."""
    x = randn(gen(2), 8, vocab, dtype=torch.float32)
    low = torch.finfo(DT[dtype]).min
    x[0] = -math.inf
    x[1] = low
    x[2, vocab // 2] = math.nan
    x[3, 1] = math.inf
    x[4] = 2.5
    x[5] = -math.inf
    x[5, vocab - 1] = 3.0
    x[6] = low
    x[6, 3] = 1.0
    x[7, 2:] = math.nan
    x = x.to(DT[dtype])
    ids = torch.tensor([1, 2, 0, 0, 3, vocab - 1, 3, -1], device=DEV)
    o = ends.token_logprobs(x, ids, top=4)
    logp, h, tl = (np64(v) for v in (o.logp, o.entropy, o.top_logp))
    assert np.isnan(logp[[0, 2, 3]]).all() and np.isnan(h[[0, 2, 3, 7]]).all() and np.isnan(tl[[0, 2, 3, 7]]).all()
    n = math.log(vocab)
    assert np.allclose(logp[[1, 4]], -n, atol=1e-5) and np.allclose(h[[1, 4]], n, atol=1e-5)
    assert (logp[[5, 6, 7]] == 0).all() and (h[[5, 6]] == 0).all()
    t = o.top_ids.cpu().numpy()
    z32, _ = scaled(x, 1.0)
    assert np.array_equal(t, ref.top(z32, 4))
    assert t[0].tolist() == [0, 1, 2, 3] and t[4].tolist() == [0, 1, 2, 3] and t[7, :2].tolist() in ([0, 1], [1, 0])
    d = ends.token_logprobs_backward(torch.zeros(8, device=DEV), x, ids, o)
    assert (d == 0).all()      # no gradient: zeros whatever the row
    a = torch.tensor([0, 1, 0, 0, 1, 1, 1, 9], dtype=torch.float32, device=DEV)
    d = ends.token_logprobs_backward(a, x, ids, o, dentropy=torch.tensor([0, 1, 0, 0, 1, 1, 1, 0.0], device=DEV))
    assert torch.isfinite(d).all() and (d[[0, 2, 3, 5, 6, 7]] == 0).all()
    want = np.where(np.arange(vocab) == 2, 1.0, 0.0) - 1 / vocab
    assert np.allclose(np64(d[1]), want, atol=2.0 ** -8 + 1e-5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(6, 5), (6, 40), (6, 3000), (6, 100003), (4000, 300)])
@pytest.mark.parametrize("top", [1, 5, 32])
def test_nan_comes_after_masked_logits(dtype, rows, vocab, top):
    """Alternatives: numbers, then -infinity, then NaN, each of equal ones by their ids."""
    top = min(top, vocab)
    x = torch.full((rows, vocab), -math.inf, device=DEV)
    x[0, 0] = math.nan
    x[1, ::2] = math.nan
    x[2, :] = math.nan
    x[2, vocab - 1] = -math.inf
    x[3, 1:] = math.nan
    x[3, 0] = -3.0
    x[4:, vocab // 2] = 7.0
    x[4:, vocab // 2 + 1] = torch.finfo(DT[dtype]).min
    x[4:, :2] = math.nan
    x = x.to(DT[dtype])
    o = ends.token_logprobs(x, top=top)
    z = np64(x[:6])
    want = [sorted(range(vocab), key=lambda j: (math.isnan(r[j]), 0.0 if math.isnan(r[j]) else -r[j], j))[:top] for r in z]
    assert o.top_ids[:6].tolist() == want
    assert (o.top_ids[4:] == o.top_ids[4]).all()
    assert np.array_equal(ref.top(z, top), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(4000, 2050), (3999, 40), (2, 128256), (9, 40000)])
def test_rows_by_warps_and_by_clusters(dtype, rows, vocab):
    """So many rows that a warp has one of many batches, so few that CTAs share one."""
    g, x, ids = logits_case(rows, vocab, dtype, seed=7)
    check_logprobs(x, ids, 0.9, 0)
    check_logprobs(x[:40], ids[:40], 0.9, 6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [33, 64, 100, 199, 300, 1000, 1500, 4000])
@pytest.mark.parametrize("rows", [1, 7, 400])
def test_many_alternatives_of_few(dtype, vocab, rows):
    """More of a row reaches the threads' bound than a warp sorts at once."""
    g, x, ids = logits_case(rows, vocab, dtype, seed=11)
    for top in (20, 31, 32):
        check_logprobs(x, ids, 1.0, top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1, 32])
def test_shared_rows_of_odd_values(dtype, top):
    """Rows shared by CTAs: masked but for one value, all masked, of equal values, with NaN."""
    vocab = 100003
    x = torch.full((5, vocab), -math.inf, device=DEV)
    x[0, 77777] = 1.0
    x[2] = 0.5
    x[3] = randn(gen(1), vocab, dtype=torch.float32)
    x[3, 50000:] = math.nan
    x[4, ::1000] = torch.arange(0, vocab, 1000, device=DEV).float().neg()
    x = x.to(DT[dtype])
    o = ends.token_logprobs(x, torch.tensor([77777, 0, 5, 1, 0], device=DEV), top=top)
    assert np.array_equal(o.top_ids.cpu().numpy(), ref.top(scaled(x, 1.0)[0], top))
    logp, h = np64(o.logp), np64(o.entropy)
    assert logp[0] == 0 and h[0] == 0 and np.isnan(logp[[1, 3]]).all() and np.isnan(h[[1, 3]]).all()
    assert abs(logp[2] + math.log(vocab)) < 1e-5 and abs(h[2] - math.log(vocab)) < 1e-5
    assert logp[4] == 0 and np64(o.top_logp)[0, 0] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1.0, 300.0])
def test_logits_that_pass_the_near_range(dtype, scale):
    """Rows whose largest value so far grows, or shrinks, past 16384 units of log 2, where sums and
    gradients go another way, and rows altogether beyond."""
    n = torch.arange(3001, device=DEV).float()
    rows = [n * 13.0, 39000 - n * 13.0, n * 0.001 + 11300, n * 0.05 + 11300, n * -0.01 - 12000, n * 0.01 + 40000,
            (n % 7) * 3000]
    x = (torch.stack(rows) / scale).to(DT[dtype])
    ids = torch.tensor([3000, 0, 3000, 2999, 0, 3000, 6], device=DEV)
    o, z, i, (bl, bh, each) = check_logprobs(x, ids, scale, 3)
    a = torch.ones(7, device=DEV)
    d = ends.token_logprobs_backward(a, x, ids, o)
    logs, p, _ = ref.distribution(z)
    want = float(f32(scale)) * ref.logits_gradient(z, i, np64(a), None)
    one = np.zeros_like(p)
    one[np.arange(7), i] = 1
    # one multiply-add takes m + log S, times log2(e), from the logit times a rounded factor: u of each
    m = np.abs(z).max(1, keepdims=True)
    pe = p * (each + 1.5 * U * np.abs(np.where(p > 0, logs, 0.0)) + 2 * U * (np.abs(z) + m) + 2.0 ** -20)
    within(d, want, scale * (pe + 4 * U * (p + one)) + (RND[dtype] + 2 * U) * np.abs(want) + TINY, "dlogits")


def rounds_to(got, want, bar, dtype, what):
    """Each element is what some number within bar of want rounds to (fp32's half step on the way to
    bf16 is in the bar)."""
    low, high = (torch.from_numpy(want + s * (bar + U * np.abs(want))).to(dtype).double().numpy() for s in (-1, 1))
    got = np64(got)
    off = (got < low) | (got > high)
    assert not off.any(), f"{what}: {off.sum()} of {off.size}, {got[off][:3]} for {want[off][:3]}"


@pytest.mark.parametrize("scale", [1.0, 0.7, 1.9])
@pytest.mark.parametrize("offset", [30.0, -1000.0, 5e3, 11000.0, 3e5])
@pytest.mark.parametrize("entropy", [False, True])
def test_gradients_of_rows_far_from_zero(scale, offset, entropy):
    """What a row's logits have in common leaves no error in its probabilities: bf16 gradients are the
    roundings of numbers within 2^-17 of p's terms, which takes the sum's 64 u and the two
    exponentials' 2^-22, and 2^-22 of log p for the multiply-add that forms it."""
    rows, vocab = 800, 40
    g = gen(int(abs(offset)) + entropy)
    top = torch.tensor(offset / scale, device=DEV).bfloat16()
    below = torch.nextafter(top, torch.tensor(-math.inf, device=DEV, dtype=torch.bfloat16))
    x = torch.where(torch.rand(rows, vocab, generator=g, device=DEV) < 0.3, below, top)
    x[:, 0] = top
    ids = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    a = torch.randn(rows, generator=g, device=DEV)
    b = torch.randn(rows, generator=g, device=DEV) if entropy else None
    o = ends.token_logprobs(x, ids, scale=scale)
    d = ends.token_logprobs_backward(a, x, ids, o, dentropy=b)
    s = float(f32(scale))
    z, i = np64(x) * s, ids.cpu().numpy()
    want = s * ref.logits_gradient(z, i, np64(a), None if b is None else np64(b))
    logs, p, h = ref.distribution(z)
    av, bv = np.abs(np64(a))[:, None], np.abs(np64(b))[:, None] if entropy else 0.0
    own = np.zeros_like(p)
    own[np.arange(rows), i] = 1
    bar = s * (p * (av + bv * (np.abs(logs + h[:, None]) + 1)) * (2.0 ** -17 + 2.0 ** -22 * np.abs(logs)) + own * av * 8 * U)
    rounds_to(d, want, bar + TINY, torch.bfloat16, "dlogits")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale,size", [(1e-20, 1e38), (1e-20, 1e20), (1e6, 1e-6), (1e6, 1e30), (1.0, 1e37)])
@pytest.mark.parametrize("top", [0, 7])
def test_extreme_scales(dtype, scale, size, top):
    """Logits of any size: their exponentials are 0 or 1 where they are far apart."""
    x = randn(gen(9), 6, 2003, scale=1.0, dtype=torch.float32)
    x[2] = -x[2].abs()
    x[3, 5:] = -math.inf
    x = (x * size).to(DT[dtype])
    x[4] = torch.finfo(DT[dtype]).min
    x[4, ::3] = -math.inf
    x[5, 1:] = torch.finfo(DT[dtype]).min
    check_logprobs(x, torch.tensor([0, 5, 2002, 1, 4, 0], device=DEV), scale, top)


def test_ties_go_to_the_lowest_id():
    """Equal values by the thousand, and values that only the scale makes equal."""
    x = (torch.randn(6, 50000, generator=gen(3), device=DEV) * 2).round()
    for y in (x, x.bfloat16(), x.int().float()):
        o = ends.token_logprobs(y, top=32)
        assert o.logp is None
        assert np.array_equal(o.top_ids.cpu().numpy(), ref.top(np64(y), 32))
    y = 1 + torch.arange(3000, device=DEV).flip(0)[None] * 2.0 ** -23
    o = ends.token_logprobs(y, scale=1 / 3, top=20)
    assert np.array_equal(o.top_ids.cpu().numpy(), ref.top(scaled(y, 1 / 3)[0], 20))
    up = torch.arange(20000, device=DEV)[None].float()   # every value a new largest one
    assert ends.token_logprobs(up, top=3).top_ids.tolist() == [[19999, 19998, 19997]]


def test_shapes_of_rows():
    g, x, ids = logits_case(24, 100, "f32")
    want = ends.token_logprobs(x, ids, top=3)
    o = ends.token_logprobs(x.view(4, 6, 100), ids.view(4, 6), top=3)
    assert o.logp.shape == o.entropy.shape == (4, 6) and o.top_ids.shape == (4, 6, 3) and o.stats.shape == (4, 6, 2)
    assert torch.equal(o.logp.view(24), want.logp) and torch.equal(o.top_ids.view(24, 3), want.top_ids)
    one = ends.token_logprobs(x[3], ids[3], top=3)
    assert one.logp.shape == () and one.top_ids.shape == (3,) and torch.equal(one.entropy, want.entropy[3])
    a = torch.randn(24, generator=g, device=DEV)
    d = ends.token_logprobs_backward(a, x, ids, want)
    assert torch.equal(ends.token_logprobs_backward(a.view(4, 6), x.view(4, 6, 100), ids.view(4, 6), o).view(24, 100), d)
    assert torch.equal(ends.token_logprobs_backward(a[3], x[3], ids[3], one), d[3])
    assert ends.token_logprobs(x[:0], ids[:0]).logp.shape == (0,)
    for bad in (ids[:-1], ids.view(4, 6), ids.float()):
        with pytest.raises((ValueError, TypeError)):
            ends.token_logprobs(x, bad)
    for top in (-1, 33):
        with pytest.raises(ValueError):
            ends.token_logprobs(x, top=top)
    with pytest.raises(dpo.DpoError):
        ends.token_logprobs(x[:, :3], top=4)
    with pytest.raises(TypeError):
        ends.token_logprobs(x.half())


def test_logprobs_gradient_by_differences():
    """Along a random direction with a step of 2^-6: the third derivative's 2^-12 / 6 of about
    one, and rounding 40 u of values near 10 over the step, together under 1e-3."""
    g, x, ids = logits_case(6, 300, "f32", masked=False)
    a, b = (torch.randn(6, generator=g, device=DEV) for _ in range(2))
    v = torch.randn(6, 300, generator=g, device=DEV)
    step = 2.0 ** -6

    def f(y):
        o = ends.token_logprobs(y, ids, scale=0.9)
        return ((a * o.logp).double().sum() + (b * o.entropy).double().sum()).item()

    d = ends.token_logprobs_backward(a, x, ids, ends.token_logprobs(x, ids, scale=0.9), dentropy=b)
    want = (d.double() * v.double()).sum().item()
    assert abs((f(x + step * v) - f(x - step * v)) / (2 * step) - want) <= 2e-3 * max(1.0, abs(want))


# ------------------------------------------------------------------ head ----

HEAD = [(1, 64, 100), (1, 8, 1), (3, 72, 33), (9, 264, 1003), (33, 520, 300), (130, 768, 2051), (257, 64, 5003), (8, 2048, 700),
        (700, 136, 129), (300, 1096, 4100), (64, 2400, 257),
        (20, 1104, 50001), (600, 1104, 30001),   # several tiles, each in parts of K, to a CTA and to a pair
        (520, 72, 20001), (64, 136, 30001), (1100, 264, 9001)]   # dx's K shared out


def head_case(t, d, v, seed=0, pitch=0, spread=2.0):
    g = gen(seed + t + 3 * d + 7 * v)
    x = randn(g, t, d + pitch)[:, :d]
    w = randn(g, v, d, scale=spread * d ** -0.5)
    return g, x, w, ids_of(g, (t,), v)


def check_head(x, w, ids, scale, top, keep):
    t, d = x.shape
    v = w.shape[0]
    s = float(f32(scale))
    z = s * (np64(x) @ np64(w).T)
    zerr = (d / 4 + 16) * U * s * (np.abs(np64(x)) @ np.abs(np64(w)).T)
    o, kept = ends.head_logprobs(x, w, ids, scale=scale, top=top, keep=keep)
    i = ids.cpu().numpy()
    logp, h = ref.logprobs(z, i)
    bl, bh, each = bars_of(z, i, v, zerr)
    within(o.logp, logp, bl, "logp")
    within(o.entropy, h, bh, "entropy")
    if top:
        got = o.top_ids.cpu().numpy()
        assert all(len(set(r)) == top for r in got)
        best = np.take_along_axis(z, ref.top(z, top), 1)
        there, ze = np.take_along_axis(z, got, 1), np.take_along_axis(zerr, got, 1) + zerr.max(1, keepdims=True)
        assert np.all(np.abs(there - best) <= ze)    # nearly equal logits may change places
        logs = ref.distribution(z)[0]
        within(o.top_logp, np.take_along_axis(logs, got, 1), np.take_along_axis(each, got, 1), "top logp")
    assert (kept is None) == (not keep)
    return o, kept, z, i, each, bh


def check_head_backward(x, w, ids, scale, a, b, o, kept, z, i, each, bh, got, gd, old=None):
    (t, d), v = x.shape, w.shape[0]
    s = float(f32(scale))
    G = s * ref.logits_gradient(z, i, np64(a), None if b is None else np64(b))
    logs, p, h = ref.distribution(z)
    real = (i >= 0) & (i < v)
    av = np.where(real, np.abs(np64(a)), 0.0)[:, None]
    bv = (np.abs(np64(b)) if b is not None else np.zeros(t))[:, None]
    pe = p * (each + 2.0 ** -11 + 2.0 ** -18)
    # what is kept of a small p may be 2^-24 of its tile's largest, which is at most 1
    pe = pe + 2.0 ** -24 * 2.0 ** -10
    lh = np.abs(logs + h[:, None])
    ge = s * (av * pe + bv * (pe * (lh + 1) + p * (each + bh[:, None] + 2.0 ** -11))) + (B + 8 * U) * np.abs(G)
    one = np.zeros_like(p)
    one[np.arange(t)[real], i[real]] = 1
    ge = ge + s * av * one * (np.take_along_axis(each, np.where(real, i, 0)[:, None], 1) + 8 * U)
    aG, aW, aX = np.abs(G), np.abs(np64(w)), np.abs(np64(x))
    dx, dw = got
    if dx is not None:
        want = G @ np64(w)
        within(dx, want, (ge + (v / 4 + 16) * U * aG) @ aW + B * np.abs(want) + TINY, "dx")
    want = G.T @ np64(x)
    bar = (ge + (t / 4 + 16) * U * aG).T @ aX
    if old is not None:
        bar, want = bar + 2 * U * (np.abs(want) + np.abs(old)), want + old
    within(dw, want, bar + (RND[gd] + 2 * U) * np.abs(want) + TINY, "dw")


@pytest.mark.parametrize("t,d,v", HEAD)
@pytest.mark.parametrize("scale,top", [(1.0, 0), (0.6, 5)])
@pytest.mark.parametrize("keep", [False, True])
def test_head(t, d, v, scale, top, keep):
    _, x, w, ids = head_case(t, d, v)
    check_head(x, w, ids, scale, min(top, v), keep)


@pytest.mark.parametrize("t,d,v", HEAD)
@pytest.mark.parametrize("gd", ["f32", "bf16"])
@pytest.mark.parametrize("scale,entropy", [(1.0, False), (0.6, True)])
def test_head_backward(t, d, v, gd, scale, entropy):
    g, x, w, ids = head_case(t, d, v, seed=1, pitch=8)
    o, kept, *rest = check_head(x, w, ids, scale, 0, True)
    a = torch.randn(t, generator=g, device=DEV)
    b = torch.randn(t, generator=g, device=DEV) if entropy else None
    for accumulate in (False, True):
        old = randn(g, v, d, dtype=DT[gd])
        dw = old.clone()
        dx = ends.head_logprobs_backward(a, kept, x, w, ids, o, dw, dentropy=b, accumulate=accumulate)
        check_head_backward(x, w, ids, scale, a, b, o, kept, *rest, (dx, dw), gd, np64(old) if accumulate else None)
    assert ends.status() == 0


def test_head_is_precise():
    """K is added up in parts, so truncation does not grow with it: 64 steps of at most one step
    2^-23 of a partial sum of size about one, 8e-6 where all add up, in each of four parts, of
    log probabilities near 10: 4e-6, and random signs halve it."""
    _, x, w, ids = head_case(64, 4096, 8000, seed=2)
    ids = ids.clamp(0, 7999)
    o, _ = ends.head_logprobs(x, w, ids)
    z = np64(x) @ np64(w).T
    logp, h = ref.logprobs(z, ids.cpu().numpy())
    assert np.linalg.norm(np64(o.logp) - logp) <= 2e-6 * np.linalg.norm(logp)
    assert np.linalg.norm(np64(o.entropy) - h) <= 2e-6 * np.linalg.norm(h)


@pytest.mark.parametrize("t,d,v", [(40, 136, 1003), (3, 64, 300)])
def test_head_confident_and_padded_rows(t, d, v):
    """Rows almost sure of their token (1 - p tiny) and padded ones: the gradient of the first is
    small and right, that of the second nothing."""
    g, x, w, ids = head_case(t, d, v, seed=3, spread=0.3)
    ids = ids.clamp(0, v - 1)
    w[ids] = x * (12.0 / x.float().square().sum(1, keepdim=True)).bfloat16()
    ids[1] = -1
    o, kept, *rest = check_head(x, w, ids, 1.0, 0, True)
    a = torch.randn(t, generator=g, device=DEV)
    dw = torch.empty_like(w)
    dx = ends.head_logprobs_backward(a, kept, x, w, ids, o, dw)
    check_head_backward(x, w, ids, 1.0, a, None, o, kept, *rest, (dx, dw), "bf16")
    assert (dx[1] == 0).all() and o.logp[1] == 0


@pytest.mark.parametrize("t,d,v", [(9, 264, 1003), (130, 768, 2051), (600, 1104, 30001)])
@pytest.mark.parametrize("gd", ["f32", "bf16"])
def test_head_backward_after_alternatives(t, d, v, gd):
    """The statistics that the backward takes come from the written logits there."""
    g, x, w, ids = head_case(t, d, v, seed=4)
    o, kept, *rest = check_head(x, w, ids, 0.8, 7, True)
    a, b = (torch.randn(t, generator=g, device=DEV) for _ in range(2))
    dw = torch.empty(v, d, dtype=DT[gd], device=DEV)
    dx = ends.head_logprobs_backward(a, kept, x, w, ids, o, dw, dentropy=b)
    check_head_backward(x, w, ids, 0.8, a, b, o, kept, *rest, (dx, dw), gd)
    assert ends.status() == 0


def test_head_of_large_and_infinite_logits():
    """Logits past 16384 units of log 2 go another way; infinite ones leave their rows no
    distribution and the other rows theirs."""
    g, x, w, ids = head_case(40, 64, 1003, seed=8)
    check_head(x, w, ids, 2e4, 0, True)
    check_head(x, w, ids, 2e4, 4, True)
    want, _ = ends.head_logprobs(x, w, ids)
    x = x.clone()
    x[3] = 3e38
    x[7, 5] = math.nan
    o, kept = ends.head_logprobs(x, w, ids, keep=True)
    rest = torch.ones(40, dtype=torch.bool, device=DEV)
    rest[[3, 7]] = False
    assert o.entropy[~rest].isnan().all()
    assert torch.equal(o.logp[rest], want.logp[rest]) and torch.equal(o.entropy[rest], want.entropy[rest])
    a = torch.ones(40, device=DEV)
    a[[3, 7]] = 0      # a masked loss: their gradient is nothing, and so is their part of dw's G
    x[3], x[7] = 0, 0  # (dw itself multiplies G with x)
    dw = torch.empty_like(w)
    dx = ends.head_logprobs_backward(a, kept, x, w, ids, o, dw)
    assert (dx[~rest] == 0).all() and torch.isfinite(dx).all() and torch.isfinite(dw).all()


def test_head_gradients_of_rows_far_from_zero():
    """Rows that differ by a constant of their logits, which fp32 holds exactly, have one gradient but
    for the roundings of e^(z - m) before it is kept: 2^-22 and 2^-24 of a log2 below 16, under 2^-19,
    which moves the mean of the kept values' and G's roundings by as much."""
    tokens, vocab, dim = 32, 5000, 64
    g = gen(17)
    x, w = (torch.zeros(n, dim, device=DEV) for n in (tokens, vocab))
    x[1:, 0] = torch.randint(64, 88, (tokens - 1,), generator=g, device=DEV).float() / -64   # 128 of them: -11000 to -8192
    x[1::2, 0] *= -1
    w[:, 0] = 8192
    x[:, 1] = 1
    w[:, 1] = torch.randint(-128, 128, (vocab,), generator=g, device=DEV).float() / 32
    x[:, 2] = 2.0 ** -8
    w[:, 2] = torch.randint(0, 8, (vocab,), generator=g, device=DEV).float()
    x[:, 8:8 + tokens] = torch.eye(tokens, device=DEV)   # dw's columns: G of each token
    x, w = x.bfloat16(), w.bfloat16()
    ids = torch.zeros(tokens, dtype=torch.long, device=DEV)
    o, kept = ends.head_logprobs(x, w, ids, keep=True)
    dw = torch.empty(vocab, dim, device=DEV)
    ends.head_logprobs_backward(torch.full((tokens,), 1.3, device=DEV), kept, x, w, ids, o, dw)
    G = np64(dw)[1:, 8:8 + tokens].T
    z = np64(x) @ np64(w).T
    want = ref.logits_gradient(z, ids.cpu().numpy(), np.full(tokens, float(f32(1.3))))[:, 1:]
    assert np.abs(G / want - 1).max() <= B + 2.0 ** -11 + 2.0 ** -18
    mean = np.abs((G / G[0] - 1).mean(1))
    assert mean.max() <= 2.0 ** -17, mean


def test_head_of_no_tokens_and_shapes():
    g, x, w, ids = head_case(24, 64, 100)
    want, kept = ends.head_logprobs(x, w, ids, top=3, keep=True)
    o, k2 = ends.head_logprobs(x.view(4, 6, 64), w, ids.view(4, 6), top=3, keep=True)
    assert torch.equal(o.logp.view(24), want.logp) and torch.equal(o.top_ids.view(24, 3), want.top_ids)
    a = torch.randn(24, generator=g, device=DEV)
    dw, dw2 = torch.empty_like(w), torch.empty_like(w)
    dx = ends.head_logprobs_backward(a, kept, x, w, ids, want, dw)
    dx2 = ends.head_logprobs_backward(a.view(4, 6), k2, x.view(4, 6, 64), w, ids.view(4, 6), o, dw2)
    assert torch.equal(dx2.view(24, 64), dx) and torch.equal(dw, dw2)
    again = ends.head_logprobs_backward(a, kept, x, w, ids, want, dw2)    # kept is still there
    assert torch.equal(again, dx) and torch.equal(dw, dw2)
    none, kept = ends.head_logprobs(x[:0], w, ids[:0], keep=True)
    assert none.logp.shape == (0,)
    assert ends.head_logprobs_backward(a[:0], kept, x[:0], w, ids[:0], none, dw).shape == (0, 64)
    assert (dw == 0).all()
    plain, _ = ends.head_logprobs(x, w, top=2)
    assert plain.logp is None and torch.equal(plain.top_ids, want.top_ids[:, :2])
    with pytest.raises(ValueError):
        ends.head_logprobs_backward(a, None, x, w, ids, want, dw)
    with pytest.raises(TypeError, match="stash_dtype"):
        ends.head_logprobs(x, w.float(), ids)
    with pytest.raises(ValueError):
        ends.head_logprobs(x, w[:, :32], ids)
    with pytest.raises(dpo.DpoError):
        ends.head_logprobs(x[:, :60], w[:, :60].contiguous(), ids)


def test_head_gradient_by_differences():
    """fp32 gradients of x and w against differences of the loss along directions that bf16 holds
    exactly (zeros and a power of two, one element): G's rounding to bf16, 2^-8, times a few."""
    g, x, w, ids = head_case(12, 64, 90, seed=6)
    x, w = x.float().mul(16).round().div(16).bfloat16(), w.float().mul(64).round().div(64).bfloat16()
    ids = ids.clamp(0, 89)
    a = torch.randn(12, generator=g, device=DEV)
    b = torch.randn(12, generator=g, device=DEV)

    def f(x, w):
        o, _ = ends.head_logprobs(x, w, ids)
        return ((a * o.logp).double().sum() + (b * o.entropy).double().sum()).item()

    o, kept = ends.head_logprobs(x, w, ids, keep=True)
    dw = torch.empty(90, 64, device=DEV)
    dx = ends.head_logprobs_backward(a, kept, x, w, ids, o, dw, dentropy=b)
    scale = dx.float().abs().max().item(), dw.abs().max().item()
    for k in range(6):
        for which, (m, grad) in enumerate(((x, dx), (w, dw))):
            i, j, h = int(ids[k]) if which else k, 7 * k + 3, 2.0 ** -4
            up, down = m.clone(), m.clone()
            up[i, j] += h
            down[i, j] -= h
            if (up[i, j].float() - m[i, j].float()).item() != h or (m[i, j].float() - down[i, j].float()).item() != h:
                continue
            d = (f(up, w) - f(down, w) if not which else f(x, up) - f(x, down)) / (2 * h)
            # the third derivative's h^2 / 6 of |x|^3 or |w|^3, at most 30 here, and 2^-8 of the terms
            assert abs(d - grad[i, j].item()) <= 2e-2 * scale[which] + h * h * 5, (which, k)


@pytest.mark.parametrize("t,d,v", [(1, 64, 100), (130, 768, 2051), (520, 72, 20001)])
@pytest.mark.parametrize("gd", ["f32", "bf16"])
def test_head_gradient_of_the_weights_alone(t, d, v, gd):
    """The C call without dx; int32 ids."""
    g, x, w, ids = head_case(t, d, v, seed=5)
    ids = torch.where((ids < 0) | (ids >= v), -1, ids).int()
    o, kept, *rest = check_head(x, w, ids, 0.9, 0, True)
    a = torch.randn(t, generator=g, device=DEV)
    for accumulate in (0, 1):
        old = randn(g, v, d, dtype=DT[gd])
        dw = old.clone()
        need = ends.dpo_head_workspace(t, d, v, True)[2]
        ws = torch.empty(need, dtype=torch.uint8, device=DEV)
        dpo.dpo_head_backward(ends.dpo_head_backward_args(
            x=x.data_ptr(), w=w.data_ptr(), ids=ends.dpo_ids(ids.data_ptr(), 1, t, t, 4), kept=kept.data_ptr(),
            logp=o.logp.data_ptr(), entropy=o.entropy.data_ptr(), stats=o.stats.data_ptr(), dlogp=a.data_ptr(),
            dw=dw.data_ptr(), tokens=t, dim=d, vocab=v, ld_x=d, scale=0.9, grad_dtype=gd == "bf16",
            accumulate=accumulate, workspace=ws.data_ptr(), workspace_bytes=need),
            torch.cuda.current_stream().cuda_stream)
        check_head_backward(x, w, ids, 0.9, a, None, o, kept, *rest, (None, dw), gd, np64(old) if accumulate else None)
    assert ends.status() == 0


def test_log_probabilities_without_the_entropy():
    """The C call without entropy, and without ids."""
    _, x, ids = logits_case(30, 513, "bf16")
    want = ends.token_logprobs(x, ids, top=3)
    stats, logp = torch.empty(30, 2, device=DEV), torch.full((30,), 9.0, device=DEV)
    tl, ti = torch.empty(30, 3, device=DEV), torch.empty(30, 3, dtype=torch.long, device=DEV)
    for given in (False, True):
        dpo.dpo_logprobs(ends.dpo_logprobs_args(
            logits=x.data_ptr(), ids=ends.dpo_ids(ids.data_ptr() if given else None, 1, 30, 30, 8),
            logp=logp.data_ptr(), stats=stats.data_ptr(), top_logp=tl.data_ptr(), top_ids=ti.data_ptr(), rows=30,
            vocab=513, ld_logits=x.stride(0), scale=1.0, dtype=dpo.DPO_BF16, top=3), torch.cuda.current_stream().cuda_stream)
        assert torch.equal(logp, want.logp if given else torch.full_like(logp, 9.0))
        for a, b in ((stats, want.stats), (tl, want.top_logp), (ti, want.top_ids)):
            assert torch.equal(a.nan_to_num(), b.nan_to_num())


def test_outputs_are_tensors_of_their_own():
    """Each in a storage of its size: one that is kept holds no other's memory, and one that PyTorch
    lets grow does not grow into another."""
    _, x, ids = logits_case(24, 100, "f32")
    _, h, w, _ = head_case(24, 64, 100)
    for o in (ends.token_logprobs(x, ids, top=5), ends.head_logprobs(h, w, ids, top=5)[0]):
        outs = [t for t in o[:5]]
        assert len({t.untyped_storage().data_ptr() for t in outs}) == 5
        for t in outs:
            assert t.is_contiguous() and t.storage_offset() == 0
            assert t.untyped_storage().nbytes() == t.numel() * t.element_size()
        before = [t.clone() for t in outs]
        o.entropy.resize_(1000).fill_(7.0)
        o.stats.resize_(1000).fill_(7.0)
        for t, b in zip((o.logp, o.top_logp, o.top_ids), (before[0], before[3], before[4])):
            assert torch.equal(t, b)


class Allocations(TorchDispatchMode):
    """Counts what is allocated."""

    def __init__(self):
        super().__init__()
        self.count = 0

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        self.count += func.overloadpacket is torch.ops.aten.empty
        return func(*args, **(kwargs or {}))


def test_modes_of_pytorch_see_allocations():
    """Outputs and workspaces are torch.empty's to a mode that watches operators, and are filled where
    deterministic algorithms ask for it: the bytes of `kept` that no token has."""
    _, x, ids = logits_case(24, 100, "f32")
    _, h, w, _ = head_case(3, 64, 300)
    table = randn(gen(1), 100, 16)
    calls = [lambda: ends.embed(ids, table), lambda: ends.dropout_add(x, None, 0.1, 1),
             lambda: ends.token_logprobs(x, ids, top=2), lambda: ends.head_logprobs(h, w, keep=True),
             lambda: ffn.add_rms_norm(table.float(), torch.ones(16, device=DEV)), lambda: ffn.pack8(table)]
    for call in calls:
        want = call()
        with Allocations() as seen:
            got = call()
        assert seen.count > 0
        for a, b in zip(want if isinstance(want, tuple) else (want,), got if isinstance(got, tuple) else (got,)):
            if torch.is_tensor(a) and a.dtype is not torch.uint8:
                assert torch.equal(a, b)
    torch.use_deterministic_algorithms(True)
    try:
        _, kept = ends.head_logprobs(h, w, keep=True)
    finally:
        torch.use_deterministic_algorithms(False)
    assert (kept[-220:] == 255).all()   # the maxima of 3 parts of 3 tokens are 36 bytes of 256


# ------------------------------------------------- more than 2^31 elements ----

def test_embedding_of_a_table_past_32_bits():
    vocab, dim = 2 ** 20 + 7, 2056
    g = gen(40)
    table = torch.zeros(vocab, dim, dtype=torch.bfloat16, device=DEV)
    ids = torch.tensor([vocab - 1, 0, vocab - 5, 2 ** 20, vocab - 1], device=DEV)
    table[ids] = randn(g, 5, dim)
    assert torch.equal(ends.embed(ids, table), table[ids])
    dy = randn(g, 5, dim)
    d = torch.full_like(table, 3.0)
    ends.embed_backward(dy, ids, d)
    sums = dy.float()
    sums[0] += sums[4]
    assert torch.equal(d[ids[:4]], sums[:4].bfloat16())
    d[ids] = 0
    assert not d.any()
    ends.embed_backward(dy, ids, d, accumulate=True)
    assert torch.equal(d[ids[:4]], sums[:4].bfloat16())
    many = ids.repeat(vocab // 5 + 1)[:vocab].flip(0)     # as many tokens, so as large an output
    assert torch.equal(ends.embed(many, table)[-5:], table[many[-5:]])


@pytest.mark.parametrize("cols", [2056, 2055])
def test_dropout_of_rows_past_32_bits(cols):
    rows = 2 ** 20 + 5
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device=DEV)
    y = ends.dropout_add(x, x, 0.25, 5, site=1)
    for r in (0, 2 ** 20 - 3, rows - 1):
        words = [ref.philox((c // 8, r, 0, 1), (5, 0))[c % 8 // 2] >> 16 * (c % 2) & 0xFFFF for c in range(cols)]
        kept = torch.tensor([w >= 16384 for w in words], device=DEV)
        assert torch.equal(y[r], torch.where(kept, 1 + 65536 / 49152, 1.0).bfloat16())


def test_logits_past_32_bits():
    rows, vocab = 70003, 32001
    g = gen(41)
    x = torch.randn(1000, vocab, generator=g, device=DEV).bfloat16().repeat(71, 1)[:rows]
    ids = torch.randint(0, vocab, (1000,), generator=g, device=DEV).repeat(71)[:rows]
    a = torch.randn(1000, generator=g, device=DEV).repeat(71)[:rows]
    for top in (0, 3):
        o = ends.token_logprobs(x, ids, top=top)
        for v in o[:5]:
            assert v is None or torch.equal(v[-1000:], v[rows - 2000:rows - 1000])
        check_logprobs(x[-7:], ids[-7:], 1.0, top)
        want, _ = ref.logprobs(np64(x[-7:]), ids[-7:].cpu().numpy())
        within(o.logp[-7:], want, 1e-5 * np.abs(want), "logp")
    d = ends.token_logprobs_backward(a, x, ids, o)
    assert torch.equal(d[-1000:], d[rows - 2000:rows - 1000])
    g64 = ref.logits_gradient(np64(x[-7:]), ids[-7:].cpu().numpy(), np64(a[-7:]))
    within(d[-7:], g64, (B + 1e-5) * np.abs(g64) + TINY, "dlogits")


def test_head_of_logits_past_32_bits():
    """40003 x 60001 of them, kept and as G; every 1000 tokens are the first ones again."""
    tokens, dim, vocab = 40003, 64, 60001
    _, x, w, ids = head_case(1000, dim, vocab, seed=9)
    x, ids = x.repeat(41, 1)[:tokens], ids.repeat(41)[:tokens]
    a = torch.randn(1000, generator=gen(42), device=DEV)
    o, kept = ends.head_logprobs(x, w, ids, keep=True)
    assert torch.equal(o.logp[39000:40000], o.logp[:1000])
    dw = torch.empty(vocab, dim, device=DEV)
    dx = ends.head_logprobs_backward(a.repeat(41)[:tokens], kept, x, w, ids, o, dw)
    assert torch.equal(dx[39000:40000], dx[:1000]) and torch.equal(dx[40000:], dx[:3])
    one, k1, *rest = check_head(x[:1000], w, ids[:1000], 1.0, 0, True)
    d1 = torch.empty_like(dw)
    dx1 = ends.head_logprobs_backward(a, k1, x[:1000], w, ids[:1000], one, d1)
    check_head_backward(x[:1000], w, ids[:1000], 1.0, a, None, one, k1, *rest, (dx1, d1), "f32")
    assert torch.equal(one.logp, o.logp[:1000])
    check_head_backward(x[:1000], w, ids[:1000], 1.0, a, None, one, k1, *rest, (dx[:1000], d1), "f32")
    # dw: 40 times theirs and the first three tokens' again, whose G is rounded; both sums are off by what
    # the bar of a product of so many terms says, of 41 and of 40 times the magnitudes
    G, X = ref.logits_gradient(rest[0], rest[1], np64(a)), np64(x[:1000])
    mag = (1 + B) * np.abs(G).T @ np.abs(X)
    bar = (41 * (tokens / 4 + 16) + 40 * (1000 / 4 + 16)) * U * mag + 2 * B * np.abs(G[:3]).T @ np.abs(X[:3])
    within(dw, 40 * np64(d1) + G[:3].T @ X[:3], bar, "dw")
    assert ends.status() == 0


# ---------------------------------------------------------- used together ----

def stage(tokens, table, w_head, dtable, dw, seed):
    """One pass of a one-stage model: embedding, a dropped branch, the head, and back."""
    inp, out = tokens[:, :-1], tokens[:, 1:]
    e = ends.embed(inp, table, scale=4.0)
    x = ends.dropout_add(e, e, 0.2, seed, site=3)
    lp, kept = ends.head_logprobs(x, w_head, out, keep=True)
    a = torch.full(out.shape, -1.0 / out.numel(), device=DEV)
    dx = ends.head_logprobs_backward(a, kept, x, w_head, out, lp, dw)
    de = dx + ends.dropout_backward(dx, 0.2, seed, site=3)
    ends.embed_backward(de, inp, dtable, scale=4.0)
    return lp.logp, dx, de


def stage_case(seed=0):
    g = gen(seed)
    tokens = ids_of(g, (4, 65), 300)
    table, w = randn(g, 300, 72, scale=0.25), randn(g, 300, 72, scale=0.2)
    return tokens, table, w, torch.empty(300, 72, device=DEV), torch.empty(300, 72, device=DEV)


def test_a_stage_against_autograd():
    """torch's own in fp32, from the same mask: x, dx and dx's branch are rounded to bf16 on the
    way, 2^-9 in the norm each, and G: 1e-2 of the norms."""
    tokens, table, w, dtable, dw = stage_case()
    logp, dx, de = stage(tokens, table, w, dtable, dw, 77)
    mask = torch.from_numpy(ref.kept_mask(256, 72, 0.2, 77, 3)[0]).to(DEV).view(4, 64, 72)
    t, h = table.float().requires_grad_(), w.float().requires_grad_()
    ids, out = tokens[:, :-1], tokens[:, 1:]
    real, ok = (ids >= 0) & (ids < 300), (out >= 0) & (out < 300)
    e = 4.0 * t[ids.clamp(0, 299)] * real[..., None]
    x = e + e * mask * (65536 / (65536 - 13107))
    logs = torch.log_softmax(x @ h.t(), -1)
    lp = torch.where(ok, logs.gather(-1, out.clamp(0, 299)[..., None])[..., 0], 0.0)
    (-lp.mean()).backward()
    rel = lambda a, b: ((a.float() - b).norm() / b.norm()).item()
    assert rel(logp, lp.detach()) < 1e-2 and rel(dtable, t.grad) < 1e-2 and rel(dw, h.grad) < 1e-2


def test_a_stage_captured_in_a_graph():
    tokens, table, w, dtable, dw = stage_case(1)
    seed = torch.tensor([5], device=DEV)
    stage(tokens, table, w, dtable, dw, seed)
    graphs, outs = [], []
    for _ in range(2):   # two graphs beside one another
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(stage(tokens, table, w, dtable, dw, seed))
        graphs.append(graph)
    for s in (6, 7):
        seed.fill_(s)
        new = ids_of(gen(s), (4, 65), 300)
        tokens.copy_(new)
        for graph, out in zip(graphs, outs):
            graph.replay()
            got = [v.clone() for v in (*out, dtable, dw)]
            d2, w2 = torch.empty_like(dtable), torch.empty_like(dw)
            want = [*stage(new, table, w, d2, w2, s), d2, w2]
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_threads_and_streams_at_once():
    cases = [stage_case(10 + i) for i in range(4)]
    want = [[*stage(*c, i), c[3].clone(), c[4].clone()] for i, c in enumerate(cases)]
    torch.cuda.synchronize()
    got, wrong = [None] * 4, []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                c = [*cases[i][:3], torch.empty_like(cases[i][3]), torch.empty_like(cases[i][4])]
                for _ in range(20):
                    got[i] = [*stage(*c, i), *c[3:]]
                    with pytest.raises(dpo.DpoError, match="dpo_dropout: p"):
                        ends.dropout_add(c[1], None, 2.0, 1)
            stream.synchronize()
        except BaseException as e:
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong
    for a, b in zip(want, got):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_a_stream_given():
    tokens, table, w, dtable, dw = stage_case(20)
    want = stage(tokens, table, w, dtable, dw, 9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    e = ends.embed(tokens[:, :-1], table, scale=4.0, stream=s)
    x = ends.dropout_add(e, e, 0.2, 9, site=3, stream=s)
    lp, kept = ends.head_logprobs(x, w, tokens[:, 1:], keep=True, stream=s)
    top = ends.token_logprobs(x, top=2, stream=s)
    d2 = torch.empty_like(dw)
    a = torch.full((4, 64), -1.0 / 256, device=DEV)
    s.wait_stream(torch.cuda.current_stream())
    dx = ends.head_logprobs_backward(a, kept, x, w, tokens[:, 1:], lp, d2, stream=s)
    s.synchronize()
    assert torch.equal(lp.logp, want[0]) and torch.equal(dx, want[1]) and torch.equal(d2, dw)
    assert top.top_ids.shape == (4, 64, 2)


def test_an_optimizers_weights_and_gradients(cuda_device):
    """The table and the tied head of a DelayedAdamW: stale weights in, gradients out, the head's
    added to the embedding's."""
    tokens, table, w, _, _ = stage_case(30)
    opt = dpo.DelayedAdamW([300 * 72], stash_dtype=dpo.DPO_BF16, grad_dtype=dpo.DPO_F32, x0=[table.float().flatten()])
    try:
        stale, grad = opt.stale(0).view(300, 72), opt.grads(0).view(300, 72)
        assert torch.equal(stale, table)
        x = ends.embed(tokens[:, :-1], stale)
        lp, kept = ends.head_logprobs(x, stale, tokens[:, 1:], keep=True)
        a = torch.full((4, 64), -1.0 / 256, device=DEV)
        dx = ends.head_logprobs_backward(a, kept, x, stale, tokens[:, 1:], lp, grad)
        one = grad.clone()
        ends.embed_backward(dx, tokens[:, :-1], grad, accumulate=True)
        two = ends.embed_backward(dx, tokens[:, :-1], torch.empty_like(grad))
        assert torch.allclose(grad, one + two, rtol=1e-6, atol=1e-9)
        opt.step(lr=1e-3)
        assert torch.isfinite(opt.stale(0)).all()
    finally:
        opt.close()
