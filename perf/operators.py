"""The operators of a pipeline stage's feed-forward half, as they are measured.

A stage of an asynchronous pipeline runs its forward at the stale weights, keeps
the activations of every microbatch in flight, and runs its backward from them
into the gradient buffers that the delayed optimizer step reads. Kinds of
case:

  "norm"  the residual's addition and the root-mean-square norm, with the
          normalised rows in 8 bits too (``save8``)
  "norm-back"  its backward, from the kept sum ("h") or from the 8-bit rows ("x8")
          of an earlier forward
  "pack"  an activation stored in 8 bits (E4M3, a power-of-two scale for each 32
          elements of a row) and read back
  "ffn"   the gated feed-forward block; with ``train`` its backward too, from the
          gate and up projections kept in 8 bits or in bf16 (``keep``), and from
          the block's input or its 8-bit normalised rows (``x8``)

Widths are those of the repository's parameter sets (768, 2048 x 8192, 4096 x
11008) and of its odd-sized tests, token counts generic.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
GROUP = 32           # elements that share a scale
EPS = 1e-5
LARGEST = 8192 * 4096 * 11008   # tokens x dim x hidden of the largest block


def listed():
    return [
        # one token of a 7B layer: latency of a single launch
        dict(name="norm-1-token", kind="norm", rows=1, cols=4096, dtype="bf16", residual=True,
             save8=False),
        # odd sizes, fp32, no residual stream
        dict(name="norm-odd-f32", kind="norm", rows=517, cols=777, dtype="f32", residual=False,
             save8=True),
        # a microbatch through a 7B layer's norm, the rows kept in 8 bits
        dict(name="norm-7b-8bit", kind="norm", rows=8192, cols=4096, dtype="bf16",
             residual=True, save8=True),
        # a 1B layer's norm, backward from the kept bf16 sum
        dict(name="norm-1b-back", kind="norm-back", rows=4096, cols=2048, dtype="bf16",
             residual=True, kept="h"),
        # a 7B layer's norm, backward from the 8-bit rows
        dict(name="norm-7b-back-8bit", kind="norm-back", rows=8192, cols=4096, dtype="bf16",
             residual=True, kept="x8"),
        # a small ragged fp32 activation: rows that end inside a group
        dict(name="pack-odd-f32", kind="pack", rows=300, cols=1555, dtype="f32"),
        # a 7B layer's hidden activation
        dict(name="pack-7b", kind="pack", rows=8192, cols=11008, dtype="bf16"),
        # evaluation of a single token: the weights' bytes count
        dict(name="ffn-7b-1-token", kind="ffn", tokens=1, dim=4096, hidden=11008, act="silu",
             train=False, keep="none", x8=False),
        # a short sequence through a 1B layer
        dict(name="ffn-1b-37-tokens", kind="ffn", tokens=37, dim=2048, hidden=8192, act="silu",
             train=False, keep="none", x8=False),
        # widths and a token count that end inside every tile, tanh-gelu gate
        dict(name="ffn-odd-step", kind="ffn", tokens=1001, dim=520, hidden=1560, act="gelu",
             train=True, keep="bf16", x8=True),
        # the ordinary step: a microbatch through a 1B layer
        dict(name="ffn-1b-step", kind="ffn", tokens=4096, dim=2048, hidden=8192, act="silu",
             train=True, keep="8bit", x8=False),
        # the largest: a microbatch through a 7B layer, all checkpoints in 8 bits
        dict(name="ffn-7b-step", kind="ffn", tokens=8192, dim=4096, hidden=11008, act="silu",
             train=True, keep="8bit", x8=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm-back", "pack", "ffn", "ffn", "ffn"])
    if kind in ("norm", "norm-back"):
        c = dict(kind=kind, rows=_log(rng, 1, 16384), cols=_log(rng, 33, 8192),
                 dtype=rng.choice(["bf16", "bf16", "f32"]), residual=rng.random() < 0.7)
        if kind == "norm":
            return dict(c, save8=rng.random() < 0.5)
        return dict(c, kept=rng.choice(["h", "x8"]))
    if kind == "pack":
        return dict(kind=kind, rows=_log(rng, 1, 8192), cols=_log(rng, 1, 11008),
                    dtype=rng.choice(["bf16", "f32"]))
    while True:
        tokens, dim, hidden = (_log(rng, 1, 8192), 8 * _log(rng, 8, 512), 8 * _log(rng, 8, 1376))
        if tokens * dim * hidden <= LARGEST:
            break
    train = rng.random() < 0.75
    return dict(kind=kind, tokens=tokens, dim=dim, hidden=hidden,
                act=rng.choice(["silu", "gelu"]), train=train,
                keep=rng.choice(["8bit", "bf16"]) if train else "none",
                x8=train and rng.random() < 0.5)


# ---------------------------------------------------------------- inputs ----

def _randn(gen, *shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)


def _activation(gen, rows, cols, dtype):
    """A residual-stream activation: a few channels an order above the others."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    loud = torch.rand(cols, generator=gen, device="cuda") < 0.01
    return (x * torch.where(loud, 12.0, 1.0)).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    if case["kind"] == "pack":
        s["x"] = _activation(gen, case["rows"], case["cols"], DT[case["dtype"]])
        return s
    if case["kind"] in ("norm", "norm-back"):
        n, d, dt = case["rows"], case["cols"], DT[case["dtype"]]
        s["w"] = _randn(gen, d, scale=0.1, dtype=dt) + 1
        if case["kind"] == "norm":
            s["x"] = _activation(gen, n, d, dt)
            s["r"] = _randn(gen, n, d, scale=0.5, dtype=dt) if case["residual"] else None
            return s
        h = _activation(gen, n, d, dt)   # what the forward of this microbatch left
        s["rstd"] = 1 / torch.sqrt(h.float().square().mean(1) + EPS)
        if case["kept"] == "h":
            s["h"] = h
        else:
            s["codes"], s["scales"] = _encode(h.float() * s["rstd"][:, None])
        s["dy"] = _randn(gen, n, d, scale=1e-3, dtype=dt)
        s["dh"] = _randn(gen, n, d, scale=1e-3, dtype=dt) if case["residual"] else None
        return s
    t, d, f = case["tokens"], case["dim"], case["hidden"]
    s["x"] = _randn(gen, t, d)
    s["wg"] = _randn(gen, f, d, scale=0.02)
    s["wu"] = _randn(gen, f, d, scale=0.02)
    s["wd"] = _randn(gen, d, f, scale=0.02)
    if case["train"]:
        s["dout"] = _randn(gen, t, d, scale=1e-3)
        s["dw"] = [torch.zeros_like(s[k]) for k in ("wg", "wu", "wd")]   # the gradient buffers
        if case["x8"]:   # the norm before the block kept its rows in 8 bits
            s["gain"] = _randn(gen, d, scale=0.1) + 1
            s["codes"], s["scales"] = _encode(s["x"].float() / s["gain"].float())
    return s


# ------------------------------------------------------------ plain forms ----

def _exponents(x):
    """e of each group of 32 along a row: the smallest with amax <= 448 * 2^e."""
    rows, cols = x.shape
    pad = -cols % GROUP
    x = torch.nn.functional.pad(x, (0, pad)).view(rows, -1, GROUP)
    amax = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(amax)               # amax = m 2^e, m in [0.5, 1)
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-126)   # 448 = 0.875 * 2^9
    return x, torch.where(amax > 0, e, -126)


def _encode(x):
    """(codes, scale bytes) of a 2-d fp32 tensor."""
    rows, cols = x.shape
    g, e = _exponents(x)
    q = torch.ldexp(g, -e[..., None]).to(torch.float8_e4m3fn)
    q = q.view(torch.uint8).view(rows, -1)[:, :cols].contiguous()
    return q, (e + 127).to(torch.uint8)


def _decode(codes, scales):
    rows, cols = codes.shape
    v = codes.view(torch.float8_e4m3fn).float()
    e = scales.int().repeat_interleave(GROUP, 1)[:, :cols] - 127
    return torch.ldexp(v, e)


def _through8(x):
    return _decode(*_encode(x))


def _act(g, kind):
    """act(g) and its derivative."""
    if kind == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    c, k = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(c * (g + k * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * k * g * g)


def _plain_norm(s):
    dt = s["x"].dtype
    h = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
    rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    xh = h * rstd
    out = dict(y=(xh * s["w"].float()).to(dt), rstd=rstd.view(-1))
    if s["r"] is not None:
        out["h"] = h.to(dt)
    if s["case"]["save8"]:   # bf16 holds every 8-bit value
        out["x8"] = _through8(xh).bfloat16()
    return out


def _plain_norm_back(s):
    rstd = s["rstd"][:, None]
    xh = s["h"].float() * rstd if "h" in s else _decode(s["codes"], s["scales"])
    dy = s["dy"].float()
    g = dy * s["w"].float()
    dx = rstd * (g - xh * (g * xh).mean(1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return dict(dx=dx.to(s["dy"].dtype), dw=(dy * xh).sum(0))


def _plain_ffn(s):
    case = s["case"]
    x, wg, wu, wd = (s[k].float() for k in ("x", "wg", "wu", "wd"))
    g, u = x @ wg.t(), x @ wu.t()
    out = (_act(g, case["act"])[0] * u) @ wd.t()
    if not case["train"]:
        return dict(out=out.bfloat16())
    if case["keep"] == "8bit":
        g, u = _through8(g), _through8(u)
    else:
        g, u = g.bfloat16().float(), u.bfloat16().float()
    if case["x8"]:
        x = _decode(s["codes"], s["scales"]) * s["gain"].float()
    a, slope = _act(g, case["act"])
    dout = s["dout"].float()
    da = dout @ wd
    dg, du = da * u * slope, da * a
    return dict(out=out.bfloat16(), dx=(dg @ wg + du @ wu).bfloat16(),
                dwg=(dg.t() @ x).bfloat16(), dwu=(du.t() @ x).bfloat16(),
                dwd=(dout.t() @ (a * u)).bfloat16())


# ------------------------------------------------------- the framework's ----

def _own_norm(s):
    from paper_2606_30634_gb300 import ffn
    n = ffn.add_rms_norm(s["x"], s["w"], residual=s["r"], eps=EPS, save8=s["case"]["save8"])
    out = dict(y=n.y, rstd=n.rstd)
    if s["r"] is not None:
        out["h"] = n.h
    if s["case"]["save8"]:
        out["x8"] = ffn.unpack8(n.x8)
    return out


def _own_norm_back(s):
    from paper_2606_30634_gb300 import ffn
    kept = dict(h=s["h"]) if "h" in s else dict(x8=ffn.Packed8(s["codes"], s["scales"]))
    dx, dw = ffn.add_rms_norm_backward(s["dy"], s["w"], s["rstd"], dh=s["dh"], **kept)
    return dict(dx=dx, dw=dw)


def _own_pack(s):
    from paper_2606_30634_gb300 import ffn
    return dict(x=ffn.unpack8(ffn.pack8(s["x"]), dtype=s["x"].dtype))


def _own_ffn(s):
    from paper_2606_30634_gb300 import ffn
    case = s["case"]
    w = (s["wg"], s["wu"], s["wd"])
    out, kept = ffn.gated_ffn(s["x"], *w, activation=case["act"], keep=case["keep"])
    if not case["train"]:
        return dict(out=out)
    if case["x8"]:
        x = dict(x8=ffn.Packed8(s["codes"], s["scales"]), gain=s["gain"])
    else:
        x = dict(x=s["x"])
    dx = ffn.gated_ffn_backward(s["dout"], kept, *w, *s["dw"], **x)
    return dict(out=out, dx=dx, dwg=s["dw"][0], dwu=s["dw"][1], dwd=s["dw"][2])


def _plain_pack(s):
    return dict(x=_through8(s["x"].float()).to(s["x"].dtype))


PLAIN = {"norm": _plain_norm, "norm-back": _plain_norm_back, "pack": _plain_pack, "ffn": _plain_ffn}
OWN = {"norm": _own_norm, "norm-back": _own_norm_back, "pack": _own_pack, "ffn": _own_ffn}


def run(s):
    return (OWN if own else PLAIN)[s["case"]["kind"]](s)


# ------------------------------------------------------------------ work ----

def work(case):
    if case["kind"] == "ffn":
        t, d, f = case["tokens"], case["dim"], case["hidden"]
        flops, size = 6 * t * d * f, 2 * (2 * t * d + 3 * d * f)
        if case["train"]:
            flops, size = 3 * flops, size + 2 * (2 * t * d + 3 * d * f)
            if case["x8"]:
                size += t * d + t * -(-d // GROUP) + 2 * d
        return dict(bytes=size, flops=flops)
    n, d = case["rows"], case["cols"]
    b = 4 if case["dtype"] == "f32" else 2
    packed = n * d + n * -(-d // GROUP)
    if case["kind"] == "pack":   # written and read back
        return dict(bytes=2 * n * d * b + 2 * packed, flops=4 * n * d)
    if case["kind"] == "norm":   # 8-bit rows: written, read back, written in bf16
        return dict(bytes=n * d * b * (4 if case["residual"] else 2) + d * b + 4 * n +
                    (2 * packed + 2 * n * d if case["save8"] else 0), flops=5 * n * d)
    kept = packed if case["kept"] == "x8" else n * d * b
    return dict(bytes=kept + n * d * b * (3 if case["residual"] else 2) + d * (b + 4) + 4 * n,
                flops=9 * n * d)


# ----------------------------------------------------------- in 64 bits ----

def _grid8(v):
    """Each value rounded to the nearest of its group's 8-bit ones: three bits of
    fraction above 2^-6, steps of 2^-9 below, times the group's power of two."""
    rows, cols = v.shape
    groups = -(-cols // GROUP)
    full = v.new_zeros(rows, groups * GROUP)
    full[:, :cols] = v
    full = full.reshape(rows * groups, GROUP)
    top = full.abs().max(1, keepdim=True).values
    unit = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -300))) - 8)
    unit = torch.where(top > 448 * unit, 2 * unit, unit).clamp(min=2.0 ** -126)
    z = full / unit
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(z / step) * step * unit).reshape(rows, -1)[:, :cols]


def _values8(codes, scales):
    """What 8-bit codes and their groups' scale bytes stand for."""
    c = codes.long()
    field, frac = c // 8 % 16, c % 8
    size = torch.where(field > 0, (8 + frac).double() * torch.exp2(field.double() - 10),
                       frac.double() * 2.0 ** -9)
    unit = torch.exp2(scales.double() - 127)[:, torch.arange(codes.shape[1], device=codes.device) // GROUP]
    return torch.where(c > 127, -size, size) * unit


def exact(case, seed):
    s = prepare(case, seed)
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and k not in ("codes", "scales")}
    if case["kind"] == "norm-back":
        if case["kept"] == "x8":
            unit = _values8(s["codes"], s["scales"])
        else:
            unit = torch.einsum("ij,i->ij", wide["h"], wide["rstd"])
        v = wide["dy"] * wide["w"]
        along = torch.einsum("ij,ij->i", v, unit) / case["cols"]
        dx = torch.einsum("ij,i->ij", v - along[:, None] * unit, wide["rstd"])
        if case["residual"]:
            dx += wide["dh"]
        return dict(dx=dx, dw=torch.einsum("ij,ij->j", wide["dy"], unit))
    x = wide["x"]
    if case["kind"] == "pack":
        return dict(x=_grid8(x))
    if case["kind"] == "norm":
        if case["residual"]:
            x = x + wide["r"]
        rms = (x.square().sum(1) / case["cols"] + EPS).sqrt()
        unit = x / rms[:, None]
        out = dict(y=unit * wide["w"], rstd=rms.reciprocal())
        if case["residual"]:
            out["h"] = x
        if case["save8"]:
            out["x8"] = _grid8(unit)
        return out
    if 18.0 * case["tokens"] * case["dim"] * case["hidden"] > 1e13:
        return None

    def gate(z):
        if case["act"] == "silu":
            return z * torch.sigmoid(z)
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))

    def gate_slope(z):   # z sigmoid(q(z)): sigmoid(q) + z q' sigmoid(q) sigmoid(-q)
        if case["act"] == "silu":
            q, dq = z, 1.0
        else:
            q = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
            dq = 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z ** 2)
        return torch.sigmoid(q) + z * dq * torch.sigmoid(q) * torch.sigmoid(-q)

    z, up = torch.mm(x, wide["wg"].T), torch.mm(x, wide["wu"].T)
    out = dict(out=torch.mm(gate(z) * up, wide["wd"].T))
    if not case["train"]:
        return out
    if case["keep"] == "8bit":
        z, up = _grid8(z), _grid8(up)
    else:
        z, up = z.bfloat16().double(), up.bfloat16().double()
    if case["x8"]:
        x = _values8(s["codes"], s["scales"]) * wide["gain"]
    back = torch.mm(wide["dout"], wide["wd"])
    dz, dup = back * up * gate_slope(z), back * gate(z)
    out["dx"] = torch.mm(dz, wide["wg"]) + torch.mm(dup, wide["wu"])
    out["dwg"], out["dwu"] = torch.mm(dz.T, x), torch.mm(dup.T, x)
    out["dwd"] = torch.mm(wide["dout"].T, gate(z) * up)
    return out
