"""The feed-forward half of a pipeline stage on tensors: residual addition with the
root-mean-square norm, the gated feed-forward block, their backward passes, and
activations kept in 8 bits (include/dpo.h, "The feed-forward half of a pipeline
stage").

A stage runs its forward and backward at ``opt.stale(i)`` and writes the weights'
gradients into ``opt.grads(i)``, which the next ``opt.step`` reads:

    n = ffn.add_rms_norm(x, w_norm, residual=r, save8=True)
    out, kept = ffn.gated_ffn(n.y, w_gate, w_up, w_down)
    ...                                       # other microbatches; n.x8, n.rstd, kept wait
    dy = ffn.gated_ffn_backward(dout, kept, w_gate, w_up, w_down, dw_gate, dw_up, dw_down,
                                x8=n.x8, gain=w_norm)
    dx, _ = ffn.add_rms_norm_backward(dy, w_norm, n.rstd, x8=n.x8, dh=dout, dweight=dw_norm)

Every step of it runs in libdpo.so's kernels; PyTorch provides memory and streams.
Tensors are on the current CUDA device; their last dimension is contiguous and the
others flatten to rows. Outputs are allocated unless given. Calls go to PyTorch's
current stream, or to ``stream=`` (a torch.cuda.Stream), on which the outputs and
workspaces are then allocated too; tensors last used on another stream need the usual
event or ``wait_stream`` before the call. ValueError and TypeError for tensors that do
not fit, DpoError for what the library refuses.
"""
from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass
from typing import NamedTuple, Optional, Tuple

import torch

from . import dpo as _dpo
from .dpo import (DPO_ACT_GELU, DPO_ACT_SILU, DPO_BF16, DPO_F32, DPO_KEEP_8BIT, DPO_KEEP_BF16,
                  DPO_KEEP_NONE, DPO_PACK8_GROUP as GROUP, dpo_packed8)

_empty, _empty_like, _byref = torch.empty, torch.empty_like, ctypes.byref
_f32, _bf16, _u8 = torch.float32, torch.bfloat16, torch.uint8

ACTIVATIONS = {"silu": DPO_ACT_SILU, "gelu": DPO_ACT_GELU}
KEEP = {"none": DPO_KEEP_NONE, "8bit": DPO_KEEP_8BIT, "bf16": DPO_KEEP_BF16}
_DTYPES = {_f32: DPO_F32, _bf16: DPO_BF16}


@dataclass(frozen=True)
class Packed8:
    """A matrix in 8 bits: E4M3 ``codes`` (uint8, rows x cols) and the scale bytes of
    each row's groups of 32 (uint8, rows x ceil(cols / 32))."""
    codes: torch.Tensor
    scales: torch.Tensor

    @property
    def shape(self):
        return self.codes.shape

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.scales.numel()


class NormOut(NamedTuple):
    y: torch.Tensor
    h: torch.Tensor                 # x + residual (x itself without one)
    rstd: torch.Tensor              # fp32, one per row
    x8: Optional[Packed8]           # the normalised rows before the weight


@dataclass(frozen=True)
class Kept:
    """What ``gated_ffn`` keeps of its projections for the backward."""
    gate: object                    # Packed8, or a bf16 tensor
    up: object
    activation: str
    keep: str

    @property
    def nbytes(self) -> int:
        if self.keep == "8bit":
            return self.gate.nbytes + self.up.nbytes
        return 2 * (self.gate.numel() + self.up.numel())


# ---------------------------------------------------------------- helpers --
# Small calls are as long as their host side, so each check costs one attribute or two.

def _on_stream(call):
    """``stream=`` of a call: it allocates and launches on that stream."""
    @functools.wraps(call)
    def on_stream(*args, stream=None, **kw):
        if stream is None:
            return call(*args, **kw)
        with torch.cuda.stream(stream):
            return call(*args, **kw)
    return on_stream


def _run(name: str, args) -> None:
    _dpo._check(getattr(_dpo.load(), name)(_byref(args), _dpo._current_stream()), None)


def _rows(t, name: str):
    """(pointer, rows, columns, pitch) of t as a matrix with contiguous rows, not copied."""
    if not t.is_cuda:
        raise ValueError(f"{name} is not a CUDA tensor")
    if t.dim() != 2:
        if t.dim() == 0:
            raise ValueError(f"{name} has no dimensions")
        try:
            t = t.view(-1, t.shape[-1])
        except RuntimeError:
            raise ValueError(f"{name}: leading dimensions do not flatten to rows") from None
    rows, cols = t.shape
    if rows != 1 and t.is_contiguous():
        return t.data_ptr(), rows, cols, cols
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name}: the last dimension is not contiguous")
    if rows == 1 and not (ld >= cols and ld % 16 == 0):
        ld = cols   # a single row may report any stride
    return t.data_ptr(), rows, cols, ld


def _dtype(t, name: str) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise TypeError(f"{name}: {t.dtype} (float32 or bfloat16)")
    return d


def _fits(t, dtype, shape, device, name: str) -> None:
    if t.dtype != dtype:
        raise TypeError(f"{name}: {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not {device}")


def _vector(t, n: int, device, name: str) -> int:
    """Pointer of n contiguous elements."""
    if t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name}: expected {n} contiguous elements")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not {device}")
    return t.data_ptr()


def _matrix(t, rows: int, cols: int, dtype, device, name: str) -> int:
    """Pointer of a contiguous weight or gradient matrix."""
    if t.dtype != dtype:
        raise TypeError(f"{name}: {t.dtype}, expected {dtype}")
    if t.shape != (rows, cols) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {rows} x {cols} matrix, "
                         f"got {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not {device}")
    return t.data_ptr()


def _packed(p: Packed8, rows: int, cols: int, device, name: str) -> dpo_packed8:
    out = []
    for t, n in ((p.codes, cols), (p.scales, -(-cols // GROUP))):
        if t.dtype != _u8:
            raise TypeError(f"{name}: {t.dtype}, expected uint8")
        ptr, r, c, ld = _rows(t, name)
        if r != rows or c != n:
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {(rows, n)}")
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, not {device}")
        out += (ptr, ld)
    return dpo_packed8(out[0], out[2], out[1], out[3])


def _new_packed(rows: int, cols: int, device, pitch: int = 1):
    """Buffers of a rows x cols matrix in 8 bits, the codes' pitch a multiple of ``pitch``."""
    ld, groups = -(-cols // pitch) * pitch, -(-cols // GROUP)
    codes = _empty((rows, ld), dtype=_u8, device=device)
    scales = _empty((rows, groups), dtype=_u8, device=device)
    return (Packed8(codes if ld == cols else codes[:, :cols], scales),
            dpo_packed8(codes.data_ptr(), scales.data_ptr(), ld, groups))


def _new(ref):
    """An uninitialised tensor of ref's shape, contiguous."""
    return (_empty_like(ref) if ref.is_contiguous()
            else _empty(ref.shape, dtype=ref.dtype, device=ref.device))


# Sizes alone decide these.
_norm_workspace = functools.lru_cache(256)(
    lambda device, rows, cols: _dpo.dpo_rmsnorm_workspace(rows, cols))
_ffn_workspace = functools.lru_cache(256)(_dpo.dpo_ffn_workspace)


# ----------------------------------------------------- activations, 8 bits --

@_on_stream
def pack8(x) -> Packed8:
    """x (fp32 or bf16, any leading dimensions) in 8 bits."""
    ptr, rows, cols, ld = _rows(x, "x")
    dt = _dtype(x, "x")
    p, q = _new_packed(rows, cols, x.device)
    _dpo._check(_dpo.load().dpo_pack8(ptr, dt, rows, cols, ld, _byref(q), _dpo._current_stream()),
                None)
    return p


@_on_stream
def unpack8(p: Packed8, *, dtype=_bf16, out=None):
    """The values p stands for (bf16 holds them exactly)."""
    rows, cols = p.codes.shape
    q = _packed(p, rows, cols, p.codes.device, "p")
    if out is None:
        out = _empty((rows, cols), dtype=dtype, device=p.codes.device)
    else:
        _fits(out, out.dtype, p.codes.shape, p.codes.device, "out")
    ptr, _, _, ld = _rows(out, "out")
    _dpo._check(_dpo.load().dpo_unpack8(_byref(q), rows, cols, ptr, _dtype(out, "out"), ld,
                                        _dpo._current_stream()), None)
    return out


# -------------------------------------------------------------------- norm --

@_on_stream
def add_rms_norm(x, weight, residual=None, *, eps: float = 1e-5, save8: bool = False) -> NormOut:
    """s = x + residual, y = s / rms(s) * weight per row, with what the backward needs:
    rstd and either h (s in x's type) or, with ``save8``, the normalised rows in 8 bits."""
    px, rows, cols, ld_x = _rows(x, "x")
    dt, device = _dtype(x, "x"), x.device
    pw = _vector(weight, cols, device, "weight")
    pr = ld_r = ph = None
    h = x
    if residual is not None:
        _fits(residual, x.dtype, x.shape, device, "residual")
        pr, _, _, ld_r = _rows(residual, "residual")
        h = _new(x)
        ph = h.data_ptr()
    y = _new(x)
    rstd = _empty(rows, dtype=_f32, device=device)
    x8, q = _new_packed(rows, cols, device) if save8 else (None, _NO_PACKED)
    _run("dpo_rmsnorm", _dpo.dpo_rmsnorm_args(
        px, pr, pw, ph, y.data_ptr(), rstd.data_ptr(), q, rows, cols, ld_x, ld_r or cols, cols, cols,
        eps, dt, _dtype(weight, "weight")))
    return NormOut(y, h, rstd, x8)


_NO_PACKED = dpo_packed8()


@_on_stream
def add_rms_norm_backward(dy, weight, rstd, *, h=None, x8: Optional[Packed8] = None, dh=None,
                          dweight=None, accumulate: bool = False):
    """(dx, dweight) from the forward's h or x8; dx is the gradient of x and of residual
    alike. ``dh``: the gradient that reaches the sum past the norm. ``dweight``: the
    buffer to write (fp32 or bf16), or with ``accumulate`` to add to; fp32 by default."""
    if (h is None) == (x8 is None):
        raise ValueError("give one of h and x8")
    if accumulate and dweight is None:
        raise ValueError("accumulate needs a dweight to add to")
    pdy, rows, cols, ld_dy = _rows(dy, "dy")
    dt, device = _dtype(dy, "dy"), dy.device
    pw = _vector(weight, cols, device, "weight")
    if rstd.dtype != _f32:
        raise TypeError(f"rstd: {rstd.dtype}, expected float32")
    prstd = _vector(rstd, rows, device, "rstd")
    ph = pdh = None
    ld_h = ld_dh = cols
    q = _NO_PACKED
    if h is not None:
        _fits(h, dy.dtype, dy.shape, device, "h")
        ph, _, _, ld_h = _rows(h, "h")
    else:
        q = _packed(x8, rows, cols, device, "x8")
    if dh is not None:
        _fits(dh, dy.dtype, dy.shape, device, "dh")
        pdh, _, _, ld_dh = _rows(dh, "dh")
    if dweight is None:
        dweight = _empty(cols, dtype=_f32, device=device)
    pdw = _vector(dweight, cols, device, "dweight")
    dx = _new(dy)
    n = _norm_workspace(device, rows, cols)
    ws = _empty(n, dtype=_u8, device=device)
    _run("dpo_rmsnorm_backward", _dpo.dpo_rmsnorm_backward_args(
        pdy, ph, q, prstd, pw, pdh, dx.data_ptr(), pdw, rows, cols, ld_dy, ld_h, ld_dh, cols, dt,
        _dtype(weight, "weight"), _dtype(dweight, "dweight"), 1 if accumulate else 0,
        ws.data_ptr(), n))
    return dx, dweight


# ------------------------------------------------- gated feed-forward block --

def _sizes(x, w_gate, w_up, w_down, name: str):
    """(pointer, pitch, tokens, dim, hidden, the weights' pointers)."""
    px, tokens, dim, ld = _rows(x, name)
    if x.dtype != _bf16:
        raise TypeError(f"{name}: {x.dtype} (bfloat16)")
    device, hidden = x.device, w_gate.shape[0]
    return px, ld, tokens, dim, hidden, (_matrix(w_gate, hidden, dim, _bf16, device, "w_gate"),
                                         _matrix(w_up, hidden, dim, _bf16, device, "w_up"),
                                         _matrix(w_down, dim, hidden, _bf16, device, "w_down"))


@_on_stream
def gated_ffn(x, w_gate, w_up, w_down, *, activation: str = "silu", keep: str = "8bit",
              out=None) -> Tuple[torch.Tensor, Optional[Kept]]:
    """(out, kept): out = (act(x w_gate^T) * (x w_up^T)) w_down^T in bf16, with fp32
    accumulation. ``keep``: what is kept of the two projections for the backward, "8bit",
    "bf16" or "none" (kept is then None)."""
    act, kp = ACTIVATIONS.get(activation), KEEP.get(keep)
    if act is None or kp is None:
        raise ValueError(f"activation {activation!r}, keep {keep!r}")
    px, ld, tokens, dim, hidden, w = _sizes(x, w_gate, w_up, w_down, "x")
    n, _ = _ffn_workspace(tokens, dim, hidden)
    device = x.device
    if out is None:
        out = _new(x)
    else:
        _fits(out, _bf16, x.shape, device, "out")
    po, _, _, ld_out = _rows(out, "out")
    kept, pg, pu, g8, u8 = None, None, None, _NO_PACKED, _NO_PACKED
    if kp == DPO_KEEP_8BIT:
        g, g8 = _new_packed(tokens, hidden, device, 16)
        u, u8 = _new_packed(tokens, hidden, device, 16)
        kept = Kept(g, u, activation, keep)
    elif kp == DPO_KEEP_BF16:
        g = _empty((tokens, hidden), dtype=_bf16, device=device)
        u = _empty_like(g)
        pg, pu = g.data_ptr(), u.data_ptr()
        kept = Kept(g, u, activation, keep)
    ws = _empty(n, dtype=_u8, device=device)
    _run("dpo_ffn_forward", _dpo.dpo_ffn_args(px, *w, po, pg, pu, g8, u8, tokens, dim, hidden, ld,
                                              ld_out, act, kp, ws.data_ptr(), n))
    return out, kept


@_on_stream
def gated_ffn_backward(dout, kept: Kept, w_gate, w_up, w_down, dw_gate, dw_up, dw_down, *, x=None,
                       x8: Optional[Packed8] = None, gain=None, accumulate: bool = False, dx=None):
    """dx, and the weights' gradients written into dw_gate, dw_up and dw_down (all fp32 or
    all bf16, ``opt.grads(i)`` reshaped), or with ``accumulate`` added to them. The block's
    input is ``x``, or the 8-bit rows ``x8`` times ``gain`` (add_rms_norm's x8 and weight)."""
    if (x is None) == (x8 is None):
        raise ValueError("give one of x and x8")
    if gain is not None and x8 is None:
        raise ValueError("gain goes with x8")
    if kept is None:
        raise ValueError("the forward kept nothing (keep='none')")
    pd, ld, tokens, dim, hidden, w = _sizes(dout, w_gate, w_up, w_down, "dout")
    device, gdt = dout.device, dw_gate.dtype
    dt = _dtype(dw_gate, "dw_gate")
    dw = (_matrix(dw_gate, hidden, dim, gdt, device, "dw_gate"),
          _matrix(dw_up, hidden, dim, gdt, device, "dw_up"),
          _matrix(dw_down, dim, hidden, gdt, device, "dw_down"))
    px = pgain = pg = pu = None
    ld_x, gain_dt, q, g8, u8 = dim, 0, _NO_PACKED, _NO_PACKED, _NO_PACKED
    if x is not None:
        _fits(x, _bf16, dout.shape, device, "x")
        px, _, _, ld_x = _rows(x, "x")
    else:
        q = _packed(x8, tokens, dim, device, "x8")
        if gain is not None:
            pgain, gain_dt = _vector(gain, dim, device, "gain"), _dtype(gain, "gain")
    if kept.keep == "8bit":
        g8 = _packed(kept.gate, tokens, hidden, device, "kept")
        u8 = _packed(kept.up, tokens, hidden, device, "kept")
    else:
        pg = _matrix(kept.gate, tokens, hidden, _bf16, device, "kept")
        pu = _matrix(kept.up, tokens, hidden, _bf16, device, "kept")
    _, n = _ffn_workspace(tokens, dim, hidden, x8 is not None)
    if dx is None:
        dx = _new(dout)
    else:
        _fits(dx, _bf16, dout.shape, device, "dx")
    pdx, _, _, ld_dx = _rows(dx, "dx")
    ws = _empty(n, dtype=_u8, device=device)
    _run("dpo_ffn_backward", _dpo.dpo_ffn_backward_args(
        pd, px, q, pgain, *w, pg, pu, g8, u8, pdx, *dw, tokens, dim, hidden, ld, ld_x, ld_dx,
        ACTIVATIONS[kept.activation], KEEP[kept.keep], dt, gain_dt, 1 if accumulate else 0,
        ws.data_ptr(), n))
    return dx


def status() -> int:
    """Error bits of the tensor-core kernels (0: healthy); waits for the device."""
    return _dpo.dpo_ffn_get_status()
