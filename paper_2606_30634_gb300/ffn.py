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
current stream, or to ``stream`` (a torch.cuda.Stream), on which the outputs and
workspaces are then allocated too; tensors last used on another stream need the usual
event or ``wait_stream`` before the call. ValueError and TypeError for tensors that do
not fit, DpoError for what the library refuses.
"""
from __future__ import annotations

import contextlib
import ctypes
from dataclasses import dataclass
from typing import NamedTuple, Optional, Tuple

import torch

from . import dpo as _dpo
from .dpo import (DPO_ACT_GELU, DPO_ACT_SILU, DPO_BF16, DPO_F32, DPO_KEEP_8BIT, DPO_KEEP_BF16,
                  DPO_KEEP_NONE, DPO_PACK8_GROUP as GROUP, dpo_packed8)

ACTIVATIONS = {"silu": DPO_ACT_SILU, "gelu": DPO_ACT_GELU}
KEEP = {"none": DPO_KEEP_NONE, "8bit": DPO_KEEP_8BIT, "bf16": DPO_KEEP_BF16}
_DTYPES = {torch.float32: DPO_F32, torch.bfloat16: DPO_BF16}


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

def _on(stream):
    """The context in which a call allocates."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _rows(t, name: str):
    """t as (rows x cols) with contiguous rows, without a copy."""
    if not t.is_cuda:
        raise ValueError(f"{name} is not a CUDA tensor")
    if t.dim() == 2:
        m = t
    elif t.dim() == 0:
        raise ValueError(f"{name} has no dimensions")
    else:
        try:
            m = t.view(-1, t.shape[-1])
        except RuntimeError:
            raise ValueError(f"{name}: leading dimensions do not flatten to rows") from None
    if m.shape[1] > 1 and m.stride(1) != 1:
        raise ValueError(f"{name}: the last dimension is not contiguous")
    return m


def _ld(m) -> int:
    """Pitch. A single row may report any stride: one that no pitch can be is replaced."""
    rows, cols = m.shape
    ld = m.stride(0)
    return ld if rows > 1 or (ld >= cols and ld % 16 == 0) else cols


def _dtype(t, name: str) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise TypeError(f"{name}: {t.dtype} (float32 or bfloat16)")
    return d


def _like(t, ref, name: str, shape=None, dtype=None):
    if t.dtype != (dtype or ref.dtype):
        raise TypeError(f"{name}: {t.dtype}, expected {dtype or ref.dtype}")
    if tuple(t.shape) != tuple(ref.shape if shape is None else shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected "
                         f"{tuple(ref.shape if shape is None else shape)}")
    if t.device != ref.device:
        raise ValueError(f"{name} is on {t.device}, not {ref.device}")
    return t


def _vector(t, n: int, ref, name: str):
    if tuple(t.shape) != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name}: expected {n} contiguous elements")
    if t.device != ref.device:
        raise ValueError(f"{name} is on {t.device}, not {ref.device}")
    return t


def _matrix(t, rows: int, cols: int, ref, name: str, dtypes=(torch.bfloat16,)):
    """A contiguous weight or gradient matrix."""
    if t.dtype not in dtypes:
        raise TypeError(f"{name}: {t.dtype}")
    if tuple(t.shape) != (rows, cols) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {rows} x {cols} matrix, "
                         f"got {tuple(t.shape)}")
    if t.device != ref.device:
        raise ValueError(f"{name} is on {t.device}, not {ref.device}")
    return t


def _packed(p: Packed8, rows: int, cols: int, ref, name: str) -> dpo_packed8:
    q, s = p.codes, p.scales
    groups = -(-cols // GROUP)
    for t, shape in ((q, (rows, cols)), (s, (rows, groups))):
        if t.dtype != torch.uint8:
            raise TypeError(f"{name}: {t.dtype}, expected uint8")
        if t.numel() != shape[0] * shape[1] or t.shape[-1] != shape[1]:
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {shape}")
        if t.device != ref.device:
            raise ValueError(f"{name} is on {t.device}, not {ref.device}")
    q, s = _rows(q, name), _rows(s, name)
    return dpo_packed8(q.data_ptr(), s.data_ptr(), _ld(q), max(_ld(s), groups))


def _new_packed(rows: int, cols: int, device, pitch: int = 1) -> Packed8:
    """Buffers of a rows x cols matrix in 8 bits, the codes' pitch a multiple of ``pitch``."""
    ld = -(-cols // pitch) * pitch
    codes = torch.empty((rows, ld), dtype=torch.uint8, device=device)
    return Packed8(codes if ld == cols else codes[:, :cols],
                   torch.empty((rows, -(-cols // GROUP)), dtype=torch.uint8, device=device))


# ----------------------------------------------------- activations, 8 bits --

def pack8(x, *, stream=None) -> Packed8:
    """x (fp32 or bf16, any leading dimensions) in 8 bits."""
    m = _rows(x, "x")
    dt = _dtype(x, "x")
    rows, cols = m.shape
    with _on(stream):
        p = _new_packed(rows, cols, x.device)
        _dpo.dpo_pack8(m, dt, rows, cols, _ld(m),
                       dpo_packed8(p.codes.data_ptr(), p.scales.data_ptr(), cols,
                                   p.scales.shape[1]), stream)
    return p


def unpack8(p: Packed8, *, dtype=torch.bfloat16, out=None, stream=None):
    """The values p stands for (bf16 holds them exactly)."""
    rows, cols = p.codes.shape
    q = _packed(p, rows, cols, p.codes, "p")
    with _on(stream):
        if out is None:
            out = torch.empty((rows, cols), dtype=dtype, device=p.codes.device)
        else:
            _like(out, p.codes, "out", dtype=out.dtype)
        m = _rows(out, "out")
        _dpo.dpo_unpack8(q, rows, cols, m, _dtype(out, "out"), _ld(m), stream)
    return out


# -------------------------------------------------------------------- norm --

def add_rms_norm(x, weight, residual=None, *, eps: float = 1e-5, save8: bool = False,
                 stream=None) -> NormOut:
    """s = x + residual, y = s / rms(s) * weight per row, with what the backward needs:
    rstd and either h (s in x's type) or, with ``save8``, the normalised rows in 8 bits."""
    m = _rows(x, "x")
    dt = _dtype(x, "x")
    rows, cols = m.shape
    _vector(weight, cols, x, "weight")
    a = _dpo.dpo_rmsnorm_args()
    r = None
    if residual is not None:
        r = _rows(_like(residual, x, "residual"), "residual")
        a.residual, a.ld_residual = r.data_ptr(), _ld(r)
    with _on(stream):
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        h = x if r is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
        x8 = None
        if save8:
            x8 = _new_packed(rows, cols, x.device)
            a.x8 = dpo_packed8(x8.codes.data_ptr(), x8.scales.data_ptr(), cols,
                               x8.scales.shape[1])
        a.x, a.weight, a.y, a.rstd = m.data_ptr(), weight.data_ptr(), y.data_ptr(), rstd.data_ptr()
        a.ld_x, a.ld_y, a.ld_h = _ld(m), cols, cols
        if r is not None:
            a.h = h.data_ptr()
        a.rows, a.cols, a.eps, a.dtype, a.weight_dtype = rows, cols, eps, dt, _dtype(weight, "weight")
        _dpo.dpo_rmsnorm(a, stream)
    return NormOut(y, h, rstd, x8)


def add_rms_norm_backward(dy, weight, rstd, *, h=None, x8: Optional[Packed8] = None, dh=None,
                          dweight=None, accumulate: bool = False, stream=None):
    """(dx, dweight) from the forward's h or x8; dx is the gradient of x and of residual
    alike. ``dh``: the gradient that reaches the sum past the norm. ``dweight``: the
    buffer to write (fp32 or bf16), or with ``accumulate`` to add to; fp32 by default."""
    if (h is None) == (x8 is None):
        raise ValueError("give one of h and x8")
    m = _rows(dy, "dy")
    dt = _dtype(dy, "dy")
    rows, cols = m.shape
    _vector(weight, cols, dy, "weight")
    if rstd.dtype != torch.float32:
        raise TypeError(f"rstd: {rstd.dtype}, expected float32")
    _vector(rstd, rows, dy, "rstd")
    a = _dpo.dpo_rmsnorm_backward_args()
    if h is not None:
        hm = _rows(_like(h, dy, "h"), "h")
        a.h, a.ld_h = hm.data_ptr(), _ld(hm)
    else:
        a.x8 = _packed(x8, rows, cols, dy, "x8")
    if dh is not None:
        dm = _rows(_like(dh, dy, "dh"), "dh")
        a.dh, a.ld_dh = dm.data_ptr(), _ld(dm)
    with _on(stream):
        dx = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
        if dweight is None:
            if accumulate:
                raise ValueError("accumulate needs a dweight to add to")
            dweight = torch.empty(cols, dtype=torch.float32, device=dy.device)
        _vector(dweight, cols, dy, "dweight")
        n = _dpo.dpo_rmsnorm_workspace(rows, cols)
        ws = torch.empty(n, dtype=torch.uint8, device=dy.device)
        a.dy, a.rstd, a.weight = m.data_ptr(), rstd.data_ptr(), weight.data_ptr()
        a.dx, a.dweight = dx.data_ptr(), dweight.data_ptr()
        a.rows, a.cols, a.ld_dy, a.ld_dx = rows, cols, _ld(m), cols
        a.dtype, a.weight_dtype = dt, _dtype(weight, "weight")
        a.dweight_dtype, a.accumulate = _dtype(dweight, "dweight"), 1 if accumulate else 0
        a.workspace, a.workspace_bytes = ws.data_ptr(), n
        _dpo.dpo_rmsnorm_backward(a, stream)
    return dx, dweight


# ------------------------------------------------- gated feed-forward block --

def _sizes(x, w_gate, w_up, w_down, name: str):
    m = _rows(x, name)
    if x.dtype != torch.bfloat16:
        raise TypeError(f"{name}: {x.dtype} (bfloat16)")
    tokens, dim = m.shape
    hidden = w_gate.shape[0]
    _matrix(w_gate, hidden, dim, x, "w_gate")
    _matrix(w_up, hidden, dim, x, "w_up")
    _matrix(w_down, dim, hidden, x, "w_down")
    return m, tokens, dim, hidden


def gated_ffn(x, w_gate, w_up, w_down, *, activation: str = "silu", keep: str = "8bit", out=None,
              stream=None) -> Tuple[torch.Tensor, Optional[Kept]]:
    """(out, kept): out = (act(x w_gate^T) * (x w_up^T)) w_down^T in bf16, with fp32
    accumulation. ``keep``: what is kept of the two projections for the backward, "8bit",
    "bf16" or "none" (kept is then None)."""
    act, kp = ACTIVATIONS.get(activation), KEEP.get(keep)
    if act is None or kp is None:
        raise ValueError(f"activation {activation!r}, keep {keep!r}")
    m, tokens, dim, hidden = _sizes(x, w_gate, w_up, w_down, "x")
    a = _dpo.dpo_ffn_args()
    kept = None
    with _on(stream):
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        om = _rows(_like(out, x, "out"), "out")
        if kp == DPO_KEEP_8BIT:
            g, u = (_new_packed(tokens, hidden, x.device, 16) for _ in range(2))
            a.gate8, a.up8 = (_packed(p, tokens, hidden, x, "kept") for p in (g, u))
            kept = Kept(g, u, activation, keep)
        elif kp == DPO_KEEP_BF16:
            g, u = (torch.empty((tokens, hidden), dtype=x.dtype, device=x.device)
                    for _ in range(2))
            a.gate, a.up = g.data_ptr(), u.data_ptr()
            kept = Kept(g, u, activation, keep)
        n, _ = _dpo.dpo_ffn_workspace(tokens, dim, hidden)
        ws = torch.empty(n, dtype=torch.uint8, device=x.device)
        a.x, a.w_gate, a.w_up, a.w_down = (t.data_ptr() for t in (m, w_gate, w_up, w_down))
        a.out, a.tokens, a.dim, a.hidden = om.data_ptr(), tokens, dim, hidden
        a.ld_x, a.ld_out, a.act, a.keep = _ld(m), _ld(om), act, kp
        a.workspace, a.workspace_bytes = ws.data_ptr(), n
        _dpo.dpo_ffn_forward(a, stream)
    return out, kept


def gated_ffn_backward(dout, kept: Kept, w_gate, w_up, w_down, dw_gate, dw_up, dw_down, *, x=None,
                       x8: Optional[Packed8] = None, gain=None, accumulate: bool = False,
                       dx=None, stream=None):
    """dx, and the weights' gradients written into dw_gate, dw_up and dw_down (all fp32 or
    all bf16, ``opt.grads(i)`` reshaped), or with ``accumulate`` added to them. The block's
    input is ``x``, or the 8-bit rows ``x8`` times ``gain`` (add_rms_norm's x8 and weight)."""
    if (x is None) == (x8 is None):
        raise ValueError("give one of x and x8")
    if gain is not None and x8 is None:
        raise ValueError("gain goes with x8")
    if kept is None:
        raise ValueError("the forward kept nothing (keep='none')")
    m, tokens, dim, hidden = _sizes(dout, w_gate, w_up, w_down, "dout")
    a = _dpo.dpo_ffn_backward_args()
    grads = (torch.bfloat16, torch.float32)
    _matrix(dw_gate, hidden, dim, dout, "dw_gate", grads)
    for t, shape, name in ((dw_up, (hidden, dim), "dw_up"), (dw_down, (dim, hidden), "dw_down")):
        _matrix(t, *shape, dout, name, (dw_gate.dtype,))
    if x is not None:
        xm = _rows(_like(x, dout, "x"), "x")
        a.x, a.ld_x = xm.data_ptr(), _ld(xm)
    else:
        a.x8 = _packed(x8, tokens, dim, dout, "x8")
        if gain is not None:
            a.gain, a.gain_dtype = _vector(gain, dim, dout, "gain").data_ptr(), _dtype(gain, "gain")
    if kept.keep == "8bit":
        a.gate8, a.up8 = (_packed(p, tokens, hidden, dout, "kept") for p in (kept.gate, kept.up))
    else:
        a.gate, a.up = (_matrix(t, tokens, hidden, dout, "kept").data_ptr()
                        for t in (kept.gate, kept.up))
    with _on(stream):
        if dx is None:
            dx = torch.empty(dout.shape, dtype=dout.dtype, device=dout.device)
        dxm = _rows(_like(dx, dout, "dx"), "dx")
        _, n = _dpo.dpo_ffn_workspace(tokens, dim, hidden, x8 is not None)
        ws = torch.empty(n, dtype=torch.uint8, device=dout.device)
        a.dout, a.w_gate, a.w_up, a.w_down = (t.data_ptr() for t in (m, w_gate, w_up, w_down))
        a.dx, a.dw_gate, a.dw_up, a.dw_down = (t.data_ptr() for t in (dxm, dw_gate, dw_up, dw_down))
        a.tokens, a.dim, a.hidden = tokens, dim, hidden
        a.ld_dout, a.ld_dx = _ld(m), _ld(dxm)
        a.act, a.keep = ACTIVATIONS[kept.activation], KEEP[kept.keep]
        a.grad_dtype, a.accumulate = _DTYPES[dw_gate.dtype], 1 if accumulate else 0
        a.workspace, a.workspace_bytes = ws.data_ptr(), n
        _dpo.dpo_ffn_backward(a, stream)
    return dx


def status() -> int:
    """Error bits of the tensor-core kernels (0: healthy); waits for the device."""
    return _dpo.dpo_ffn_get_status()
