"""The feed-forward half of a pipeline stage on tensors: residual addition with the
root-mean-square norm, the gated feed-forward block, their backward passes, and
activations kept in 8 bits (include/dpo.h, "The feed-forward half of a pipeline
stage").

A stage runs its forward and backward at ``opt.stale(i)`` and writes the weights'
gradients into ``opt.grads(i)``, which the next ``opt.step`` reads. The block takes its
weights in bf16, so their optimizer is made with ``stash_dtype=DPO_BF16`` (DelayedMuon's
default; DelayedAdamW's is fp32, which the norm's weight may have):

    n = ffn.add_rms_norm(x, w_norm, residual=r, save8=True)
    out, kept = ffn.gated_ffn(n.y, w_gate, w_up, w_down)
    ...                                       # other microbatches; n.x8, n.rstd, kept wait
    dy = ffn.gated_ffn_backward(dout, kept, w_gate, w_up, w_down, dw_gate, dw_up, dw_down,
                                x8=n.x8, gain=w_norm)
    dx, _ = ffn.add_rms_norm_backward(dy, w_norm, n.rstd, x8=n.x8, dh=dout, dweight=dw_norm)

Every step of it runs in libdpo.so's kernels; PyTorch provides memory and streams, and
dpo_tensors (csrc/dpo_tensors.cpp) checks the tensors and makes the calls. Tensors are on
the current CUDA device; their last dimension is contiguous and the others flatten to
rows. Outputs are allocated unless given. Calls go to PyTorch's current stream, or to
``stream=`` (a torch.cuda.Stream), on which the outputs and workspaces are then allocated
too; tensors last used on another stream need the usual event or ``wait_stream`` before
the call, and ``record_stream`` if they are freed before it has run. Autograd does not see
these calls: outputs require no gradient, and the backward passes are the calls here.
ValueError and TypeError for tensors that do not fit, DpoError for what the library
refuses.
"""
from __future__ import annotations

import ctypes
import importlib.util
from typing import NamedTuple, Optional, Tuple

import torch

from . import build as _build
from . import dpo as _dpo
from .dpo import DPO_ACT_GELU, DPO_ACT_SILU, DPO_KEEP_8BIT, DPO_KEEP_BF16, DPO_KEEP_NONE

ACTIVATIONS = {"silu": DPO_ACT_SILU, "gelu": DPO_ACT_GELU}
KEEP = {"none": DPO_KEEP_NONE, "8bit": DPO_KEEP_8BIT, "bf16": DPO_KEEP_BF16}

# What dpo_tensors calls, in the order of its bind().
_CALLS = ("dpo_pack8", "dpo_unpack8", "dpo_rmsnorm", "dpo_rmsnorm_backward",
          "dpo_rmsnorm_workspace", "dpo_ffn_forward", "dpo_ffn_backward", "dpo_ffn_workspace",
          "dpo_embed", "dpo_embed_backward", "dpo_embed_workspace", "dpo_dropout", "dpo_logprobs",
          "dpo_logprobs_backward", "dpo_head", "dpo_head_backward", "dpo_head_workspace",
          "dpo_last_error")


class _Tensors:
    """dpo_tensors (csrc/dpo_tensors.cpp), loaded and bound to dpo.load()'s library by the
    first call. Raises when it cannot be built or loaded: there is no other implementation."""

    def __getattr__(self, name):
        lib = _dpo.load()
        path = _build.build(only=["dpo_tensors.so"])["dpo_tensors.so"]
        spec = importlib.util.spec_from_file_location("dpo_tensors", path)
        mod = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(mod)
        mod.bind(_dpo.DpoError,
                 *(ctypes.cast(getattr(lib, c), ctypes.c_void_p).value for c in _CALLS))
        global _t
        _t = mod
        return getattr(mod, name)


_t = _Tensors()


class Packed8(NamedTuple):
    """A tensor in 8 bits: E4M3 ``codes`` (uint8, its shape) and the scale bytes of the
    groups of 32 along its last dimension (uint8, ceil(n / 32) of them)."""
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


class Kept(NamedTuple):
    """What ``gated_ffn`` keeps of its projections for the backward: each a matrix of all
    tokens, a Packed8 or a bf16 tensor."""
    gate: object
    up: object
    activation: str
    keep: str

    @property
    def nbytes(self) -> int:
        if self.keep == "8bit":
            return self.gate.nbytes + self.up.nbytes
        return 2 * (self.gate.numel() + self.up.numel())


# ----------------------------------------------------- activations, 8 bits --

def pack8(x, *, stream=None) -> Packed8:
    """x (fp32 or bf16, any leading dimensions, which the result keeps) in 8 bits."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return pack8(x)
    return Packed8(*_t.pack8(x))


def unpack8(p: Packed8, *, dtype=torch.bfloat16, out=None, stream=None):
    """The values p stands for (bf16 holds them exactly)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return unpack8(p, dtype=dtype, out=out)
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise TypeError(f"dtype {dtype} (float32 or bfloat16)")
    return _t.unpack8(p[0], p[1], out, dtype is torch.bfloat16)


# -------------------------------------------------------------------- norm --

def add_rms_norm(x, weight, residual=None, *, eps: float = 1e-5, save8: bool = False,
                 stream=None) -> NormOut:
    """s = x + residual, y = s / rms(s) * weight per row, with what the backward needs:
    rstd and either h (s in x's type) or, with ``save8``, the normalised rows in 8 bits."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return add_rms_norm(x, weight, residual, eps=eps, save8=save8)
    y, h, rstd, codes, scales = _t.add_rms_norm(x, weight, residual, eps, save8)
    return NormOut(y, h, rstd, Packed8(codes, scales) if save8 else None)


def add_rms_norm_backward(dy, weight, rstd, *, h=None, x8: Optional[Packed8] = None, dh=None,
                          dweight=None, accumulate: bool = False, stream=None):
    """(dx, dweight) from the forward's h or x8; dx is the gradient of x and of residual
    alike. ``dh``: the gradient that reaches the sum past the norm. ``dweight``: the
    buffer to write (fp32 or bf16), or with ``accumulate`` to add to; fp32 by default."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return add_rms_norm_backward(dy, weight, rstd, h=h, x8=x8, dh=dh, dweight=dweight,
                                         accumulate=accumulate)
    if (h is None) == (x8 is None):
        raise ValueError("give one of h and x8")
    if accumulate and dweight is None:
        raise ValueError("accumulate needs a dweight to add to")
    codes, scales = (None, None) if x8 is None else x8
    return _t.add_rms_norm_backward(dy, weight, rstd, h, codes, scales, dh, dweight, accumulate)


# ------------------------------------------------- gated feed-forward block --

def gated_ffn(x, w_gate, w_up, w_down, *, activation: str = "silu", keep: str = "8bit", out=None,
              stream=None) -> Tuple[torch.Tensor, Optional[Kept]]:
    """(out, kept): out = (act(x w_gate^T) * (x w_up^T)) w_down^T in bf16, with fp32
    accumulation. ``keep``: what is kept of the two projections for the backward, "8bit",
    "bf16" or "none" (kept is then None)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return gated_ffn(x, w_gate, w_up, w_down, activation=activation, keep=keep, out=out)
    act, kp = ACTIVATIONS.get(activation), KEEP.get(keep)
    if act is None or kp is None:
        raise ValueError(f"activation {activation!r}, keep {keep!r}")
    out, g, gs, u, us = _t.gated_ffn(x, w_gate, w_up, w_down, act, kp, out)
    if kp == DPO_KEEP_NONE:
        return out, None
    if kp == DPO_KEEP_8BIT:
        g, u = Packed8(g, gs), Packed8(u, us)
    return out, Kept(g, u, activation, keep)


def gated_ffn_backward(dout, kept: Kept, w_gate, w_up, w_down, dw_gate, dw_up, dw_down, *, x=None,
                       x8: Optional[Packed8] = None, gain=None, accumulate: bool = False,
                       dx=None, stream=None):
    """dx, and the weights' gradients written into dw_gate, dw_up and dw_down (all fp32 or
    all bf16, ``opt.grads(i)`` reshaped), or with ``accumulate`` added to them. The block's
    input is ``x``, or the 8-bit rows ``x8`` times ``gain`` (add_rms_norm's x8 and weight)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return gated_ffn_backward(dout, kept, w_gate, w_up, w_down, dw_gate, dw_up, dw_down,
                                      x=x, x8=x8, gain=gain, accumulate=accumulate, dx=dx)
    if (x is None) == (x8 is None):
        raise ValueError("give one of x and x8")
    if gain is not None and x8 is None:
        raise ValueError("gain goes with x8")
    if kept is None:
        raise ValueError("the forward kept nothing (keep='none')")
    g, u, activation, keep = kept
    (g, gs), (u, us) = (g, u) if keep == "8bit" else ((g, None), (u, None))
    codes, scales = (None, None) if x8 is None else x8
    return _t.gated_ffn_backward(dout, ACTIVATIONS[activation], KEEP[keep], g, gs, u, us, w_gate,
                                 w_up, w_down, dw_gate, dw_up, dw_down, x, codes, scales, gain,
                                 accumulate, dx)


def status() -> int:
    """Error bits of the tensor-core kernels (0: healthy), until dpo.dpo_ffn_clear_status
    clears them; waits for the device."""
    return _dpo.dpo_ffn_get_status()
