"""The feed-forward half of a pipeline stage in 64 bits (numpy): the definitions that
include/dpo.h states for dpo_pack8, dpo_rmsnorm, dpo_ffn_forward and their backward
passes, written from the formulas. Test infrastructure; shares no code with the package.
"""
from __future__ import annotations

import numpy as np

GROUP = 32


# --------------------------------------------------------------- 8 bits ----

def e4m3_values() -> np.ndarray:
    """The value of each of the 256 codes."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + f / 8) * np.exp2(e - 7.0), f / 8 * 2.0 ** -6)
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >= 128, -v, v)


_VALUES = e4m3_values()
_POSITIVE = _VALUES[:127]     # finite and increasing


def scale_bytes(x: np.ndarray) -> np.ndarray:
    """s of each group of 32 along a row: the smallest in [1, 254] with
    amax <= 448 * 2^(s - 127) over the finite magnitudes."""
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    a = np.zeros((rows, groups * GROUP))
    a[:, :cols] = np.where(np.isfinite(x), np.abs(x), 0.0)
    amax = a.reshape(rows, groups, GROUP).max(-1)
    s = np.ones(amax.shape, dtype=np.int64)
    pos = amax > 0
    m, e = np.frexp(amax[pos] / 448.0)          # amax / 448 = m 2^e, m in [0.5, 1)
    s[pos] = np.maximum(1, np.where(m == 0.5, e - 1, e) + 127)
    return s.astype(np.uint8)


def encode(x: np.ndarray):
    """(codes, scale bytes): each value to the nearest code, ties to the even code."""
    x = np.asarray(x, dtype=np.float64)
    s = scale_bytes(x)
    unit = np.exp2(np.repeat(s.astype(np.float64) - 127, GROUP, 1)[:, :x.shape[1]])
    z = np.abs(np.where(np.isfinite(x), x, 0.0)) / unit
    hi = np.searchsorted(_POSITIVE, z)           # first code >= z
    hi = np.minimum(hi, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = z - _POSITIVE[lo], _POSITIVE[hi] - z
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = code + np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8), s


def decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    unit = np.exp2(np.repeat(scales.astype(np.float64) - 127, GROUP, 1)[:, :codes.shape[1]])
    return _VALUES[codes] * unit


# ----------------------------------------------------------------- norm ----

def rms_norm(x, weight, eps, residual=None):
    """(y, s, rstd, normalised rows)."""
    s = x if residual is None else x + residual
    rstd = 1.0 / np.sqrt((s * s).mean(1) + eps)
    n = s * rstd[:, None]
    return n * weight, s, rstd, n


def rms_norm_backward(dy, weight, rstd, n, dh=None):
    """(dx, dweight) at the normalised rows n."""
    g = dy * weight
    dx = rstd[:, None] * (g - n * (g * n).mean(1, keepdims=True))
    return (dx if dh is None else dx + dh), (dy * n).sum(0)


# ------------------------------------------------------------------ ffn ----

def act(z, kind):
    """act(z) and its derivative."""
    if kind == "silu":
        s = 1 / (1 + np.exp(-z))
        return z * s, s + z * s * (1 - s)
    c = np.sqrt(2 / np.pi)
    t = np.tanh(c * (z + 0.044715 * z ** 3))
    return (0.5 * z * (1 + t),
            0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z ** 2))


def ffn(x, w_gate, w_up, w_down, kind):
    """(out, G, U, A)."""
    g, u = x @ w_gate.T, x @ w_up.T
    a = act(g, kind)[0] * u
    return a @ w_down.T, g, u, a


def ffn_backward(dout, x, g, u, w_gate, w_up, w_down, kind):
    """dx, dw_gate, dw_up, dw_down and the intermediate dG, dU, A at given G and U."""
    a, slope = act(g, kind)
    da = dout @ w_down
    dg, du, h = da * u * slope, da * a, a * u
    return dg @ w_gate + du @ w_up, dg.T @ x, du.T @ x, dout.T @ h, dg, du, h
