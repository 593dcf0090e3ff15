"""The 64-bit definitions of the feed-forward operators (oracle/ffn.py) against closed
forms and central differences, and the binding's refusals; no GPU."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest

from oracle import ffn as ref
from paper_2606_30634_gb300 import dpo


def rng(seed=0):
    return np.random.RandomState(seed)


# ---------------------------------------------------------------- 8 bits ----

def test_code_table():
    v = ref.e4m3_values()
    assert v[0] == 0 and v[126] == 448 and np.isnan(v[127]) and np.isnan(v[255])
    assert v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[56] == 1.0
    assert np.all(np.diff(v[:127]) > 0) and np.array_equal(v[128:255], -v[:127])


@pytest.mark.parametrize("amax,unit", [(448.0, 1.0), (448.0000001, 2.0), (1.0, 2.0 ** -8),
                                       (1.75, 2.0 ** -8), (1.7500001, 2.0 ** -7), (0.0, 2.0 ** -126),
                                       (1e-38, 2.0 ** -126), (3e38, 2.0 ** 120)])
def test_scales(amax, unit):
    x = np.zeros((1, 40))
    x[0, 3] = -amax
    s = ref.scale_bytes(x)
    assert s.shape == (1, 2) and 2.0 ** (int(s[0, 0]) - 127) == unit and s[0, 1] == 1


def test_rounding_and_round_trip():
    v = ref.e4m3_values()
    x = v[:254][np.isfinite(v[:254])]
    x = np.concatenate([x, np.full(-x.size % 32, 448.0)]).reshape(1, -1)
    x[0, ::32] = 448.0                               # every group at scale 1
    q, s = ref.encode(x)
    assert np.all(s == 127) and np.array_equal(ref.decode(q, s), x)
    mid = np.zeros((1, 32))
    mid[0, :5] = [448.0, (1 + 1.125) / 2, (1.125 + 1.25) / 2, 2.0 ** -10, 3 * 2.0 ** -10]
    assert ref.decode(*ref.encode(mid))[0, :5].tolist() == [448.0, 1.0, 1.25, 0.0, 2.0 ** -8]
    odd = np.array([[np.inf, -np.inf, np.nan, 2.0, -3.0]])
    d = ref.decode(*ref.encode(odd))[0]
    assert np.isnan(d[:3]).all() and d[3] == 2.0 and d[4] == -3.0


# -------------------------------------------------------------- gradients ----

def difference(f, x, i, h=1e-5):
    """df/dx[i] of a scalar function by central differences."""
    a, b = x.copy(), x.copy()
    a[i] += h
    b[i] -= h
    return (f(a) - f(b)) / (2 * h)


# Central differences: truncation h^2 f''' / 6 ~ 1e-10 and rounding 2^-52 f / h ~ 1e-10
# of sums of order 10; 1e-6 leaves both far behind.
def close(a, b):
    assert abs(a - b) <= 1e-6 * max(1.0, abs(a)), (a, b)


def test_norm_gradient_by_differences():
    r = rng(1)
    x, w, dy, dh = r.randn(3, 7), r.randn(7), r.randn(3, 7), r.randn(3, 7)

    def loss(x, w):
        y, s, _, _ = ref.rms_norm(x, w, 1e-3)
        return (y * dy).sum() + (s * dh).sum()

    _, _, rstd, n = ref.rms_norm(x, w, 1e-3)
    dx, dw = ref.rms_norm_backward(dy, w, rstd, n, dh)
    for i in np.ndindex(3, 7):
        close(dx[i], difference(lambda v: loss(v, w), x, i))
    for i in range(7):
        close(dw[i], difference(lambda v: loss(x, v), w, i))


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_ffn_gradient_by_differences(kind):
    r = rng(2)
    x, wg, wu, wd = r.randn(4, 5), r.randn(6, 5), r.randn(6, 5), r.randn(5, 6)
    dout = r.randn(4, 5)
    loss = lambda *a: (ref.ffn(*a, kind)[0] * dout).sum()
    _, g, u, _ = ref.ffn(x, wg, wu, wd, kind)
    grads = ref.ffn_backward(dout, x, g, u, wg, wu, wd, kind)[:4]
    args = [x, wg, wu, wd]
    for k in range(4):
        for i in np.ndindex(*args[k].shape):
            f = lambda v: loss(*args[:k], v, *args[k + 1:])
            close(grads[k][i], difference(f, args[k], i))


# -------------------------------------------------------------- refusals ----
# Host-side checks return before any CUDA call: the addresses are never used.

BASE = 1 << 40
STEP = 1 << 34


def addr(i):
    return BASE + i * STEP


def packed(i, ld=4096, lds=128):
    return dpo.dpo_packed8(addr(i), addr(i + 1), ld, lds)


def norm_args(**kw):
    d = dict(x=addr(0), residual=addr(1), weight=addr(2), h=addr(3), y=addr(4), rstd=addr(5),
             x8=packed(6), rows=8, cols=4096, ld_x=4096, ld_residual=4096, ld_h=4096, ld_y=4096,
             eps=1e-5, dtype=dpo.DPO_BF16, weight_dtype=dpo.DPO_BF16)
    return dpo.dpo_rmsnorm_args(**{**d, **kw})


def norm_back_args(**kw):
    d = dict(dy=addr(0), h=addr(1), rstd=addr(2), weight=addr(3), dh=addr(4), dx=addr(5),
             dweight=addr(6), rows=8, cols=4096, ld_dy=4096, ld_h=4096, ld_dh=4096, ld_dx=4096,
             dtype=dpo.DPO_BF16, weight_dtype=dpo.DPO_BF16, dweight_dtype=dpo.DPO_F32,
             workspace=addr(7), workspace_bytes=1 << 30)
    return dpo.dpo_rmsnorm_backward_args(**{**d, **kw})


def ffn_args(**kw):
    d = dict(x=addr(0), w_gate=addr(1), w_up=addr(2), w_down=addr(3), out=addr(4),
             gate=addr(5), up=addr(6), gate8=packed(7, 512, 16), up8=packed(9, 512, 16), tokens=8,
             dim=256, hidden=512, ld_x=256, ld_out=256, act=0, keep=dpo.DPO_KEEP_8BIT,
             workspace=addr(11), workspace_bytes=1 << 20)
    return dpo.dpo_ffn_args(**{**d, **kw})


def ffn_back_args(**kw):
    d = dict(dout=addr(0), x=addr(1), w_gate=addr(2), w_up=addr(3), w_down=addr(4), gate=addr(5),
             up=addr(6), gate8=packed(7, 512, 16), up8=packed(9, 512, 16), dx=addr(11),
             dw_gate=addr(12), dw_up=addr(13), dw_down=addr(14), tokens=8, dim=256, hidden=512,
             ld_dout=256, ld_x=256, ld_dx=256, act=0, keep=dpo.DPO_KEEP_8BIT,
             grad_dtype=dpo.DPO_BF16, workspace=addr(15), workspace_bytes=1 << 20)
    return dpo.dpo_ffn_backward_args(**{**d, **kw})


def refused(name, args, code):
    L = dpo.load()
    rc = getattr(L, name)(ctypes.byref(args) if args is not None else None, None)
    msg = L.dpo_last_error(None).decode()
    assert rc == code, (rc, msg)
    assert msg.startswith(name), msg


E, A, T = dpo.DPO_EINVAL, dpo.DPO_EALIGN, dpo.DPO_EDTYPE


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), E), (dict(cols=0), E), (dict(cols=dpo.DPO_RMSNORM_MAX_COLS + 1), E),
    (dict(dtype=5), T), (dict(dtype=dpo.DPO_F32), T), (dict(x=None), E), (dict(weight=None), E),
    (dict(rstd=None), E), (dict(ld_x=4095), E), (dict(ld_y=1), E), (dict(eps=-1.0), E),
    (dict(eps=float("nan")), E), (dict(x=addr(0) + 1), A), (dict(rstd=addr(5) + 2), A),
    (dict(y=addr(3)), E), (dict(y=addr(0) + 8192 * 7), E), (dict(h=addr(1)), E),
    (dict(x8=packed(6, 100)), E), (dict(x8=packed(6, 4096, 127)), E),
    (dict(x8=dpo.dpo_packed8(addr(6), None, 4096, 128)), E)])
def test_norm_refusals(kw, code):
    refused("dpo_rmsnorm", norm_args(**kw), code)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), E), (dict(cols=0), E), (dict(dtype=3), T), (dict(dweight_dtype=2), T),
    (dict(dy=None), E), (dict(h=None), E), (dict(ld_h=4000), E), (dict(dweight=addr(6) + 1), A),
    (dict(rstd=None), E)])
def test_norm_backward_refusals(kw, code):
    refused("dpo_rmsnorm_backward", norm_back_args(**kw), code)


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), E), (dict(dim=0), E), (dict(dim=250), E), (dict(hidden=516), E), (dict(act=2), E),
    (dict(keep=3), E), (dict(x=None), E), (dict(w_up=None), E), (dict(out=None), E),
    (dict(workspace=None), E), (dict(workspace_bytes=100), E), (dict(x=addr(0) + 2), A),
    (dict(ld_x=255), E), (dict(ld_x=257), A), (dict(ld_out=260), A), (dict(out=addr(0)), E),
    (dict(workspace=addr(11) + 16), A), (dict(gate8=packed(7, 500, 16)), E),
    (dict(gate8=packed(7, 520, 16)), A), (dict(up8=packed(9, 512, 17)), E),
    (dict(keep=dpo.DPO_KEEP_BF16, gate=None), E), (dict(tokens=1 << 40), E),
    (dict(gate8=packed(9, 512, 16)), E)])
def test_ffn_refusals(kw, code):
    refused("dpo_ffn_forward", ffn_args(**kw), code)


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), E), (dict(hidden=4), E), (dict(act=-1), E), (dict(keep=dpo.DPO_KEEP_NONE), E),
    (dict(grad_dtype=2), T), (dict(dout=None), E), (dict(x=None), E), (dict(dw_up=None), E),
    (dict(dw_gate=addr(13)), E), (dict(workspace_bytes=8 * 512 * 2), E), (dict(workspace=None), E),
    (dict(gain=addr(20)), E), (dict(x=None, x8=packed(16, 256, 7)), E),
    (dict(x=None, x8=packed(16, 256, 8), gain=addr(20), gain_dtype=9), T),
    (dict(dx=addr(0)), E), (dict(ld_dx=260), A), (dict(gate8=packed(7, 528, 16)), E)])
def test_ffn_backward_refusals(kw, code):
    refused("dpo_ffn_backward", ffn_back_args(**kw), code)


def test_pack_refusals():
    L = dpo.load()
    p = packed(2, 64, 2)
    call = lambda x=addr(0), dt=dpo.DPO_BF16, r=4, c=64, ld=64, q=p: L.dpo_pack8(
        x, dt, r, c, ld, ctypes.byref(q) if q is not None else None, None)
    assert call(dt=7) == T and call(r=-1) == E and call(c=-5) == E and call(ld=63) == E
    assert call(x=None) == E and call(q=None) == E and call(x=addr(0) + 1) == A
    assert call(q=packed(2, 63, 2)) == E and call(q=packed(2, 64, 1)) == E
    assert call(q=packed(0, 64, 2)) == E           # the codes over x
    assert call(r=0) == dpo.DPO_OK and call(c=0) == dpo.DPO_OK
    assert L.dpo_last_error(None).decode().startswith("dpo_pack8")


def test_null_arguments():
    for name in ("dpo_rmsnorm", "dpo_rmsnorm_backward", "dpo_ffn_forward", "dpo_ffn_backward"):
        refused(name, None, E)
    assert dpo.load().dpo_ffn_get_status(None) == E
    assert dpo.load().dpo_rmsnorm_workspace(4, 0, None) == E


def test_workspace_sizes():
    f, b = dpo.dpo_ffn_workspace(1001, 520, 1560)
    assert f >= 1001 * 1560 * 2 and b >= 3 * 1001 * 1560 * 2
    assert dpo.dpo_ffn_workspace(1001, 520, 1560, True)[1] >= b + 1001 * 520 * 2
    with pytest.raises(dpo.DpoError) as e:
        dpo.dpo_ffn_workspace(4, 12, 64)
    assert e.value.code == E


def test_calls_of_no_rows_return_before_the_device():
    L = dpo.load()
    assert L.dpo_rmsnorm(ctypes.byref(norm_args(rows=0)), None) == dpo.DPO_OK
    assert L.dpo_rmsnorm_backward(ctypes.byref(norm_back_args(rows=0, accumulate=1)), None) == 0
    assert L.dpo_ffn_forward(ctypes.byref(ffn_args(tokens=0)), None) == dpo.DPO_OK
    assert L.dpo_ffn_backward(ctypes.byref(ffn_back_args(tokens=0, accumulate=1)), None) == 0
