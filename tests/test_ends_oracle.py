"""The 64-bit definitions of the pipeline's ends (oracle/ends.py) against known answers,
closed forms and central differences, and what the calls refuse before they touch the
device; no GPU."""
from __future__ import annotations

import ctypes
import os

import numpy as np
import pytest

from oracle import ends as ref
from paper_2606_30634_gb300 import dpo, ends
from test_abi_cpu import declared_functions

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ------------------------------------------------------------ definitions ----

def test_philox_known_answers():
    n = 0
    with open(os.path.join(ROOT, "tests", "golden", "philox4x32_10_kat.txt")) as f:
        for line in f:
            if not line.startswith("#") and line.strip():
                w = [int(v, 16) for v in line.split()]
                assert ref.philox(w[:4], w[4:6]) == w[6:]
                n += 1
    assert n >= 3


def test_mask_share_and_independence():
    """4096 elements at p = 0.3: six standard deviations of a fair draw are 0.043; two masks
    agree where both keep or both drop, 0.58 of them, with six of 0.047."""
    a, share = ref.kept_mask(16, 256, 0.3, 12345, 0)
    assert share == 19661 / 65536 and abs((1 - a.mean()) - share) < 0.043
    for other in (ref.kept_mask(16, 256, 0.3, 12345, 1)[0], ref.kept_mask(16, 256, 0.3, 12346, 0)[0],
                  np.roll(a, 1, 0), np.roll(a, 1, 1)):
        assert abs((a == other).mean() - 0.58) < 0.047
    assert ref.kept_mask(2, 9, 0.0, 1, 0)[0].all()


def test_embedding_closed_forms():
    table = np.arange(12.0).reshape(4, 3)
    out = ref.embed(np.array([[2, -1], [4, 0]]), table, 2.0)
    assert out.tolist() == [[[12, 14, 16], [0, 0, 0]], [[0, 0, 0], [0, 2, 4]]]
    g, mag, count = ref.embed_backward(np.ones((5, 3)) * np.array([1, -2, 3, 4, 5])[:, None],
                                       np.array([1, 1, 9, 3, -100]), 4, 0.5)
    assert g[:, 0].tolist() == [0, -0.5, 0, 2] and mag[:, 0].tolist() == [0, 1.5, 0, 2]
    assert count.tolist() == [0, 2, 0, 1]


def test_distribution_closed_forms():
    z = np.array([[0.0, 0, 0, 0], [5, -np.inf, 5, -np.inf], [-3e38] * 4, [7, -np.inf, -np.inf, -np.inf]])
    logp, h = ref.logprobs(z, np.array([1, 2, 3, 0]))
    assert np.allclose(logp, [-np.log(4), -np.log(2), -np.log(4), 0], atol=1e-15)
    assert np.allclose(h, [np.log(4), np.log(2), np.log(4), 0], atol=1e-15)
    logp, h = ref.logprobs(np.array([[-np.inf] * 3, [np.nan, 0, 1], [np.inf, 0, 1]]), np.array([0, 1, -1]))
    assert np.isnan(logp[:2]).all() and logp[2] == 0 and np.isnan(h).all()
    assert ref.top(np.array([[1.0, 3, 3, np.nan, 2]]), 5).tolist() == [[1, 2, 4, 0, 3]]


def test_nan_is_behind_masked_logits():
    z = np.array([[np.nan, -np.inf, 1.0, np.nan, -np.inf], [np.inf, np.nan, np.inf, 0.0, -0.0]])
    assert ref.top(z, 5).tolist() == [[2, 1, 4, 0, 3], [0, 2, 3, 4, 1]]


def test_gradient_by_differences():
    """Step 1e-5: truncation 1e-10 and rounding 1e-11 of values near 1, under 1e-8."""
    r = np.random.RandomState(0)
    z, ids = r.randn(5, 7) * 2, np.array([0, 3, -1, 6, 7])
    a, b = r.randn(5), r.randn(5)

    def f(v):
        logp, h = ref.logprobs(v, ids)
        return (a * logp + b * h).sum()

    g = ref.logits_gradient(z, ids, a, b)
    for i in np.ndindex(*z.shape):
        u, v = z.copy(), z.copy()
        u[i] += 1e-5
        v[i] -= 1e-5
        assert abs((f(u) - f(v)) / 2e-5 - g[i]) < 1e-8
    masked = z.copy()
    masked[:, 2] = -np.inf
    g = ref.logits_gradient(masked, ids, a, b)
    assert np.isfinite(g).all() and (g[:, 2] == 0).all()


# --------------------------------------------------------------- refusals ----

BASE = 1 << 32


def addr(i):
    return BASE + i * (1 << 28)


def ids_at(i=9, rows=1, cols=64, ld=64, size=8):
    return ends.dpo_ids(addr(i), rows, cols, ld, size)


def embed_args(**kw):
    d = dict(ids=ids_at(), table=addr(0), out=addr(1), vocab=1000, dim=64, ld_table=64, ld_out=64, scale=1.0,
             table_dtype=dpo.DPO_BF16, out_dtype=dpo.DPO_BF16)
    return ends.dpo_embed_args(**{**d, **kw})


def embed_back_args(**kw):
    d = dict(dy=addr(0), ids=ids_at(), dtable=addr(1), vocab=1000, dim=64, ld_dy=64, ld_dtable=64, scale=1.0,
             dtype=dpo.DPO_BF16, grad_dtype=dpo.DPO_F32, workspace=addr(2), workspace_bytes=1 << 24)
    return ends.dpo_embed_backward_args(**{**d, **kw})


def drop_args(**kw):
    d = dict(x=addr(0), residual=addr(1), y=addr(2), rows=64, cols=64, ld_x=64, ld_residual=64, ld_y=64,
             dtype=dpo.DPO_BF16, p=0.1)
    return ends.dpo_dropout_args(**{**d, **kw})


def log_args(**kw):
    d = dict(logits=addr(0), ids=ids_at(), logp=addr(1), entropy=addr(2), stats=addr(3), top_logp=addr(4),
             top_ids=addr(5), rows=64, vocab=1000, ld_logits=1000, scale=1.0, dtype=dpo.DPO_F32, top=4)
    return ends.dpo_logprobs_args(**{**d, **kw})


def log_back_args(**kw):
    d = dict(logits=addr(0), ids=ids_at(), stats=addr(1), entropy=addr(2), dlogp=addr(3), dentropy=addr(4),
             dlogits=addr(5), rows=64, vocab=1000, ld_logits=1000, ld_dlogits=1000, scale=1.0,
             dtype=dpo.DPO_F32)
    return ends.dpo_logprobs_backward_args(**{**d, **kw})


def head_args(**kw):
    d = dict(x=addr(0), w=addr(1), ids=ids_at(), logp=addr(2), entropy=addr(3), stats=addr(4),
             top_logp=addr(5), top_ids=addr(6), kept=addr(7), tokens=64, dim=64, vocab=1000, ld_x=64,
             scale=1.0, top=4, workspace=addr(8), workspace_bytes=1 << 27)
    return ends.dpo_head_args(**{**d, **kw})


def head_back_args(**kw):
    d = dict(x=addr(0), w=addr(1), ids=ids_at(), kept=addr(2), logp=addr(3), entropy=addr(4), stats=addr(5),
             dlogp=addr(6), dentropy=addr(7), dx=addr(8), dw=addr(10), tokens=64, dim=64, vocab=1000,
             ld_x=64, ld_dx=64, scale=1.0, grad_dtype=dpo.DPO_F32, workspace=addr(11),
             workspace_bytes=1 << 27)
    return ends.dpo_head_backward_args(**{**d, **kw})


def refused(name, args, code, match=""):
    lib = ends.lib()
    assert getattr(lib, name)(ctypes.byref(args), None) == code
    msg = lib.dpo_last_error(None).decode()
    assert msg.startswith(name + ":") and match in msg, msg


INF, NAN = float("inf"), float("nan")
E, A, D = dpo.DPO_EINVAL, dpo.DPO_EALIGN, dpo.DPO_EDTYPE
CASES = [
    ("dpo_embed", embed_args, [
        (dict(table=None), E), (dict(out=None), E), (dict(vocab=0), E), (dict(dim=0), E),
        (dict(vocab=1 << 31), E), (dict(ld_table=63), E), (dict(ld_out=63), E), (dict(scale=NAN), E),
        (dict(scale=INF), E), (dict(table_dtype=7), D), (dict(out_dtype=-1), D), (dict(table=addr(0) + 1), A),
        (dict(out=addr(1) + 1), A), (dict(out=addr(0) + 128 * 999), E), (dict(out=addr(9)), E),
        (dict(ids=ids_at(size=2)), D), (dict(ids=ids_at(rows=-1)), E), (dict(ids=ids_at(rows=2, ld=63)), E),
        (dict(ids=ids_at(rows=1 << 20, cols=1 << 20)), E), (dict(ids=ends.dpo_ids(addr(9) + 4, 1, 64, 64, 8)), A),
        (dict(ids=ends.dpo_ids(None, 1, 64, 64, 8)), E)]),
    ("dpo_embed_backward", embed_back_args, [
        (dict(dy=None), E), (dict(dtable=None), E), (dict(workspace=None), E), (dict(workspace_bytes=100), E),
        (dict(workspace=addr(2) + 128), A), (dict(ld_dy=63), E), (dict(ld_dtable=63), E), (dict(scale=NAN), E),
        (dict(dtype=5), D), (dict(grad_dtype=5), D), (dict(dtable=addr(1) + 2), A), (dict(dtable=addr(0)), E),
        (dict(workspace=addr(1)), E), (dict(dim=0), E)]),
    ("dpo_dropout", drop_args, [
        (dict(x=None), E), (dict(y=None), E), (dict(p=1.0), E), (dict(p=-0.1), E), (dict(p=NAN), E),
        (dict(p=1 - 2.0 ** -18), E), (dict(dtype=3), D), (dict(ld_x=63), E), (dict(ld_y=63), E),
        (dict(ld_residual=63), E), (dict(x=addr(0) + 1), A), (dict(seed_source=addr(5) + 4), A),
        (dict(y=addr(0) + 2), E), (dict(y=addr(0), ld_y=128), E), (dict(y=addr(1) + 64), E),
        (dict(residual=addr(0), y=addr(0)), E), (dict(rows=-1), E), (dict(seed_source=addr(2)), E)]),
    ("dpo_logprobs", log_args, [
        (dict(logits=None), E), (dict(logp=None), E), (dict(stats=None), E), (dict(top_ids=None), E),
        (dict(top_logp=None), E), (dict(top=33), E), (dict(top=-1), E), (dict(vocab=3, top=4), E),
        (dict(vocab=0, top=0), E), (dict(scale=0.0), E), (dict(scale=-1.0), E), (dict(scale=NAN), E),
        (dict(dtype=2), D), (dict(ld_logits=999), E), (dict(rows=63), E), (dict(logits=addr(0) + 2), A),
        (dict(logp=addr(0)), E), (dict(entropy=addr(1)), E)]),
    ("dpo_logprobs_backward", log_back_args, [
        (dict(logits=None), E), (dict(dlogits=None), E), (dict(stats=None), E), (dict(dlogp=None), E),
        (dict(entropy=None), E), (dict(ids=ends.dpo_ids(None, 1, 64, 64, 8)), E), (dict(scale=0.0), E),
        (dict(dlogits=addr(0), ld_dlogits=1008), E), (dict(dlogits=addr(0) + 4), E), (dict(dtype=9), D),
        (dict(ld_dlogits=999), E), (dict(rows=65), E), (dict(dlogits=addr(3)), E)]),
    ("dpo_head", head_args, [
        (dict(x=None), E), (dict(w=None), E), (dict(dim=60, ld_x=64), E), (dict(vocab=0, top=0), E),
        (dict(vocab=(1 << 26) + 1), E), (dict(tokens=-1), E), (dict(x=addr(0) + 8), A), (dict(ld_x=68), A),
        (dict(ld_x=56), E), (dict(w=addr(1) + 2), A), (dict(kept=addr(7) + 16), A), (dict(scale=INF), E),
        (dict(entropy=None), E), (dict(top=33), E), (dict(ids=ids_at(cols=63)), E),
        (dict(kept=None, workspace=None), E), (dict(kept=None, workspace_bytes=16), E), (dict(logp=addr(0)), E)]),
    ("dpo_head_backward", head_back_args, [
        (dict(x=None), E), (dict(w=None), E), (dict(dw=None), E), (dict(kept=None), E), (dict(logp=None), E),
        (dict(dlogp=None), E), (dict(workspace=None), E), (dict(workspace_bytes=16), E), (dict(grad_dtype=4), D),
        (dict(dw=addr(10) + 8), A), (dict(ld_dx=60), E), (dict(ld_dx=68), A), (dict(dx=addr(0)), E),
        (dict(dw=addr(1)), E), (dict(dim=4), E), (dict(ids=ends.dpo_ids(None, 1, 64, 64, 8)), E),
        (dict(tokens=1 << 40), E)]),
]


@pytest.mark.parametrize("name,make,kw,code", [(n, m, kw, c) for n, m, rows in CASES for kw, c in rows],
                         ids=[f"{n}-{i}" for n, _, rows in CASES for i in range(len(rows))])
def test_refusals(name, make, kw, code):
    refused(name, make(**kw), code)


def test_calls_without_arguments():
    for name, _, _ in CASES:
        assert getattr(ends.lib(), name)(None, None) == dpo.DPO_EINVAL


def test_workspace_sizes():
    assert ends.dpo_embed_workspace(0, 10, 8) > 0
    small, large = ends.dpo_embed_workspace(1000, 100, 64), ends.dpo_embed_workspace(1 << 20, 100, 64)
    assert small < large == ends.dpo_embed_workspace(65536, 100, 64)   # a span's
    with pytest.raises(dpo.DpoError):
        ends.dpo_embed_workspace(-1, 10, 8)
    with pytest.raises(dpo.DpoError):
        ends.dpo_head_workspace(10, 12, 100)
    assert all(v % 256 == 0 for v in ends.dpo_head_workspace(10, 64, 101, True))


def test_binding_types_every_entry_point():
    names = declared_functions(os.path.join(ROOT, "include", "dpo.h"))
    assert set(ends.EXPORTS) <= set(names)
    for n in ends.EXPORTS:
        assert getattr(ends.lib(), n).argtypes is not None
