"""The feed-forward calls from plain C (tests/c_abi/ffn_consumer.c): the same results as the
tensor calls give, bit for bit."""
from __future__ import annotations

import struct
import subprocess

import numpy as np
import pytest
import torch

from paper_2606_30634_gb300 import dpo, ffn
from test_c_consumer import _build_consumer
from test_ffn_gpu import ffn_case, randn

pytestmark = pytest.mark.gpu


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().tobytes()


@pytest.mark.parametrize("t,d,f", [(37, 136, 264), (300, 768, 2048)])
def test_plain_c_block(tmp_path, t, d, f):
    g, x, *w = ffn_case(t, d, f, seed=80)
    r, wn, dout = randn(g, t, d), 1 + randn(g, d, scale=0.1), randn(g, t, d, scale=1e-2)
    inp, outp = tmp_path / "in.bin", tmp_path / "out.bin"
    with open(inp, "wb") as file:
        file.write(struct.pack("<qqq", t, d, f))
        for v in (x, r, wn, *w, dout):
            file.write(bits(v))
    exe = _build_consumer(str(tmp_path), "ffn_consumer")
    run = subprocess.run([exe, str(inp), str(outp)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, f"the C consumer failed:\n{run.stdout}\n{run.stderr}"

    n = ffn.add_rms_norm(x, wn, r, save8=True)
    out, kept = ffn.gated_ffn(n.y, *w)
    dw = [torch.empty(v.shape, device=v.device) for v in w]
    dy = ffn.gated_ffn_backward(dout, kept, *w, *dw, x8=n.x8, gain=wn)
    dx, dwn = ffn.add_rms_norm_backward(dy, wn, n.rstd, x8=n.x8, dh=dout)
    raw, at = open(outp, "rb").read(), 0
    for name, v in (("out", out), ("dx", dx), ("dw_norm", dwn), ("dw_gate", dw[0]), ("dw_up", dw[1]),
                    ("dw_down", dw[2])):
        size = v.numel() * v.element_size()
        want = v.contiguous().view(torch.uint8).cpu().numpy().reshape(-1)
        assert np.array_equal(np.frombuffer(raw, np.uint8, size, at), want), name
        at += size
    status, code = struct.unpack_from("<Ii", raw, at)
    message = raw[at + 8:].split(b"\0")[0].decode()
    assert status == 0 and code == dpo.DPO_EINVAL
    assert message.startswith("dpo_ffn_forward") and str(f + 1) in message
