"""build.py: a library is built for its own user alone. No GPU."""
from __future__ import annotations

import os
import shutil

import pytest

from paper_2606_30634_gb300 import build, dpo, ffn, synth


@pytest.fixture
def out(tmp_path, monkeypatch):
    """An output folder of its own that holds the kernels' libraries and no dpo_tensors.so,
    with nothing loaded yet and no host compiler that could build the latter."""
    libs = build.build()
    for name in ("libdpo.so", "libdpo_synth.so"):
        shutil.copy(libs[name], tmp_path / name)   # newer than its sources
    monkeypatch.setattr(build, "OUT", str(tmp_path))
    monkeypatch.setattr(build, "CXX", str(tmp_path / "no-compiler"))
    monkeypatch.setattr(dpo, "_lib", None)
    monkeypatch.setattr(synth, "_lib", None)
    monkeypatch.setattr(ffn, "_t", ffn._Tensors())
    monkeypatch.delenv("DPO_LIBRARY", raising=False)
    return tmp_path


def test_the_optimizers_do_not_need_the_tensor_module(out):
    assert dpo.load().dpo_init is not None and synth.load() is not None
    assert sorted(os.listdir(out)) == ["libdpo.so", "libdpo_synth.so"]
    with pytest.raises((RuntimeError, OSError)):   # and it fails loudly where it is needed
        ffn._t.pack8


def test_a_module_of_another_pytorch_is_built_again(tmp_path, monkeypatch):
    path = build.build()["dpo_tensors.so"]
    monkeypatch.setattr(build, "OUT", str(tmp_path))
    for f in os.listdir(os.path.dirname(path)):
        if f.startswith("dpo_tensors.so"):   # newer than its sources
            shutil.copy(os.path.join(os.path.dirname(path), f), tmp_path / f)
    built = []
    monkeypatch.setattr(build, "_compile", lambda src, *a: built.append(src) or "")
    monkeypatch.setattr(build, "_run", lambda cmd, what: open(cmd[cmd.index("-o") + 1], "w").close())
    build.build(only=["dpo_tensors.so"])
    assert built == []
    import torch
    monkeypatch.setattr(torch, "__version__", "0.0")
    build.build(only=["dpo_tensors.so"])
    assert built == ["csrc/dpo_tensors.cpp"]
    build.build(only=["dpo_tensors.so"])
    assert len(built) == 1
