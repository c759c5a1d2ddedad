"""What the build compiles: the library with nvcc alone, the extension module of llm.py where PyTorch is there."""

import importlib.util

import pytest


@pytest.mark.parametrize("torch_there", [True, False])
def test_the_library_is_built_without_pytorch(monkeypatch, torch_there):
    from paper_2308_15164_b200 import build as b

    ran = []
    monkeypatch.setattr(b, "_run", lambda cmd, verbose=False: ran.append(cmd))
    monkeypatch.setattr(b, "_module_command", lambda target: ["module", target])
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: (object() if torch_there else None) if name == "torch" else find(name, *a))
    monkeypatch.setenv("NVCC", "nvcc")
    assert b.build(force=True) == b.LIB
    assert ran[0][0] == "nvcc" and b.LIB in ran[0]
    assert ran[1:] == ([["module", b.MODULE]] if torch_there else [])
