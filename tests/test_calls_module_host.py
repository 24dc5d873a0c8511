"""Extension modules that the binding cannot use: a warning, and every call goes through ctypes."""
import sys
import types

import pytest
import torch

import paper_2603_05232_amd
from paper_2603_05232_amd import binding

NAMES = ("act_lift_quant", "slide_sparse_gemm", "slide_sparse_gemm_fused", "mx4_quant", "mx4_dequant", "mx4_product", "expert_route", "expert_combine")


def _module(names, **attributes):
    m = types.ModuleType("paper_2603_05232_amd._calls")
    m.torch_version = str(torch.__version__)
    for name in names:
        setattr(m, name, lambda *args: 1)
    vars(m).update(attributes)
    return m


@pytest.mark.parametrize("stale", [_module(NAMES, torch_version="1.0", bind=lambda *args: None, bind_mx4=lambda *args: None),       # of another torch
                                   _module(NAMES[:3], bind=lambda *args: None),                                                     # of before the 4-bit operators
                                   _module(NAMES, bind=lambda *args: None),
                                   _module(NAMES[:4], bind=lambda *args: None, bind_mx4=lambda *args: None)])
def test_a_module_of_another_build(monkeypatch, stale):
    lib = binding.load()
    monkeypatch.setitem(sys.modules, "paper_2603_05232_amd._calls", stale)
    monkeypatch.setattr(paper_2603_05232_amd, "_calls", stale, raising=False)
    with pytest.warns(RuntimeWarning, match="ctypes"):
        calls = binding._load_calls(lib)
    assert all(getattr(calls, name)() is None for name in NAMES)


def test_the_module_of_this_build():
    calls = binding._load_calls(binding.load())
    assert calls is sys.modules["paper_2603_05232_amd._calls"] and all(hasattr(calls, name) for name in NAMES)
