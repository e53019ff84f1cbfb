"""Tensors on another device than the layer's are refused before anything is called (no GPU: what is looked at is all that the tensors have)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2311_14272_b200 import binding as B

HERE, ELSEWHERE = torch.device("cuda", 0), torch.device("cuda", 1)


@pytest.fixture
def layer(monkeypatch):
    called = []
    for name in ("crisp_spmm8_quantized", "crisp_set_epilogue8", "crisp_set_epilogue"):
        monkeypatch.setattr(B, name, lambda *a, _name=name: called.append(_name))
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    L = object.__new__(B.HybridLayer)
    L.torch, L.desc, L.device, L._gpu = torch, B.make_desc(256, 128, 4, 4, 128, 128, 1.0), HERE, None
    L.handle = L.handle8 = L.mask = 0
    L._bias = L._bias8 = None
    L.called = called
    return L


def test_activations_that_were_quantised_on_another_device(layer):
    y = SimpleNamespace(device=HERE, dtype=torch.bfloat16, shape=(256, 8), stride=lambda: (8, 1), data_ptr=lambda: 4096)
    with pytest.raises(AssertionError):
        layer.spmm8(B.Activations8(128, 8, SimpleNamespace(device=ELSEWHERE)), y)
    with pytest.raises(AssertionError):
        layer.spmm8(B.Activations8(64, 8, SimpleNamespace(device=HERE)), y)
    assert not layer.called
    assert layer.spmm8(B.Activations8(128, 8, SimpleNamespace(device=HERE)), y) is y and layer.called == ["crisp_spmm8_quantized"]


@pytest.mark.parametrize("call,kept", [("set_epilogue8", "_bias8"), ("set_epilogue", "_bias")])
def test_a_bias_on_another_device(layer, call, kept):
    def bias(device, **other):
        return SimpleNamespace(**{**dict(device=device, is_cuda=True, dtype=torch.float32, numel=lambda: 256, is_contiguous=lambda: True), **other})
    for bad in (bias(ELSEWHERE), bias(HERE, dtype=torch.bfloat16), bias(HERE, numel=lambda: 255), bias(HERE, is_contiguous=lambda: False)):
        with pytest.raises(AssertionError):
            getattr(layer, call)(bad)
    assert not layer.called and getattr(layer, kept) is None
    good = bias(HERE)
    assert getattr(layer, call)(good) is layer and getattr(layer, kept) is good and len(layer.called) == 1
    getattr(layer, call)(None, relu=True)
    assert getattr(layer, kept) is None and len(layer.called) == 2


def test_masks_on_another_device_than_their_weights():
    w = SimpleNamespace(device=HERE, dtype=torch.float32)
    mask = SimpleNamespace(device=ELSEWHERE, mask=4096)
    with pytest.raises(AssertionError, match="one device"):
        B.AdamW([w, w], masks=[None, mask])
