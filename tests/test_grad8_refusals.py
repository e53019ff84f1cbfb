"""What the weight gradients refuse, before anything is launched (no GPU: the addresses are never followed), and the sizes that they name."""
import ctypes as C
from types import SimpleNamespace

import pytest
import torch

from paper_2311_14272_b200 import binding as B
from paper_2311_14272_b200 import build as build_mod


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return B.load()


def grad(conv=None, **other):
    d = dict(rows=32, k=64, ncols=100, conv=None, d_dy=4096, ld_dy=32, dy_layout=1, dw_dtype=1, d_act=4096, mask=None, d_dw=4096, ld_dw=64, accumulate=0, skip_fill=0, d_status=None)
    d.update(other)
    g = B.WeightGrad8(**d)
    if conv is not None:
        g.keep = B.ConvDesc(*conv)
        g.conv = C.pointer(g.keep)
    return g


@pytest.mark.parametrize("other,code", [
    (dict(rows=0), B.BAD_SHAPE), (dict(k=0), B.BAD_SHAPE), (dict(ncols=0), B.BAD_SHAPE), (dict(ncols=-5), B.BAD_SHAPE), (dict(ncols=1 << 31), B.UNSUPPORTED),
    (dict(k=1 << 20), B.UNSUPPORTED), (dict(dy_layout=2), B.INVALID_ARG), (dict(dw_dtype=2), B.INVALID_ARG), (dict(accumulate=2), B.INVALID_ARG), (dict(skip_fill=-1), B.INVALID_ARG),
    # 10 x 10 pixels of 64 channels under one tap are what the descriptor says; these are not
    (dict(conv=(1, 10, 10, 32, 1, 1, 0, 0)), B.BAD_SHAPE), (dict(conv=(1, 10, 9, 64, 1, 1, 0, 0)), B.BAD_SHAPE), (dict(conv=(0, 10, 10, 64, 1, 1, 0, 0)), B.BAD_SHAPE),
    (dict(conv=(1, 10, 10, 64, 1, 1, -1, 0)), B.BAD_SHAPE), (dict(conv=(1, 10, 10, 64, 0, 1, 0, 0)), B.BAD_SHAPE), (dict(conv=(1, 2, 2, 16, 2, 2, 0, 0)), B.BAD_SHAPE),
    (dict(conv=(1, 1, 1, 16, 4, 1, 0, 0)), B.BAD_SHAPE), (dict(conv=(1, 10, 10, 1, 1 << 16, 1 << 16, 1 << 30, 0)), B.BAD_SHAPE),
    (dict(conv=(1 << 30, 1 << 30, 1 << 30, 64, 1, 1, 0, 0)), B.BAD_SHAPE),
])
def test_descriptions(lib, other, code):
    g, n = grad(**other), C.c_size_t()
    assert lib.crisp_weight_grad8_sizes(C.byref(g), C.byref(n)) == code
    assert lib.crisp_weight_grad8(C.byref(g), 4096, None) == code


@pytest.mark.parametrize("other,code", [
    (dict(d_dy=None), B.INVALID_ARG), (dict(d_dy=4097), B.INVALID_ARG), (dict(d_act=None), B.INVALID_ARG), (dict(d_act=4096 + 128), B.INVALID_ARG), (dict(d_dw=None), B.INVALID_ARG),
    (dict(d_dw=4098), B.INVALID_ARG), (dict(d_dw=4097, dw_dtype=0), B.INVALID_ARG), (dict(d_status=4098), B.INVALID_ARG), (dict(ld_dy=31), B.BAD_SHAPE),
    (dict(ld_dy=99, dy_layout=0), B.BAD_SHAPE), (dict(ld_dw=63), B.BAD_SHAPE),
])
def test_arguments(lib, other, code):
    assert lib.crisp_weight_grad8(C.byref(grad(**other)), 4096, None) == code


def test_workspaces(lib):
    n = C.c_size_t()
    assert lib.crisp_weight_grad8_sizes(None, C.byref(n)) == B.INVALID_ARG and lib.crisp_weight_grad8_sizes(C.byref(grad()), None) == B.INVALID_ARG
    assert lib.crisp_weight_grad8(None, 4096, None) == B.INVALID_ARG
    assert lib.crisp_weight_grad8(C.byref(grad(ld_dy=33)), None, None) == B.INVALID_ARG and lib.crisp_weight_grad8(C.byref(grad()), 4096 + 64, None) == B.INVALID_ARG
    # one that TMA cannot address is brought into a form that it can
    assert B.crisp_weight_grad8_sizes(grad(ld_dy=33)) > B.crisp_weight_grad8_sizes(grad())


def tensor(shape, strides=None, dtype=torch.bfloat16, device=torch.device("cuda", 0)):
    t = torch.empty(shape, dtype=dtype)
    return SimpleNamespace(shape=t.shape, stride=lambda: strides or t.stride(), dtype=dtype, device=device, data_ptr=lambda: 4096)


def test_tensors_that_do_not_fit(lib, monkeypatch):
    called = []
    monkeypatch.setattr(B, "crisp_weight_grad8", lambda *a: called.append(a))
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    L = object.__new__(B.HybridLayer)
    L.torch, L.desc, L.device, L._gpu, L.mask, L.handle, L.handle8, L._grad_status = torch, B.make_desc(32, 64, 4, 4, 128, 128, 1.0), torch.device("cuda", 0), None, 0, 0, 0, None
    elsewhere = torch.device("cuda", 1)
    act, dy = B.Activations8(64, 100, tensor((8,))), tensor((100, 32))
    for bad in (dict(dy=tensor((32, 100))), dict(dy=tensor((100, 31))), dict(dy=tensor((100, 32), dtype=torch.float32)), dict(dy=tensor((100, 32), device=elsewhere)),
                dict(dy=tensor((100, 32), (1, 100))), dict(act=B.Activations8(63, 100, tensor((8,)))), dict(act=B.Activations8(64, 99, tensor((8,)))),
                dict(act=B.Activations8(64, 100, tensor((8,), device=elsewhere))), dict(masked=True), dict(accumulate=True), dict(dw=tensor((32, 64))),
                dict(dw=tensor((32, 63), dtype=torch.float32)), dict(dw=tensor((32, 64), (1, 32), torch.float32)), dict(dw=tensor((32, 64), dtype=torch.float32, device=elsewhere))):
        with pytest.raises(AssertionError):
            L.weight_gradient8(**{**dict(dy=dy, act=act, tokens=True), **bad})
    image, dy = B.Activations8(16, 100, tensor((8,))), tensor((1, 9, 9, 32))
    for bad in (dict(dy_nhwc=tensor((1, 9, 8, 32))), dict(dy_nhwc=tensor((1, 9, 9, 31))), dict(act=B.Activations8(15, 100, tensor((8,)))), dict(pad=1), dict(kernel_h=3),
                dict(dy_nhwc=tensor((1, 9, 9, 32), (9 * 9 * 40, 9 * 40 + 8, 40, 1))), dict(dy_nhwc=tensor((1, 9, 9, 32), (9 * 9 * 64, 9 * 64, 64, 2)))):
        with pytest.raises(AssertionError):
            L.weight_gradient8_conv(**{**dict(dy_nhwc=dy, act=image, kernel_h=2, kernel_w=2, pad=0), **bad})
    assert not called
