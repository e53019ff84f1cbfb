"""What the group norm's calls and the way back from 8 bits refuse, before anything is launched (no GPU: the addresses are never followed), and the sizes that they name."""
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


def desc(**other):
    d = dict(batch=2, pixels=9, channels=32, groups=4, activation=1, dtype=0, eps=1e-5)
    d.update(other)
    return B.GroupNormDesc(*[d[n] for n in ("batch", "pixels", "channels", "groups", "activation", "dtype", "eps")])


@pytest.mark.parametrize("other,code", [
    (dict(batch=-1), B.BAD_SHAPE), (dict(pixels=0), B.BAD_SHAPE), (dict(channels=0), B.BAD_SHAPE), (dict(groups=0), B.BAD_SHAPE), (dict(groups=5), B.BAD_SHAPE),
    (dict(groups=-4), B.BAD_SHAPE), (dict(groups=64), B.BAD_SHAPE), (dict(activation=4), B.INVALID_ARG), (dict(activation=-1), B.INVALID_ARG),
    (dict(dtype=3), B.INVALID_ARG), (dict(eps=-1e-5), B.INVALID_ARG), (dict(eps=float("nan")), B.INVALID_ARG), (dict(eps=float("inf")), B.INVALID_ARG),
    (dict(pixels=1 << 31), B.UNSUPPORTED), (dict(batch=1 << 40), B.UNSUPPORTED), (dict(channels=1 << 20, groups=1), B.UNSUPPORTED),
    (dict(batch=1 << 14, pixels=1 << 26), B.UNSUPPORTED),
])
def test_descriptors(lib, other, code):
    d, n = desc(**other), C.c_size_t()
    for backward in (0, 1):
        assert lib.crisp_group_norm_sizes(C.byref(d), backward, C.byref(n)) == code
    assert lib.crisp_group_norm(C.byref(d), 4096, 32, None, None, 4096, 32, 4096, None, None, 4096, None) == code
    assert lib.crisp_group_norm_backward(C.byref(d), 4096, 32, 4096, 32, None, 4096, None, None, 4096, 32, None, None, 4096, None) == code


FORWARD = dict(x=4096, ldx=32, gamma=4096, beta=4096, y=4096, ldy=32, stats=4096, x8=None, y8=None, workspace=4096)
BACKWARD = dict(dy=4096, ld_dy=32, x=4096, ldx=32, x8=None, stats=4096, gamma=4096, beta=4096, dx=4096, ld_dx=32, dgamma=4096, dbeta=4096, workspace=4096)


@pytest.mark.parametrize("other,code", [
    (dict(x=None), B.INVALID_ARG), (dict(x=4097), B.INVALID_ARG), (dict(y=None), B.INVALID_ARG), (dict(y=4097), B.INVALID_ARG), (dict(stats=None), B.INVALID_ARG),
    (dict(stats=4100), B.INVALID_ARG), (dict(gamma=4098), B.INVALID_ARG), (dict(beta=4098), B.INVALID_ARG), (dict(y8=4096 + 128), B.INVALID_ARG),
    (dict(x8=4096 + 16), B.INVALID_ARG), (dict(workspace=4096 + 8), B.INVALID_ARG), (dict(ldx=31), B.BAD_SHAPE), (dict(ldy=31), B.BAD_SHAPE),
])
def test_forward(lib, other, code):
    d = desc()
    assert lib.crisp_group_norm(C.byref(d), *{**FORWARD, **other}.values(), None) == code
    assert lib.crisp_group_norm(None, *FORWARD.values(), None) == B.INVALID_ARG


@pytest.mark.parametrize("other,code", [
    (dict(dy=None), B.INVALID_ARG), (dict(dy=4097), B.INVALID_ARG), (dict(dx=None), B.INVALID_ARG), (dict(dx=4099), B.INVALID_ARG), (dict(x=None), B.INVALID_ARG),
    (dict(x8=4096), B.INVALID_ARG), (dict(x=None, x8=4096 + 64), B.INVALID_ARG), (dict(stats=None), B.INVALID_ARG), (dict(stats=4100), B.INVALID_ARG),
    (dict(gamma=4097), B.INVALID_ARG), (dict(dgamma=4098), B.INVALID_ARG), (dict(dbeta=4098), B.INVALID_ARG), (dict(workspace=None), B.INVALID_ARG),
    (dict(workspace=4096 + 4), B.INVALID_ARG), (dict(ld_dy=31), B.BAD_SHAPE), (dict(ldx=31), B.BAD_SHAPE), (dict(ld_dx=31), B.BAD_SHAPE),
])
def test_backward(lib, other, code):
    d = desc()
    assert lib.crisp_group_norm_backward(C.byref(d), *{**BACKWARD, **other}.values(), None) == code


def test_sizes(lib):
    n = C.c_size_t()
    assert lib.crisp_group_norm_sizes(C.byref(desc()), 2, C.byref(n)) == B.INVALID_ARG and lib.crisp_group_norm_sizes(C.byref(desc()), 0, None) == B.INVALID_ARG
    assert B.crisp_group_norm_sizes(desc(), False) == 0                      # one kernel
    assert B.crisp_group_norm_sizes(desc(), True) >= 2 * 2 * 32 * 4
    # a group of more channels than a CTA holds: two kernels, with partial sums of every group in between
    assert B.crisp_group_norm_sizes(desc(channels=1 << 15, groups=2), False) >= 2 * 2 * 8
    # one call more than the sums need is no call: nothing to do
    assert lib.crisp_group_norm(C.byref(desc(batch=0)), None, 32, None, None, None, 32, None, None, None, None, None) == B.OK
    assert lib.crisp_group_norm_backward(C.byref(desc(batch=0)), None, 32, None, 32, None, None, None, None, None, 32, None, None, None, None) == B.OK


@pytest.mark.parametrize("args,code", [
    ((None, 0, 64, 8, 4096, 8), B.INVALID_ARG), ((4096 + 16, 0, 64, 8, 4096, 8), B.INVALID_ARG), ((4096, 2, 64, 8, 4096, 8), B.INVALID_ARG),
    ((4096, 0, 64, 8, None, 8), B.INVALID_ARG), ((4096, 0, 64, 8, 4097, 8), B.INVALID_ARG), ((4096, 0, 64, 8, 4096, 7), B.BAD_SHAPE),
    ((4096, 1, 64, 8, 4096, 63), B.BAD_SHAPE), ((4096, 0, 0, 8, 4096, 8), B.BAD_SHAPE), ((4096, 0, 64, 0, 4096, 8), B.BAD_SHAPE),
])
def test_back_from_8_bits(lib, args, code):
    assert lib.crisp_dequantize8(*args, None) == code


def tensor(shape, strides=None, dtype=torch.bfloat16, device=torch.device("cuda", 0)):
    t = torch.empty(shape, dtype=dtype)
    return SimpleNamespace(shape=t.shape, stride=lambda: strides or t.stride(), dtype=dtype, device=device, is_cuda=True, numel=t.numel, is_contiguous=lambda: strides is None,
                           data_ptr=lambda: 4096)


def test_tensors_that_do_not_fit(lib, monkeypatch):
    called = []
    monkeypatch.setattr(B, "crisp_group_norm", lambda *a: called.append(a))
    monkeypatch.setattr(B, "crisp_group_norm_backward", lambda *a: called.append(a))
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_network", False)                                # (what the compiled code does not take, the Python code refuses)
    norm = B.GroupNorm(32, 4)
    elsewhere = torch.device("cuda", 1)
    for bad in (tensor((2, 3, 3, 31)), tensor((32,)), tensor((2, 3, 3, 32), dtype=torch.float64), tensor((2, 3, 3, 32), (288, 1, 96, 3)),
                tensor((2, 3, 3, 32), (288, 96, 32, 2)), tensor((2, 3, 3, 32), (300, 96, 32, 1))):
        with pytest.raises(AssertionError):
            norm.forward(bad)
    good = tensor((2, 3, 3, 32))
    with pytest.raises(AssertionError):
        norm.forward(good, plain_y=False)
    for p in (tensor((32,), dtype=torch.bfloat16), tensor((31,), dtype=torch.float32), tensor((32,), dtype=torch.float32, device=elsewhere)):
        with pytest.raises(AssertionError):
            B.GroupNorm(32, 4, weight=p).forward(good)
    stats = tensor((2, 4, 2), dtype=torch.float32)
    for dy, x, s in ((good, tensor((2, 3, 3, 32), dtype=torch.float32), stats), (good, tensor((2, 3, 3, 32), device=elsewhere), stats),
                     (good, tensor((2, 3, 4, 32)), stats), (good, good, tensor((2, 4), dtype=torch.float32)), (good, good, tensor((2, 4, 2))),
                     (good, good, tensor((2, 4, 2), dtype=torch.float32, device=elsewhere)), (good, B.Activations8(32, 17, good), stats),
                     (good, B.Activations8(64, 18, good), stats), (good, B.Activations8(32, 18, tensor((8,), device=elsewhere)), stats)):
        with pytest.raises(AssertionError):
            norm.backward(dy, x, s)
    assert not called
    with pytest.raises(KeyError):
        B.GroupNorm(32, 4, activation="gelu")
    with pytest.raises(B.CrispError):
        B.GroupNorm(32, 5)


def test_the_most_samples_and_pixels(lib):
    n = C.c_size_t()
    for backward in (0, 1):
        for most, other in ((dict(batch=(1 << 31) - 1, pixels=1), "batch"), (dict(pixels=(1 << 31) - 65537, batch=1), "pixels")):
            assert lib.crisp_group_norm_sizes(C.byref(desc(**most)), backward, C.byref(n)) == B.OK
            most[other] += 1
            assert lib.crisp_group_norm_sizes(C.byref(desc(**most)), backward, C.byref(n)) == B.UNSUPPORTED
        for batch in (32767, 32768, 65536, 1 << 20):
            assert lib.crisp_group_norm_sizes(C.byref(desc(batch=batch, pixels=1)), backward, C.byref(n)) == B.OK
