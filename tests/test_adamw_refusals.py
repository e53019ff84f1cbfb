"""What crisp_adamw refuses, before anything is launched (no GPU: the addresses are never followed)."""
import ctypes as C

import numpy as np
import pytest

import adamw_reference as ref
from paper_2311_14272_b200 import binding as B
from paper_2311_14272_b200 import build as build_mod


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return B.load()


def call(lib, tensor=None, params=None, n=1, twice=False):
    arr = (B.AdamwTensor * 2)()
    for i in range(2):
        T = arr[i]
        T.rows, T.k, T.d_w, T.ld_w, T.w_dtype, T.grad_dtype = 8, 16, 4096 + (0 if twice else 65536 * i), 16, 1, 1
        T.d_grad, T.ld_grad, T.d_m, T.d_v, T.d_m_exp, T.d_v_exp = 1 << 20, 16, 1 << 21, 1 << 22, 1 << 23, 1 << 24
    for name, value in (tensor or {}).items():
        setattr(arr[0], name, value)
    p = B.AdamwParams(1e-3, 0.9, 0.999, 1e-8, 1e-2, 1, 0, 8, 0)
    for name, value in (params or {}).items():
        setattr(p, name, value)
    return lib.crisp_adamw(n, arr, C.byref(p), None)


@pytest.mark.parametrize("tensor,code", [
    (dict(rows=-1), B.BAD_SHAPE), (dict(k=-1), B.BAD_SHAPE), (dict(k=1 << 31), B.UNSUPPORTED), (dict(rows=1 << 45), B.UNSUPPORTED),
    (dict(w_dtype=2), B.INVALID_ARG), (dict(grad_dtype=-1), B.INVALID_ARG), (dict(d_w=None), B.INVALID_ARG), (dict(d_m=None), B.INVALID_ARG),
    (dict(d_v=None), B.INVALID_ARG), (dict(d_w=4098), B.INVALID_ARG), (dict(d_grad=(1 << 20) + 2), B.INVALID_ARG), (dict(d_m=(1 << 21) + 8), B.INVALID_ARG),
    (dict(d_v=(1 << 22) + 4), B.INVALID_ARG), (dict(d_m_exp=None), B.INVALID_ARG), (dict(d_v_exp=None), B.INVALID_ARG), (dict(ld_w=15), B.BAD_SHAPE),
    (dict(ld_grad=15), B.BAD_SHAPE), (dict(d_copy_bf16=4097, ld_copy=16), B.INVALID_ARG), (dict(d_copy_bf16=4096, ld_copy=15), B.BAD_SHAPE),
    (dict(d_copy_bf16=4096, ld_copy=16, w_dtype=0), B.INVALID_ARG),
])
def test_tensors_that_are_refused(lib, tensor, code):
    assert call(lib, tensor) == code


@pytest.mark.parametrize("params", [
    dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(lr=float("nan")),
    dict(weight_decay=float("inf")), dict(step=0), dict(state_bits=16), dict(reserved=1), dict(d_lr=6), dict(d_step=4), dict(d_grad_scale=2),
])
def test_scalars_that_are_refused(lib, params):
    assert call(lib, params=params) == B.INVALID_ARG


def test_the_same_weights_twice_and_missing_tables(lib):
    assert call(lib, n=2, twice=True) == B.INVALID_ARG
    assert call(lib, n=-1) == B.INVALID_ARG
    assert lib.crisp_adamw(1, None, C.byref(B.AdamwParams(1e-3, 0.9, 0.999, 1e-8, 0, 1, 0, 32, 0)), None) == B.INVALID_ARG
    assert lib.crisp_adamw(0, None, None, None) == B.INVALID_ARG
    assert lib.crisp_adamw(0, None, C.byref(B.AdamwParams(1e-3, 0.9, 0.999, 1e-8, 0, 1, 0, 32, 0)), None) == B.OK
    assert call(lib, dict(d_grad=None), n=1) == B.OK and call(lib, dict(rows=0), n=1) == B.OK        # nothing to do


def test_moments_refusals(lib):
    good = [1 << 20, 1 << 21, 1 << 22, 1 << 23, 100, 1 << 24, 1 << 25, None]
    assert lib.crisp_adamw_moments(*good[:4], -1, *good[5:]) == B.BAD_SHAPE
    assert lib.crisp_adamw_moments(*good[:4], 0, *good[5:]) == B.OK
    for at, value in ((0, None), (1, None), (2, None), (3, None), (5, None), (6, None), (0, (1 << 20) + 8), (5, (1 << 24) + 1)):
        bad = list(good)
        bad[at] = value
        assert lib.crisp_adamw_moments(*bad) == B.INVALID_ARG


def test_reference_holds_values_as_the_format_says():
    """The reference's own forms: every code stands for itself, and rounding is unbiased to the resolution of its random numbers."""
    for root, codes in ((False, [c for c in range(256) if c & 127 != 127]), (True, range(256))):
        value = ref.decode(np.array(list(codes), np.uint8), np.array([127, 127], np.uint8), root)
        # a block whose largest value is the format's own: scale 1
        for v in value:
            held, _, e = ref.hold(np.array([v, 496.0 if root else 448.0]), np.array([0.999, 0.999]), root)
            assert held[0] == v and e[0] == 0
    random = (2 * np.arange(1024) + 1) / 2048
    for x in (1.0 / 3, 0.3, 100.1, 0.002):
        held, step, _ = ref.hold(np.full(1024, x), random, False)
        assert abs(held.mean() - x) <= step[0] / 2048 * 1.01
