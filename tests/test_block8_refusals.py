"""What the 8-bit calls refuse, before anything is launched (no GPU: the addresses are never followed)."""
import ctypes as C

import numpy as np
import pytest

import block8_reference as ref
from paper_2311_14272_b200 import binding as B
from paper_2311_14272_b200 import build as build_mod


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return B.load()


def test_sizes(lib):
    assert B.crisp_quantize8_sizes(128, 8) == 1024 + 512
    assert B.crisp_quantize8_sizes(129, 9) == 2 * 2 * 1024 + 2 * 512
    assert B.crisp_quantize8_sizes(4096, 8192) == 4096 * 8192 + 32 * 64 * 512
    for k, ncols, code in ((0, 1, B.BAD_SHAPE), (1, 0, B.BAD_SHAPE), (-1, 5, B.BAD_SHAPE), (4096 * 128 + 1, 1, B.UNSUPPORTED), (4096, 1 << 30, B.UNSUPPORTED),
                           (1, 1 << 62, B.UNSUPPORTED)):
        with pytest.raises(B.CrispError) as e:
            B.crisp_quantize8_sizes(k, ncols)
        assert e.value.code == code
    assert lib.crisp_quantize8_sizes(1, 1, None) == B.INVALID_ARG


@pytest.mark.parametrize("args,code", [
    ((None, 8, 0, 64, 8, 4096), B.INVALID_ARG), ((4096, 8, 0, 64, 8, None), B.INVALID_ARG), ((4097, 8, 0, 64, 8, 4096), B.INVALID_ARG),
    ((4096, 8, 0, 64, 8, 4096 + 128), B.INVALID_ARG), ((4096, 8, 2, 64, 8, 4096), B.INVALID_ARG), ((4096, 7, 0, 64, 8, 4096), B.BAD_SHAPE),
    ((4096, 63, 1, 64, 8, 4096), B.BAD_SHAPE), ((4096, 8, 0, 0, 8, 4096), B.BAD_SHAPE), ((4096, 8, 0, 64, -1, 4096), B.BAD_SHAPE),
])
def test_quantize_refusals(lib, args, code):
    assert lib.crisp_quantize8(*args, None) == code


def test_null_handles_and_masks(lib):
    out, n, info = C.c_void_p(), C.c_size_t(), B.LaunchInfo()
    assert lib.crisp_encode8_sizes(None, C.byref(n)) == B.INVALID_ARG
    assert lib.crisp_encode8(4096, 8, None, 4096, None, C.byref(out)) == B.INVALID_ARG and not out.value
    assert lib.crisp_encode8(4096, 8, None, 4096, None, None) == B.INVALID_ARG
    assert lib.crisp_decode8(None, 4096, 8, None) == B.INVALID_ARG
    assert lib.crisp_spmm8(None, 4096, 8, 0, 8, 4096, 4096, 8, 0, 0, None) == B.INVALID_ARG
    assert lib.crisp_spmm8_quantized(None, 4096, 8, 4096, 8, 0, 0, None) == B.INVALID_ARG
    assert lib.crisp_set_epilogue8(None, None, 0) == B.INVALID_ARG
    assert lib.crisp_last_launch8(None, C.byref(info)) == B.INVALID_ARG
    assert lib.crisp_device_status8(None, None, None) == B.INVALID_ARG
    assert lib.crisp_reset_status8(None, None) == B.INVALID_ARG
    assert lib.crisp_set_tuning8(None, 0, 0, 0, -1) == B.INVALID_ARG
    lib.crisp_destroy8(None)


def test_reference_holds_values_as_the_format_says():
    codes = np.arange(127)
    field, part = codes >> 3, codes & 7
    values = np.where(field > 0, (1 + part / 8) * 2.0**(field - 7), part / 8 * 2.0**-6)
    assert np.array_equal(ref.nearest(values), values) and values.max() == 448
    assert [ref.exponent(v) for v in (448.0, 448.5, 224.0, 1.0, 0.0, 2.0**-140)] == [0, 1, -1, -8, -126, -126]
    # halfway: to the even code
    assert list(ref.nearest(np.array([17.0, 19.0, 2.0**-10, 3 * 2.0**-10]))) == [16.0, 20.0, 0.0, 2.0**-8]
