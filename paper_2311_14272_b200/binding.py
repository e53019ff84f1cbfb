"""ctypes binding of libcrisp's C ABI (see include/crisp.h).

Argument marshalling only: every step of the path runs in the CUDA kernels of
``libcrisp.so``.  PyTorch supplies device buffers and streams.  There is no CPU or
PyTorch fallback: if the shared library is missing, loading raises.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import operator
import os
import re
import sys
from array import array
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcrisp.so")

OK, INVALID_ARG, UNSUPPORTED, BAD_SHAPE, BUFFER_TOO_SMALL, CUDA_ERROR, TIMEOUT = range(7)
PATH_DIRECT, PATH_DENSE, PATH_SPARSE, PATH_SPARSE2 = 0, 1, 2, 3
PATH_NAMES = {0: "direct", 1: "dense_tcgen05", 2: "sparse_tcgen05", 3: "sparse_tcgen05_two_addends"}


class LayerDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("k", C.c_int32), ("n", C.c_int32), ("m", C.c_int32),
                ("block_rows", C.c_int32), ("block_k", C.c_int32), ("keep_ratio", C.c_double),
                ("score_mode", C.c_int32)]


class RankLayer(C.Structure):
    _fields_ = [("d_scores", C.c_void_p), ("d_max_key", C.c_void_p), ("nrt", C.c_int32), ("nblk", C.c_int32),
                ("block_elems", C.c_int64), ("min_keep", C.c_int32), ("reserved", C.c_int32)]


class PruneLayer(C.Structure):
    _fields_ = [("desc", LayerDesc), ("d_w_bf16", C.c_void_p), ("ld_w", C.c_int64), ("d_grads", C.c_void_p),
                ("ld_grads", C.c_void_p), ("grad_dtypes", C.c_void_p), ("samples", C.c_int32), ("d_saliency", C.c_void_p),
                ("ld_s", C.c_int64), ("d_mask_buf", C.c_void_p), ("d_workspace", C.c_void_p), ("kkeep", C.c_int32),
                ("d_canonical_buf", C.c_void_p), ("d_exec_buf", C.c_void_p)]


class AdamwTensor(C.Structure):
    _fields_ = [("rows", C.c_int64), ("k", C.c_int64), ("d_w", C.c_void_p), ("ld_w", C.c_int64), ("w_dtype", C.c_int32), ("grad_dtype", C.c_int32),
                ("d_copy_bf16", C.c_void_p), ("ld_copy", C.c_int64), ("d_grad", C.c_void_p), ("ld_grad", C.c_int64), ("d_m", C.c_void_p),
                ("d_v", C.c_void_p), ("d_m_exp", C.c_void_p), ("d_v_exp", C.c_void_p), ("mask", C.c_void_p)]


class AdamwParams(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double),
                ("step", C.c_int64), ("seed", C.c_uint64), ("state_bits", C.c_int32), ("reserved", C.c_int32), ("d_lr", C.c_void_p),
                ("d_step", C.c_void_p), ("d_grad_scale", C.c_void_p)]


class ConvDesc(C.Structure):
    _fields_ = [("batch", C.c_int32), ("height", C.c_int32), ("width", C.c_int32), ("channels", C.c_int32),
                ("kernel_h", C.c_int32), ("kernel_w", C.c_int32), ("pad", C.c_int32), ("y_layout", C.c_int32)]


class GroupNormDesc(C.Structure):
    _fields_ = [("batch", C.c_int64), ("pixels", C.c_int64), ("channels", C.c_int32), ("groups", C.c_int32), ("activation", C.c_int32),
                ("dtype", C.c_int32), ("eps", C.c_double)]


class WeightGrad8(C.Structure):
    _fields_ = [("rows", C.c_int32), ("k", C.c_int32), ("ncols", C.c_int64), ("conv", C.POINTER(ConvDesc)), ("d_dy", C.c_void_p), ("ld_dy", C.c_int64),
                ("dy_layout", C.c_int32), ("dw_dtype", C.c_int32), ("d_act", C.c_void_p), ("mask", C.c_void_p), ("d_dw", C.c_void_p), ("ld_dw", C.c_int64),
                ("accumulate", C.c_int32), ("skip_fill", C.c_int32), ("d_status", C.c_void_p), ("wait_limit_cycles", C.c_uint64)]


class LaunchInfo(C.Structure):
    _fields_ = [("path", C.c_int32), ("tile_cols", C.c_int32), ("accumulators", C.c_int32), ("stack", C.c_int32),
                ("epilogue_warps", C.c_int32), ("stages", C.c_int32), ("ctas", C.c_int32), ("conv", C.c_int32),
                ("stage_blocks", C.c_int32)]

    def as_dict(self):
        return {f: int(getattr(self, f)) for f, _ in self._fields_}


class BytesModel(C.Structure):
    _fields_ = [("nnz", C.c_int64), ("vals_bytes", C.c_int64), ("idx_bytes", C.c_int64),
                ("blk_col_bytes", C.c_int64), ("x_bytes", C.c_int64), ("y_bytes", C.c_int64),
                ("useful_macs", C.c_int64), ("slot_macs", C.c_int64), ("path", C.c_int32)]

    def as_dict(self):
        return {f: int(getattr(self, f)) for f, _ in self._fields_}


class CrispError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = crisp_status_string(code) if _lib is not None else str(code)
        super().__init__(f"{where}: {msg} (status {code})")


_lib = None
_native = None                                            # the hot ones of the same calls on plain integers (csrc/calls.cpp)
_network = None                                           # what goes over all tensors of a network (csrc/network.cpp); False: not built


def _bind_network():
    """csrc/network.cpp for the library that is loaded, or False in a tree where it could not be built (it needs torch's headers) or was built for
    another torch or Python."""
    global _network
    lib = load()
    if _network is not False:
        import torch                                      # (the module's libraries)
        release = ".".join(re.findall(r"\d+", torch.__version__)[:3])
        try:
            from . import _network as module
            if getattr(module, "built_for", None) == "%s %d.%d" % (release, *sys.version_info[:2]):
                module.bind(*[C.cast(f, C.c_void_p).value for f in (lib.crisp_decode, lib.crisp_spmm8_sizes, lib.crisp_spmm8, lib.crisp_decode8,
                                                                        lib.crisp_encode8_sizes, lib.crisp_encode8, lib.crisp_destroy8, lib.crisp_adamw,
                                                                        lib.crisp_adamw_moments, lib.crisp_quantize8_sizes, lib.crisp_group_norm_sizes,
                                                                        lib.crisp_group_norm, lib.crisp_group_norm_backward, lib.crisp_weight_grad8_sizes,
                                                                        lib.crisp_weight_grad8)])
                _network = module
            else:
                _network = False
        except ImportError:
            _network = False
    return _network


class _CtypesCalls:
    """The calls of csrc/calls.cpp through ctypes: the same arguments and results, 1.5 us slower each.  For a tree where that
    module could not be built (it needs Python's headers)."""

    def __init__(self, lib):
        self._lib = lib
        self.spmm, self.decode = lib.crisp_spmm, lib.crisp_decode

    def spmm_conv(self, handle, activation, *rest):
        *conv, y, ldy, y_dtype, stream = rest
        if any(v != C.c_int32(v).value for v in conv):
            return BAD_SHAPE
        return self._lib.crisp_spmm_conv(handle, activation, ConvDesc(*conv), y, ldy, y_dtype, stream)

    def build_mask(self, saliency, ld, desc, mask_buf, workspace, stream, replaced):
        self._lib.crisp_mask_destroy(replaced)
        mask = C.c_void_p()
        code = self._lib.crisp_build_mask(saliency, ld, LayerDesc.from_address(desc), mask_buf, workspace, stream, C.byref(mask))
        return code, mask.value or 0

    def encode_sizes(self, mask):
        canonical, execution = C.c_size_t(), C.c_size_t()
        code = self._lib.crisp_encode_sizes(mask, C.byref(canonical), C.byref(execution))
        return code, canonical.value, execution.value

    def encode(self, w, ld, mask, canonical_buf, exec_buf, stream, replaced):
        self._lib.crisp_destroy(replaced)
        handle = C.c_void_p()
        code = self._lib.crisp_encode(w, ld, mask, canonical_buf, exec_buf, stream, C.byref(handle))
        return code, handle.value or 0


def load(path: Optional[str] = None):
    """Load libcrisp.so (built in-tree by ``paper_2311_14272_b200.build``)."""
    global _lib, _native
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise FileNotFoundError(
            f"{p} not found: build it with `python -m paper_2311_14272_b200.build` "
            "(there is no fallback implementation)")
    lib = C.CDLL(p)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    P = C.POINTER
    sig = {
        "crisp_keep_count": [P(LayerDesc), P(i32), P(i32)],
        "crisp_mask_sizes": [P(LayerDesc), P(sz), P(sz)],
        "crisp_build_mask": [vp, i64, P(LayerDesc), vp, vp, vp, P(vp)],
        "crisp_build_mask_static": [vp, i64, P(LayerDesc), vp, vp, P(vp)],
        "crisp_mask_export": [vp, vp, vp, vp],
        "crisp_mask_info": [vp, P(LayerDesc), P(i32), P(i32), P(i32)],
        "crisp_encode_sizes": [vp, P(sz), P(sz)],
        "crisp_encode": [vp, i64, vp, vp, vp, vp, P(vp)],
        "crisp_encoded_counts": [vp, P(i64), P(i64), P(i64)],
        "crisp_export": [vp, vp, vp, vp, vp],
        "crisp_decode": [vp, vp, i64, vp],
        "crisp_spmm": [vp, vp, i64, i64, vp, i64, i32, vp],
        "crisp_spmm_conv": [vp, vp, P(ConvDesc), vp, i64, i32, vp],
        "crisp_saliency_accumulate": [vp, i32, i64, i32, i32, vp, i64, i32, vp],
        "crisp_saliency_finish": [vp, i64, vp, i64, i32, i32, i32, vp, i64, vp],
        "crisp_saliency_finish_max": [vp, i64, vp, i64, i32, i32, i32, vp, i64, vp, vp],
        "crisp_build_mask_ex": [vp, i64, P(LayerDesc), vp, vp, C.c_uint32, vp, P(vp)],
        "crisp_mask_reselect": [vp, i32, vp, vp],
        "crisp_prune_fraction": [C.c_double, i32, i32, P(C.c_double)],
        "crisp_keep_ratio_for_count": [P(LayerDesc), i32, P(C.c_double)],
        "crisp_set_path": [vp, i32],
        "crisp_set_epilogue": [vp, vp, i32],
        "crisp_device_status": [vp, vp, P(i32)],
        "crisp_last_launch": [vp, P(LaunchInfo)],
        "crisp_last_resident_bytes": [vp, P(i64)],
        "crisp_set_tuning": [vp, i32, C.c_uint64, i32],
        "crisp_set_stage_blocks": [vp, i32],
        "crisp_reset_status": [vp, vp],
        "crisp_bytes_model": [vp, i64, i32, P(BytesModel)],
        "crisp_mask_scores": [P(LayerDesc), vp, P(vp), P(vp)],
        "crisp_global_rank_sizes": [i32, P(RankLayer), P(sz)],
        "crisp_prune_score": [i32, P(PruneLayer), vp],
        "crisp_prune_encode_sizes": [i32, P(PruneLayer), P(sz), P(sz)],
        "crisp_prune_encode": [i32, P(PruneLayer), vp, P(vp), P(vp)],
        "crisp_destroy_layers": [i32, P(vp), P(vp)],
        "crisp_global_rank": [i32, P(RankLayer), C.c_double, vp, vp, vp],
        "crisp_encode8_sizes": [vp, P(sz)],
        "crisp_encode8": [vp, i64, vp, vp, vp, P(vp)],
        "crisp_decode8": [vp, vp, i64, vp],
        "crisp_quantize8_sizes": [i64, i64, P(sz)],
        "crisp_quantize8": [vp, i64, i32, i64, i64, vp, vp],
        "crisp_dequantize8": [vp, i32, i64, i64, vp, i64, vp],
        "crisp_weight_grad8_sizes": [P(WeightGrad8), P(sz)],
        "crisp_weight_grad8": [P(WeightGrad8), vp, vp],
        "crisp_group_norm_sizes": [P(GroupNormDesc), i32, P(sz)],
        "crisp_group_norm": [P(GroupNormDesc), vp, i64, vp, vp, vp, i64, vp, vp, vp, vp, vp],
        "crisp_group_norm_backward": [P(GroupNormDesc), vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp, vp, vp],
        "crisp_spmm8_sizes": [vp, i64, P(sz)],
        "crisp_spmm8": [vp, vp, i64, i32, i64, vp, vp, i64, i32, i32, vp],
        "crisp_spmm8_quantized": [vp, vp, i64, vp, i64, i32, i32, vp],
        "crisp_set_epilogue8": [vp, vp, i32],
        "crisp_last_launch8": [vp, P(LaunchInfo)],
        "crisp_device_status8": [vp, vp, P(i32)],
        "crisp_reset_status8": [vp, vp],
        "crisp_set_tuning8": [vp, i32, i32, C.c_uint64, i32],
        "crisp_adamw": [i32, P(AdamwTensor), P(AdamwParams), vp],
        "crisp_adamw_moments": [vp, vp, vp, vp, i64, vp, vp, vp],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = C.c_int
    lib.crisp_mask_destroy.argtypes = [vp]
    lib.crisp_mask_destroy.restype = None
    lib.crisp_destroy.argtypes = [vp]
    lib.crisp_destroy.restype = None
    lib.crisp_destroy8.argtypes = [vp]
    lib.crisp_destroy8.restype = None
    lib.crisp_status_string.argtypes = [C.c_int]
    lib.crisp_status_string.restype = C.c_char_p
    try:
        from . import _calls as native
        native.bind(*[C.cast(getattr(lib, "crisp_" + name), vp).value for name in
                      ("spmm", "spmm_conv", "decode", "build_mask", "encode_sizes", "encode", "mask_destroy", "destroy")])
    except ImportError:
        native = _CtypesCalls(lib)
    _lib, _native = lib, native
    if _network:
        _bind_network()
    return lib


def crisp_status_string(code: int) -> str:
    return load().crisp_status_string(code).decode()


status_string = crisp_status_string


def _check(code: int, where: str):
    if code != OK:
        raise CrispError(code, where)


def _ptr(t) -> int:
    """Device (or host) address of a torch tensor / numpy array / int."""
    if t is None:
        return 0
    if isinstance(t, int):
        return t
    if hasattr(t, "data_ptr"):
        return t.data_ptr()
    return t.ctypes.data


def _bind_current_stream():
    """The address of torch's current stream on the current device.  torch.cuda.current_stream() builds a Stream object on
    every call, 3.2 us of the 9.6 us that a small product used to spend on the host; the two C functions it asks in the
    end take 0.2 us.  They are not public: without them the public call stays."""
    global _current_stream
    import torch
    torch.cuda.current_stream()                  # initialises CUDA, or says why it cannot
    device, raw = getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if device is not None and raw is not None:
        _current_stream = lambda: raw(device())
    else:
        _current_stream = lambda: torch.cuda.current_stream().cuda_stream
    return _current_stream()


_current_stream = _bind_current_stream


def _bind_current_device():
    """The current device, through the C function that torch.cuda.current_device() asks in the end (as _bind_current_stream has it for the stream)."""
    global _current_device
    import torch
    torch.cuda.current_device()                  # initialises CUDA
    _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _current_device()


_current_device = _bind_current_device


def _stream(stream) -> int:
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_desc(rows, k, n, m, block_rows, block_k, keep_ratio, score_mode=0) -> LayerDesc:
    return LayerDesc(rows, k, n, m, block_rows, block_k, float(keep_ratio), score_mode)


# ------------------------------------------------------------------ raw entry points

def crisp_keep_count(desc: LayerDesc):
    nblk, kkeep = C.c_int32(), C.c_int32()
    _check(load().crisp_keep_count(C.byref(desc), C.byref(nblk), C.byref(kkeep)), "crisp_keep_count")
    return nblk.value, kkeep.value


def crisp_mask_sizes(desc: LayerDesc):
    a, b = C.c_size_t(), C.c_size_t()
    _check(load().crisp_mask_sizes(C.byref(desc), C.byref(a), C.byref(b)), "crisp_mask_sizes")
    return a.value, b.value


def crisp_saliency_accumulate(d_grad, grad_dtype: int, ld_g: int, rows: int, k: int, d_acc, ld_acc: int, first: bool,
                              stream=None):
    _check(load().crisp_saliency_accumulate(_ptr(d_grad), grad_dtype, ld_g, rows, k, _ptr(d_acc), ld_acc,
                                            1 if first else 0, _stream(stream)), "crisp_saliency_accumulate")


def crisp_saliency_finish(d_acc, ld_acc: int, d_w, ld_w: int, rows: int, k: int, samples: int, d_saliency, ld_s: int,
                          stream=None):
    _check(load().crisp_saliency_finish(_ptr(d_acc), ld_acc, _ptr(d_w), ld_w, rows, k, samples, _ptr(d_saliency), ld_s,
                                        _stream(stream)), "crisp_saliency_finish")


def crisp_saliency_finish_max(d_acc, ld_acc: int, d_w, ld_w: int, rows: int, k: int, samples: int, d_saliency, ld_s: int,
                              d_mask_workspace, stream=None):
    _check(load().crisp_saliency_finish_max(_ptr(d_acc), ld_acc, _ptr(d_w), ld_w, rows, k, samples, _ptr(d_saliency),
                                            ld_s, _ptr(d_mask_workspace), _stream(stream)), "crisp_saliency_finish_max")


MASK_MAX_KNOWN = 1


def crisp_build_mask_ex(d_saliency, ld_s: int, desc: LayerDesc, d_mask_buf, d_workspace, flags: int, stream=None) -> int:
    out = C.c_void_p()
    _check(load().crisp_build_mask_ex(_ptr(d_saliency), ld_s, C.byref(desc), _ptr(d_mask_buf), _ptr(d_workspace),
                                      flags, _stream(stream), C.byref(out)), "crisp_build_mask_ex")
    return out.value


def crisp_mask_reselect(mask: int, kkeep: int, d_workspace, stream=None):
    _check(load().crisp_mask_reselect(mask, kkeep, _ptr(d_workspace), _stream(stream)), "crisp_mask_reselect")


def crisp_prune_fraction(kappa: float, n: int, m: int) -> float:
    out = C.c_double()
    _check(load().crisp_prune_fraction(float(kappa), n, m, C.byref(out)), "crisp_prune_fraction")
    return out.value


def crisp_keep_ratio_for_count(desc: LayerDesc, kkeep: int) -> float:
    out = C.c_double()
    _check(load().crisp_keep_ratio_for_count(C.byref(desc), kkeep, C.byref(out)), "crisp_keep_ratio_for_count")
    return out.value


def crisp_mask_scores(desc: LayerDesc, d_workspace):
    """-> (address of the [nrt, nblk] uint64 block scores, address of the max-key word) inside a workspace
    that crisp_build_mask has filled."""
    a, b = C.c_void_p(), C.c_void_p()
    _check(load().crisp_mask_scores(C.byref(desc), _ptr(d_workspace), C.byref(a), C.byref(b)), "crisp_mask_scores")
    return a.value, b.value


def make_rank_layers(layers):
    """layers: iterable of (d_scores, d_max_key, nrt, nblk, block_elems, min_keep) -> ctypes array."""
    layers = list(layers)
    arr = (RankLayer * len(layers))()
    for i, (sc, mk, nrt, nblk, be, keep) in enumerate(layers):
        arr[i] = RankLayer(_ptr(sc), _ptr(mk), nrt, nblk, be, keep, 0)
    return arr


def crisp_global_rank_sizes(rank_layers) -> int:
    out = C.c_size_t()
    _check(load().crisp_global_rank_sizes(len(rank_layers), rank_layers, C.byref(out)), "crisp_global_rank_sizes")
    return out.value


def crisp_global_rank(rank_layers, prune_fraction: float, d_workspace, d_kkeep, stream=None):
    _check(load().crisp_global_rank(len(rank_layers), rank_layers, float(prune_fraction), _ptr(d_workspace),
                                    _ptr(d_kkeep), _stream(stream)), "crisp_global_rank")


def crisp_prune_score(layers, stream=None):
    """layers: ctypes array of PruneLayer."""
    _check(load().crisp_prune_score(len(layers), layers, _stream(stream)), "crisp_prune_score")


def crisp_prune_encode_sizes(layers):
    """-> (canonical bytes, execution bytes) of every layer, for the kept counts in the array."""
    a, b = (C.c_size_t * len(layers))(), (C.c_size_t * len(layers))()
    _check(load().crisp_prune_encode_sizes(len(layers), layers, a, b), "crisp_prune_encode_sizes")
    return list(a), list(b)


def crisp_prune_encode(layers, stream=None):
    """-> (masks, handles)"""
    m, h = (C.c_void_p * len(layers))(), (C.c_void_p * len(layers))()
    _check(load().crisp_prune_encode(len(layers), layers, _stream(stream), m, h), "crisp_prune_encode")
    return list(m), list(h)


def crisp_adamw(tensors, params: AdamwParams, stream=None):
    """tensors: ctypes array of AdamwTensor."""
    _check(load().crisp_adamw(len(tensors), tensors, C.byref(params), _stream(stream)), "crisp_adamw")


def crisp_adamw_moments(d_m, d_m_exp, d_v, d_v_exp, count: int, d_m_bf16, d_root_bf16, stream=None):
    _check(load().crisp_adamw_moments(_ptr(d_m), _ptr(d_m_exp), _ptr(d_v), _ptr(d_v_exp), count, _ptr(d_m_bf16), _ptr(d_root_bf16),
                                      _stream(stream)), "crisp_adamw_moments")


def crisp_build_mask(d_saliency, ld_s: int, desc: LayerDesc, d_mask_buf, d_workspace, stream=None) -> int:
    out = C.c_void_p()
    _check(load().crisp_build_mask(_ptr(d_saliency), ld_s, C.byref(desc), _ptr(d_mask_buf), _ptr(d_workspace),
                                   _stream(stream), C.byref(out)), "crisp_build_mask")
    return out.value


STATIC_SCRATCH_BYTES = 256 * 1024


def crisp_build_mask_static(d_saliency, ld_s: int, desc: LayerDesc, d_mask_buf, stream=None) -> int:
    """crisp_build_mask without a caller-provided workspace: the scratch is a fixed array inside
    the library, for callers that may not allocate device memory.  Layers whose workspace exceeds
    STATIC_SCRATCH_BYTES raise CrispError(BUFFER_TOO_SMALL).  Calls share that array, so they must
    not overlap on the GPU."""
    out = C.c_void_p()
    _check(load().crisp_build_mask_static(_ptr(d_saliency), ld_s, C.byref(desc), _ptr(d_mask_buf),
                                          _stream(stream), C.byref(out)), "crisp_build_mask_static")
    return out.value


def crisp_mask_info(mask: int):
    d, a, b, c = LayerDesc(), C.c_int32(), C.c_int32(), C.c_int32()
    _check(load().crisp_mask_info(mask, C.byref(d), C.byref(a), C.byref(b), C.byref(c)), "crisp_mask_info")
    return d, a.value, b.value, c.value


def crisp_mask_export(mask: int, h_blk_col, h_nm_bits, stream=None):
    _check(load().crisp_mask_export(mask, _ptr(h_blk_col), _ptr(h_nm_bits), _stream(stream)), "crisp_mask_export")


def crisp_encode_sizes(mask: int):
    a, b = C.c_size_t(), C.c_size_t()
    _check(load().crisp_encode_sizes(mask, C.byref(a), C.byref(b)), "crisp_encode_sizes")
    return a.value, b.value


def crisp_encode(d_w, ld_w: int, mask: int, d_canonical, d_exec, stream=None) -> int:
    out = C.c_void_p()
    _check(load().crisp_encode(_ptr(d_w), ld_w, mask, _ptr(d_canonical), _ptr(d_exec), _stream(stream),
                               C.byref(out)), "crisp_encode")
    return out.value


def crisp_encoded_counts(handle: int):
    a, b, c = C.c_int64(), C.c_int64(), C.c_int64()
    _check(load().crisp_encoded_counts(handle, C.byref(a), C.byref(b), C.byref(c)), "crisp_encoded_counts")
    return a.value, b.value, c.value


def crisp_export(handle: int, h_blk_col, h_vals, h_idx, stream=None):
    _check(load().crisp_export(handle, _ptr(h_blk_col), _ptr(h_vals), _ptr(h_idx), _stream(stream)), "crisp_export")


def crisp_decode(handle: int, d_w_dense, ld: int, stream=None):
    _check(load().crisp_decode(handle, _ptr(d_w_dense), ld, _stream(stream)), "crisp_decode")


def crisp_spmm(handle: int, d_x, ldx: int, ncols: int, d_y, ldy: int, y_dtype: int = 0, stream=None):
    _check(load().crisp_spmm(handle, _ptr(d_x), ldx, ncols, _ptr(d_y), ldy, y_dtype, _stream(stream)), "crisp_spmm")


def crisp_spmm_conv(handle: int, d_act_nhwc, conv: ConvDesc, d_y, ldy: int, y_dtype: int = 0, stream=None):
    _check(load().crisp_spmm_conv(handle, _ptr(d_act_nhwc), C.byref(conv), _ptr(d_y), ldy, y_dtype, _stream(stream)),
           "crisp_spmm_conv")


def crisp_set_epilogue(handle: int, d_bias_f32, relu: int):
    _check(load().crisp_set_epilogue(handle, _ptr(d_bias_f32), int(relu)), "crisp_set_epilogue")


def crisp_set_path(handle: int, path: int):
    _check(load().crisp_set_path(handle, path), "crisp_set_path")


def crisp_device_status(handle: int, stream=None) -> int:
    s = C.c_int32()
    _check(load().crisp_device_status(handle, _stream(stream), C.byref(s)), "crisp_device_status")
    return s.value


def crisp_last_launch(handle: int) -> dict:
    """Kernel family (`path`) and tile configuration of the last product launched through the handle."""
    info = LaunchInfo()
    _check(load().crisp_last_launch(handle, C.byref(info)), "crisp_last_launch")
    return info.as_dict()


def crisp_last_resident_bytes(handle: int) -> int:
    """Bytes of weight tiles that the last product's CTAs kept in shared memory for all of their tiles."""
    out = C.c_int64()
    _check(load().crisp_last_resident_bytes(handle, C.byref(out)), "crisp_last_resident_bytes")
    return out.value


def crisp_set_tuning(handle: int, tile_boxes: int = 0, wait_limit_cycles: int = 0, skip_fill: int = -1):
    _check(load().crisp_set_tuning(handle, tile_boxes, wait_limit_cycles, skip_fill), "crisp_set_tuning")


def crisp_set_stage_blocks(handle: int, max_blocks: int = 0):
    """Most kept blocks one pipeline stage may take (1, 2, 4; 0 = chosen by the library)."""
    _check(load().crisp_set_stage_blocks(handle, max_blocks), "crisp_set_stage_blocks")


def crisp_reset_status(handle: int, stream=None):
    _check(load().crisp_reset_status(handle, _stream(stream)), "crisp_reset_status")


def crisp_bytes_model(handle: int, ncols: int, y_dtype: int = 0) -> dict:
    b = BytesModel()
    _check(load().crisp_bytes_model(handle, ncols, y_dtype, C.byref(b)), "crisp_bytes_model")
    return b.as_dict()


def crisp_destroy_layers(masks, handles):
    """masks, handles: ctypes arrays of c_void_p of one length (nulls are skipped)."""
    _check(load().crisp_destroy_layers(len(masks), masks, handles), "crisp_destroy_layers")


def crisp_mask_destroy(mask: int):
    if mask:
        load().crisp_mask_destroy(mask)


def crisp_destroy(handle: int):
    if handle:
        load().crisp_destroy(handle)


# ------------------------------------------------------------------ the 8-bit product

def crisp_encode8_sizes(mask: int) -> int:
    out = C.c_size_t()
    _check(load().crisp_encode8_sizes(mask, C.byref(out)), "crisp_encode8_sizes")
    return out.value


def crisp_encode8(d_w, ld_w: int, mask: int, d_buf, stream=None) -> int:
    out = C.c_void_p()
    _check(load().crisp_encode8(_ptr(d_w), ld_w, mask, _ptr(d_buf), _stream(stream), C.byref(out)), "crisp_encode8")
    return out.value


def crisp_decode8(handle8: int, d_w_dense, ld: int, stream=None):
    _check(load().crisp_decode8(handle8, _ptr(d_w_dense), ld, _stream(stream)), "crisp_decode8")


def crisp_quantize8_sizes(k: int, ncols: int) -> int:
    out = C.c_size_t()
    _check(load().crisp_quantize8_sizes(k, ncols, C.byref(out)), "crisp_quantize8_sizes")
    return out.value


def crisp_quantize8(d_x, ldx: int, x_layout: int, k: int, ncols: int, d_act, stream=None):
    _check(load().crisp_quantize8(_ptr(d_x), ldx, x_layout, k, ncols, _ptr(d_act), _stream(stream)), "crisp_quantize8")


def crisp_dequantize8(d_act, y_layout: int, k: int, ncols: int, d_y, ldy: int, stream=None):
    _check(load().crisp_dequantize8(_ptr(d_act), y_layout, k, ncols, _ptr(d_y), ldy, _stream(stream)), "crisp_dequantize8")


def crisp_weight_grad8_sizes(grad: WeightGrad8) -> int:
    out = C.c_size_t()
    _check(load().crisp_weight_grad8_sizes(C.byref(grad), C.byref(out)), "crisp_weight_grad8_sizes")
    return out.value


def crisp_weight_grad8(grad: WeightGrad8, d_workspace, stream=None):
    _check(load().crisp_weight_grad8(C.byref(grad), _ptr(d_workspace), _stream(stream)), "crisp_weight_grad8")


def crisp_group_norm_sizes(desc: GroupNormDesc, backward: bool) -> int:
    out = C.c_size_t()
    _check(load().crisp_group_norm_sizes(C.byref(desc), int(backward), C.byref(out)), "crisp_group_norm_sizes")
    return out.value


def crisp_group_norm(desc: GroupNormDesc, d_x, ldx: int, d_gamma, d_beta, d_y, ldy: int, d_stats, d_x8, d_y8, d_workspace, stream=None):
    _check(load().crisp_group_norm(C.byref(desc), _ptr(d_x), ldx, _ptr(d_gamma), _ptr(d_beta), _ptr(d_y), ldy, _ptr(d_stats), _ptr(d_x8), _ptr(d_y8),
                                   _ptr(d_workspace), _stream(stream)), "crisp_group_norm")


def crisp_group_norm_backward(desc: GroupNormDesc, d_dy, ld_dy: int, d_x, ldx: int, d_x8, d_stats, d_gamma, d_beta, d_dx, ld_dx: int, d_dgamma, d_dbeta,
                              d_workspace, stream=None):
    _check(load().crisp_group_norm_backward(C.byref(desc), _ptr(d_dy), ld_dy, _ptr(d_x), ldx, _ptr(d_x8), _ptr(d_stats), _ptr(d_gamma), _ptr(d_beta),
                                            _ptr(d_dx), ld_dx, _ptr(d_dgamma), _ptr(d_dbeta), _ptr(d_workspace), _stream(stream)),
           "crisp_group_norm_backward")


def crisp_spmm8_sizes(handle8: int, ncols: int) -> int:
    out = C.c_size_t()
    _check(load().crisp_spmm8_sizes(handle8, ncols, C.byref(out)), "crisp_spmm8_sizes")
    return out.value


def crisp_spmm8(handle8: int, d_x, ldx: int, x_layout: int, ncols: int, d_act, d_y, ldy: int, y_layout: int, y_dtype: int = 0, stream=None):
    _check(load().crisp_spmm8(handle8, _ptr(d_x), ldx, x_layout, ncols, _ptr(d_act), _ptr(d_y), ldy, y_layout, y_dtype, _stream(stream)),
           "crisp_spmm8")


def crisp_spmm8_quantized(handle8: int, d_act, ncols: int, d_y, ldy: int, y_layout: int, y_dtype: int = 0, stream=None):
    _check(load().crisp_spmm8_quantized(handle8, _ptr(d_act), ncols, _ptr(d_y), ldy, y_layout, y_dtype, _stream(stream)), "crisp_spmm8_quantized")


def crisp_set_epilogue8(handle8: int, d_bias_f32, relu: int):
    _check(load().crisp_set_epilogue8(handle8, _ptr(d_bias_f32), int(relu)), "crisp_set_epilogue8")


def crisp_last_launch8(handle8: int) -> dict:
    """Tile, grid and stages of the last 8-bit product through the handle; `stack`: CTAs that shared one tile's blocks."""
    info = LaunchInfo()
    _check(load().crisp_last_launch8(handle8, C.byref(info)), "crisp_last_launch8")
    return info.as_dict()


def crisp_device_status8(handle8: int, stream=None) -> int:
    s = C.c_int32()
    _check(load().crisp_device_status8(handle8, _stream(stream), C.byref(s)), "crisp_device_status8")
    return s.value


def crisp_reset_status8(handle8: int, stream=None):
    _check(load().crisp_reset_status8(handle8, _stream(stream)), "crisp_reset_status8")


def crisp_set_tuning8(handle8: int, tile_cols: int = 0, split: int = 0, wait_limit_cycles: int = 0, skip_fill: int = -1):
    _check(load().crisp_set_tuning8(handle8, tile_cols, split, wait_limit_cycles, skip_fill), "crisp_set_tuning8")


def crisp_destroy8(handle8: int):
    if handle8:
        load().crisp_destroy8(handle8)


_AS_IT_IS = contextlib.nullcontext()


def _allocating_for(stream):
    """A context in which the stream of a call is the current one, so that torch allocates memory for it (None: the current one as it is; a torch stream or an
    address, 0 for the default stream)."""
    if stream is None:
        return _AS_IT_IS
    import torch
    if isinstance(stream, int):                          # (ExternalStream(0) would be a stream out of torch's pool)
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


def _pitch(t) -> int:
    """Elements from one row of a matrix to the next (torch gives a single row any stride)."""
    return t.stride()[0] if t.shape[0] > 1 else t.shape[1]


def _on(device):
    """A context in which `device` is the current one."""
    if device.index == _current_device():
        return _AS_IT_IS
    import torch
    return torch.cuda.device(device)


def _pixel_pitch(t, what) -> int:
    """Elements from one pixel of a channels-last tensor to the next."""
    shape, strides = t.shape, t.stride()
    assert strides[-1] == 1 or shape[-1] == 1, f"the channels of {what} are not consecutive"
    pitch, count = None, 1                                                   # of the innermost dimension that has one; pixels inside the present one
    for size, stride in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if size == 1:
            continue
        if pitch is None:
            pitch = stride
        assert stride == pitch * count, f"the pixels of {what} do not lie one pitch apart"
        count *= size
    return shape[-1] if pitch is None else pitch


class Activations8:
    """Activations in 8 bits (quantize8, GroupNorm.forward): a buffer of the library's form.  Layers of the same k multiply it (HybridLayer.spmm8), and it is the
    checkpoint that a layer's weight gradient and a norm's backward pass take."""

    def __init__(self, k, ncols, buffer):
        self.k, self.ncols, self.buffer = k, ncols, buffer

    def dequantize(self, tokens=False, y=None, stream=None):
        """The bf16 values that it stands for: [k, ncols], or with tokens=True [ncols, k]."""
        import torch
        shape, device = (self.ncols, self.k) if tokens else (self.k, self.ncols), self.buffer.device
        with _on(device):
            if y is None:
                with _allocating_for(stream):
                    y = torch.empty_strided(shape, (shape[1], 1), dtype=torch.bfloat16, device=device)
            else:
                assert y.device == device and y.dtype == torch.bfloat16 and y.shape == shape and (y.stride()[1] == 1 or shape[1] == 1), \
                    "Y is a bf16 matrix of the activations' shape on their device, with consecutive elements in a row"
            crisp_dequantize8(self.buffer, int(tokens), self.k, self.ncols, y, _pitch(y), stream)
        return y


def quantize8(x, tokens=False, stream=None):
    """X in 8 bits, for any layer of its k: x is a bf16 CUDA matrix [k, ncols], or with tokens=True [ncols, k] (NHWC activations: x.view(-1, channels))."""
    import torch
    assert x.is_cuda and x.dtype == torch.bfloat16 and len(x.shape) == 2 and (x.stride()[1] == 1 or x.shape[1] == 1), \
        "X is a bf16 CUDA matrix, [k, ncols] or with tokens=True [ncols, k], with consecutive elements in a row"
    ncols, k = x.shape if tokens else reversed(x.shape)
    with _on(x.device):
        act = _buffer8(k, ncols, x.device, stream)
        crisp_quantize8(x, _pitch(x), int(tokens), k, ncols, act.buffer, stream)
    return act


def _buffer8(k, ncols, device, stream):
    import torch
    with _allocating_for(stream):
        return Activations8(k, ncols, torch.empty_strided((crisp_quantize8_sizes(k, ncols),), (1,), dtype=torch.uint8, device=device))


_status_words = {}                                        # by device: words of a block that no layer has yet


def _status_word(device):
    """A zeroed word in the device's memory, a layer's own, out of a block of 64: one that each layer allocates and clears is half of the time in which it is made (8.6 and 17.6 us)."""
    try:
        return _status_words[device].pop()
    except (KeyError, IndexError):
        import torch
        words = list(torch.zeros(64, dtype=torch.int32, device=device).split(1))
        word = words.pop()
        if device.type != "cuda" or not torch.cuda.is_current_stream_capturing():    # (a block that is made in a capture is zeros once that is replayed: for this layer alone)
            _status_words[device] = words
        return word


# -------------------------------------------------- buffer-owning convenience wrapper

class HybridLayer:
    """Owns the device buffers of one pruned layer and forwards to the C ABI.

    ``build_mask`` -> ``encode`` -> ``spmm`` mirror crisp_build_mask / crisp_encode /
    crisp_spmm; tensors are torch CUDA tensors (bf16 tensors or their int16/uint16 views).
    """

    def __init__(self, rows, k, n, m, block_rows, block_k, keep_ratio, score_mode=0, device="cuda"):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        self.desc = make_desc(rows, k, n, m, block_rows, block_k, keep_ratio, score_mode)
        self.nblk, self.kkeep = crisp_keep_count(self.desc)
        self.nrt = (rows + block_rows - 1) // block_rows
        mask_bytes, ws_bytes = crisp_mask_sizes(self.desc)
        self.mask_buf = torch.empty(mask_bytes, dtype=torch.uint8, device=self.device)
        self.workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=self.device)
        self.device = self.mask_buf.device                   # with its index: results lie beside the buffers, whatever device is current by then
        self.mask = 0
        self.handle = 0
        self.handle8 = 0
        self.buf8 = None
        self._bias8 = None
        self._grad_status = _status_word(self.device)
        self.canonical_buf = None
        self.exec_buf = None
        self._gpu = self.device.index if (_network or _bind_network()) else None       # (decode makes its tensors through it)

    # build_mask, encode, decode, spmm and spmm_conv are made once per layer and pass; for small layers their host time is the
    # time of the pass, so they hand plain integers to the library (and ask a tensor for all its strides at once, which is cheaper
    # than for one).
    def build_mask(self, saliency, stream=None):
        strides = saliency.stride()
        assert saliency.is_cuda and saliency.dtype == self.torch.float32 and strides[1] == 1
        old, self.mask = self.mask, 0
        code, self.mask = _native.build_mask(saliency.data_ptr(), strides[0], C.addressof(self.desc), self.mask_buf.data_ptr(),
                                             self.workspace.data_ptr(), _stream(stream), old)
        if code:
            raise CrispError(code, "crisp_build_mask")
        return self

    def rank_layer(self, min_keep=0):
        """This layer's entry for crisp_global_rank (valid after build_mask, until the workspace is reused)."""
        sc, mk = crisp_mask_scores(self.desc, self.workspace)
        return (sc, mk, self.nrt, self.nblk, self.desc.block_rows * self.desc.block_k, min_keep)

    def set_kkeep(self, kkeep: int):
        """Keep ratio that makes the next build_mask keep exactly `kkeep` blocks per row tile."""
        self.desc.keep_ratio = crisp_keep_ratio_for_count(self.desc, kkeep)
        self.nblk, self.kkeep = crisp_keep_count(self.desc)
        assert self.kkeep == kkeep
        mask_bytes, ws_bytes = crisp_mask_sizes(self.desc)
        if self.mask_buf.numel() < mask_bytes:
            self.mask_buf = self.torch.empty(mask_bytes, dtype=self.torch.uint8, device=self.device)
        return self

    def build_mask_max_known(self, saliency, stream=None):
        """build_mask when the workspace already holds the layer maximum (crisp_saliency_finish_max wrote it)."""
        assert saliency.is_cuda and saliency.dtype == self.torch.float32 and saliency.stride(1) == 1
        crisp_mask_destroy(self.mask)
        self.mask = crisp_build_mask_ex(saliency, saliency.stride(0), self.desc, self.mask_buf, self.workspace,
                                        MASK_MAX_KNOWN, stream)
        return self

    def reselect(self, kkeep: int, stream=None):
        """Keep only the `kkeep` best blocks per row tile of the mask just built (no pass over the saliency)."""
        crisp_mask_reselect(self.mask, kkeep, self.workspace, stream)
        self.desc.keep_ratio = crisp_keep_ratio_for_count(self.desc, kkeep)
        self.kkeep = kkeep
        return self

    def export_mask(self, stream=None):
        import numpy as np
        wpr = self.nblk * self.desc.block_k // 32
        blk_col = np.zeros((self.nrt, self.kkeep), dtype=np.int32)
        nm_bits = np.zeros((self.nrt * self.desc.block_rows, wpr), dtype=np.uint32)
        crisp_mask_export(self.mask, blk_col, nm_bits, stream)
        return blk_col, nm_bits

    def encode(self, w, stream=None):
        strides = w.stride()
        assert w.is_cuda and w.element_size() == 2 and strides[1] == 1
        code, canonical_bytes, exec_bytes = _native.encode_sizes(self.mask)
        if code:
            raise CrispError(code, "crisp_encode_sizes")
        self._reserve(canonical_bytes, exec_bytes, stream)
        old, self.handle = self.handle, 0
        code, self.handle = _native.encode(w.data_ptr(), strides[0], self.mask, self.canonical_buf.data_ptr(), self.exec_buf.data_ptr(),
                                           _stream(stream), old)
        if code:
            raise CrispError(code, "crisp_encode")
        return self

    def _reserve(self, canonical_bytes, exec_bytes, stream=None):
        if self.canonical_buf is None or self.canonical_buf.numel() < canonical_bytes:
            with _allocating_for(stream):
                self.canonical_buf = self.torch.empty(canonical_bytes, dtype=self.torch.uint8, device=self.device)
        if self.exec_buf is None or self.exec_buf.numel() < exec_bytes:
            with _allocating_for(stream):
                self.exec_buf = self.torch.empty(exec_bytes, dtype=self.torch.uint8, device=self.device)

    def export(self, stream=None):
        import numpy as np
        nb, nv, nw = crisp_encoded_counts(self.handle)
        blk_col = np.zeros(nb, dtype=np.int32)
        vals = np.zeros(nv, dtype=np.uint16)
        idx = np.zeros(nw, dtype=np.uint32)
        crisp_export(self.handle, blk_col, vals, idx, stream)
        return blk_col.reshape(self.nrt, self.kkeep), vals, idx

    # (of the calls in Python empty_strided is the cheapest that allocates: 1.1 us against 3.2 for new_empty and 4.2 for empty)
    def decode(self, stream=None):
        desc, torch = self.desc, self.torch
        k = desc.k
        if stream is not None:
            with self._on_device(), _allocating_for(stream):
                return self.decode()
        if self._gpu is not None:
            code, w = _network.decode(self.handle, desc.rows, k, self._gpu, _current_stream())
            if code:
                raise CrispError(code, "crisp_decode")
            return w
        w = torch.empty_strided((desc.rows, k), (k, 1), dtype=torch.bfloat16, device=self.device)
        code = _native.decode(self.handle, w.data_ptr(), k, _current_stream())
        if code:
            raise CrispError(code, "crisp_decode")
        return w

    def spmm(self, x, y=None, y_dtype=0, stream=None):
        shape, strides = x.shape, x.stride()
        assert x.is_cuda and x.element_size() == 2 and strides[1] == 1 and shape[0] == self.desc.k
        ncols = shape[1]
        if y is None:
            if stream is not None:
                with self._on_device(), _allocating_for(stream):
                    return self.spmm(x, None, y_dtype)
            y = self.torch.empty_strided((self.desc.rows, ncols), (ncols, 1), device=self.device,
                                         dtype=self.torch.float32 if y_dtype else self.torch.bfloat16)
        code = _native.spmm(self.handle, x.data_ptr(), strides[0], ncols, y.data_ptr(), y.stride()[0], y_dtype, _stream(stream))
        if code:
            raise CrispError(code, "crisp_spmm")
        return y

    def spmm_conv(self, act_nhwc, kernel_h, kernel_w, pad, y=None, y_dtype=0, stream=None, nhwc_out=False):
        """Convolution (stride 1) of an NHWC bf16 activation with this layer's weights, without an X matrix.
        nhwc_out: Y is [batch, ho, wo, rows] (the next convolution's activation) instead of [rows, batch*ho*wo]."""
        assert act_nhwc.is_cuda and act_nhwc.element_size() == 2 and act_nhwc.is_contiguous() and act_nhwc.dim() == 4
        b, h, w, c = act_nhwc.shape
        if y is None:
            ho, wo = h + 2 * pad - kernel_h + 1, w + 2 * pad - kernel_w + 1
            dt = self.torch.float32 if y_dtype else self.torch.bfloat16
            with _allocating_for(stream):
                y = self.torch.empty((b, ho, wo, self.desc.rows) if nhwc_out else (self.desc.rows, b * ho * wo), dtype=dt, device=self.device)
        ldy = y.stride()[2 if nhwc_out else 0]
        code = _native.spmm_conv(self.handle, act_nhwc.data_ptr(), b, h, w, c, kernel_h, kernel_w, pad, 1 if nhwc_out else 0,
                                 y.data_ptr(), ldy, y_dtype, _stream(stream))
        if code:
            raise CrispError(code, "crisp_spmm_conv")
        return y

    def set_epilogue(self, bias=None, relu=False):
        """Y = act(W X + bias) for later products; `bias` is an fp32 CUDA tensor [rows] that this object keeps."""
        if bias is not None:
            assert bias.device == self.device and bias.dtype == self.torch.float32 and bias.numel() == self.desc.rows and bias.is_contiguous(), \
                "a bias is an fp32 tensor of as many consecutive elements as the layer has rows, on its device"
        self._bias = bias
        crisp_set_epilogue(self.handle, bias, 1 if relu else 0)
        return self

    def set_path(self, path: int):
        crisp_set_path(self.handle, path)

    def _on_device(self):
        """A context in which the layer's device is the current one."""
        return _AS_IT_IS if self.device.index == _current_device() else self.torch.cuda.device(self.device)

    # The layer in 8 bits, beside or instead of its bf16 encoding (masks of 128 x 128 blocks).
    def encode8(self, w, stream=None):
        """Compress the weights under the mask to e4m3 with a scale for each kept block (crisp_encode8).  The epilogue of an encoding before is not carried over."""
        if self._gpu is not None and self._gpu == _current_device():
            done = _network.encode8(self.mask, w, self.desc.rows, self.desc.k, self._gpu, self.buf8, self.handle8, _stream(stream))
            if done is not None and not done[2]:
                code, handle, _ = done
                if not (code and handle):                    # (refused before anything was done, the encoding before stays, and its epilogue with it)
                    self.handle8, self._bias8 = handle, None
                if code:
                    raise CrispError(code, "crisp_encode8")
                return self
        assert w.is_cuda and w.dtype == self.torch.bfloat16 and (w.stride()[1] == 1 or w.shape[1] == 1) and w.shape == (self.desc.rows, self.desc.k), \
            "weights are a bf16 CUDA matrix of the layer's shape with consecutive columns"
        assert w.device == self.device, "weights on another device than the layer"
        size = crisp_encode8_sizes(self.mask)
        with self._on_device():
            if self.buf8 is None or self.buf8.numel() < size:
                with _allocating_for(stream):
                    self.buf8 = self.torch.empty(size, dtype=self.torch.uint8, device=self.device)
            old, self.handle8 = self.handle8, 0
            crisp_destroy8(old)
            self._bias8 = None
            self.handle8 = crisp_encode8(w, _pitch(w), self.mask, self.buf8, stream)
        return self

    def decode8(self, stream=None):
        """The dense bf16 weights that the 8-bit encoding stands for."""
        if stream is not None:
            with self._on_device(), _allocating_for(stream):
                return self.decode8()
        if self._gpu is not None and self._gpu == _current_device():
            code, w = _network.decode8(self.handle8, self.desc.rows, self.desc.k, self._gpu, _current_stream())
            if code:
                raise CrispError(code, "crisp_decode8")
            return w
        with self._on_device():
            w = self.torch.empty_strided((self.desc.rows, self.desc.k), (self.desc.k, 1), dtype=self.torch.bfloat16, device=self.device)
            crisp_decode8(self.handle8, w, self.desc.k)
        return w

    def quantize8(self, x, tokens=False, stream=None):
        """X in 8 bits, for this layer and others of its k: x is [k, ncols], or with tokens=True [ncols, k]."""
        ncols = self._columns8(x, tokens)
        k = self.desc.k
        with self._on_device():
            with _allocating_for(stream):
                act = self.torch.empty_strided((crisp_quantize8_sizes(k, ncols),), (1,), dtype=self.torch.uint8, device=self.device)
            crisp_quantize8(x, _pitch(x), int(tokens), k, ncols, act, stream)
        return Activations8(k, ncols, act)

    def _columns8(self, x, tokens):
        shape = x.shape
        assert x.device == self.device and x.dtype == self.torch.bfloat16 and len(shape) == 2 and (x.stride()[1] == 1 or shape[1] == 1) and shape[1 if tokens else 0] == self.desc.k, \
            "X is a bf16 CUDA matrix, [k, ncols] or with tokens=True [ncols, k], with consecutive elements in a row"
        return shape[0 if tokens else 1]

    def spmm8(self, x, y=None, y_dtype=0, tokens=False, stream=None):
        """act(W X + bias) in 8 bits.  x: [k, ncols] -> Y [rows, ncols]; with tokens=True [ncols, k] -> Y [ncols, rows]; or what quantize8 returned, with tokens for
        the layout of Y."""
        torch, rows, k = self.torch, self.desc.rows, self.desc.k
        if y is None and stream is None and self._gpu is not None and type(x) is torch.Tensor and self._gpu == _current_device():
            done = _network.product8(self.handle8, x, rows, k, self._gpu, tokens, y_dtype, _current_stream())
            if done is not None:
                if done[0]:
                    raise CrispError(done[0], "crisp_spmm8")
                return done[1]
        if y is None and stream is not None:
            with self._on_device(), _allocating_for(stream):
                return self.spmm8(x, None, y_dtype, tokens)
        held = isinstance(x, Activations8)
        ncols = x.ncols if held else self._columns8(x, tokens)
        assert not held or (x.k == k and x.buffer.device == self.device), "activations of another k or on another device"
        shape = (ncols, rows) if tokens else (rows, ncols)
        dtype = torch.float32 if y_dtype else torch.bfloat16
        if y is None:
            y = torch.empty_strided(shape, (shape[1], 1), dtype=dtype, device=self.device)
        else:
            assert y.device == self.device and y.dtype == dtype and y.shape == shape and (y.stride()[1] == 1 or shape[1] == 1), \
                "Y has the product's shape and type, and consecutive elements in a row"
        with self._on_device():
            if held:
                crisp_spmm8_quantized(self.handle8, x.buffer, ncols, y, _pitch(y), int(tokens), y_dtype, stream)
                return y
            with _allocating_for(stream):                    # the workspace is given back when this returns: to the stream that uses it
                act = torch.empty_strided((crisp_spmm8_sizes(self.handle8, ncols),), (1,), dtype=torch.uint8, device=self.device)
            crisp_spmm8(self.handle8, x, _pitch(x), int(tokens), ncols, act, y, _pitch(y), int(tokens), y_dtype, stream)
        return y

    def weight_gradient8(self, dy, act, dw=None, dw_dtype=1, tokens=False, masked=False, accumulate=False, stream=None):
        """dW = dY X^T [rows, k] from the activations that quantize8 (or a GroupNorm) kept in 8 bits.  dy: bf16 [rows, ncols], or with tokens=True [ncols, rows].
        masked: 0 outside the layer's mask, and blocks that are not kept are not computed (what AdamW takes under the mask); else every weight's gradient, as a
        saliency takes it.  dw: where to write it, bf16 (dw_dtype 0) or fp32 (1); accumulate: to add it there.  gradient_status says whether a wait ran out."""
        if dw is None and stream is None and not accumulate and self._gpu is not None and self._gpu == _current_device() and (self.mask or not masked):
            done = _network.gradient8(dy, act.buffer, self._grad_status, self.mask if masked else 0, self.desc.rows, self.desc.k, act.k, act.ncols, 0, 0, 0, tokens, dw_dtype,
                                      self._gpu, _current_stream())
            if done is not None:
                if done[0]:
                    raise CrispError(done[0], "crisp_weight_grad8")
                return done[1]
        shape = (act.ncols, self.desc.rows) if tokens else (self.desc.rows, act.ncols)
        assert act.k == self.desc.k, "activations of another k"
        assert dy.shape == shape, "dY is [rows, ncols], or with tokens=True [ncols, rows], with the activations' columns"
        return self._gradient8(dy, _pitch(dy), act, act.ncols, None, tokens, dw, dw_dtype, masked, accumulate, stream)

    def weight_gradient8_conv(self, dy_nhwc, act, kernel_h, kernel_w, pad, dw=None, dw_dtype=1, masked=False, accumulate=False, stream=None):
        """The same of a convolution (stride 1).  dy_nhwc: bf16 [batch, ho, wo, rows], dense but for the pitch of a pixel; act: the 8-bit form of the NHWC activation
        [batch, ho + kernel_h - 1 - 2 pad, wo + kernel_w - 1 - 2 pad, channels] (quantize8(x.view(-1, channels), tokens=True))."""
        if dw is None and stream is None and not accumulate and kernel_h > 0 and self._gpu is not None and self._gpu == _current_device() and (self.mask or not masked):
            done = _network.gradient8(dy_nhwc, act.buffer, self._grad_status, self.mask if masked else 0, self.desc.rows, self.desc.k, act.k, act.ncols, kernel_h, kernel_w,
                                      pad, True, dw_dtype, self._gpu, _current_stream())
            if done is not None:
                if done[0]:
                    raise CrispError(done[0], "crisp_weight_grad8")
                return done[1]
        batch, ho, wo, rows = dy_nhwc.shape
        height, width = ho + kernel_h - 1 - 2 * pad, wo + kernel_w - 1 - 2 * pad
        assert rows == self.desc.rows and act.k * kernel_h * kernel_w == self.desc.k and act.ncols == batch * height * width and min(height, width) > 0, \
            "dY, activations and kernel are not those of one convolution of the layer"
        pitch = _pixel_pitch(dy_nhwc, "dY")
        return self._gradient8(dy_nhwc, pitch, act, batch * ho * wo, ConvDesc(batch, height, width, act.k, kernel_h, kernel_w, pad, 1), True, dw, dw_dtype, masked,
                               accumulate, stream)

    def _gradient8(self, dy, ld, act, ncols, conv, tokens, dw, dw_dtype, masked, accumulate, stream):
        torch, rows, k = self.torch, self.desc.rows, self.desc.k
        dtype = torch.float32 if dw_dtype else torch.bfloat16
        assert dy.device == self.device and dy.dtype == torch.bfloat16 and (dy.stride()[-1] == 1 or dy.shape[-1] == 1), \
            "dY is a bf16 tensor on the layer's device with consecutive elements in a row"
        assert act.buffer.device == self.device, "activations on another device than the layer"
        assert not masked or self.mask, "the layer has no mask yet"
        assert not accumulate or dw is not None, "there is nothing to add to"
        assert dw is None or (dw.device == self.device and dw.dtype == dtype and dw.shape == (rows, k) and (dw.stride()[1] == 1 or k == 1)), \
            "dW has the weights' shape and the type asked for, on the layer's device, and consecutive elements in a row"
        with self._on_device():
            with _allocating_for(stream):
                if dw is None:
                    dw = torch.empty_strided((rows, k), (k, 1), dtype=dtype, device=self.device)
                g = WeightGrad8(rows, k, ncols, C.pointer(conv) if conv is not None else None, _ptr(dy), ld, int(tokens), int(bool(dw_dtype)), _ptr(act.buffer),
                                self.mask if masked else None, _ptr(dw), _pitch(dw), int(accumulate), 0, _ptr(self._grad_status))
                size = crisp_weight_grad8_sizes(g)                           # (given back when the call returns: to the stream that uses it)
                workspace = torch.empty_strided((size,), (1,), dtype=torch.uint8, device=self.device) if size else None
            crisp_weight_grad8(g, workspace, stream)
        return dw

    def gradient_status(self) -> int:
        """0, or TIMEOUT where a wait within a weight gradient has run out since reset_gradient_status was last called (that one's dW is not to be used).  Waits for
        all that runs on the device."""
        self.torch.cuda.synchronize(self.device)
        return int(self._grad_status.item())

    def reset_gradient_status(self, stream=None):
        """gradient_status says 0 again, of the gradients that come behind this call on the stream."""
        with self._on_device(), _allocating_for(stream):
            self._grad_status.zero_()

    def set_epilogue8(self, bias=None, relu=False):
        """Y = act(W X + bias) for later 8-bit products; `bias` is an fp32 CUDA tensor [rows] that this object keeps."""
        if bias is not None:
            assert bias.device == self.device and bias.dtype == self.torch.float32 and bias.numel() == self.desc.rows and bias.is_contiguous(), \
                "a bias is an fp32 tensor of as many consecutive elements as the layer has rows, on its device"
        self._bias8 = bias
        crisp_set_epilogue8(self.handle8, bias, 1 if relu else 0)
        return self

    def device_status8(self, stream=None) -> int:
        return crisp_device_status8(self.handle8, stream)

    def last_launch8(self) -> dict:
        return crisp_last_launch8(self.handle8)

    def set_tuning8(self, tile_cols=0, split=0, wait_limit_cycles=0, skip_fill=-1):
        crisp_set_tuning8(self.handle8, tile_cols, split, wait_limit_cycles, skip_fill)
        return self

    def reset_status8(self, stream=None):
        crisp_reset_status8(self.handle8, stream)

    def device_status(self, stream=None) -> int:
        return crisp_device_status(self.handle, stream)

    def last_launch(self) -> dict:
        return crisp_last_launch(self.handle)

    def last_resident_bytes(self) -> int:
        return crisp_last_resident_bytes(self.handle)

    def set_tuning(self, tile_boxes=0, wait_limit_cycles=0, skip_fill=-1):
        crisp_set_tuning(self.handle, tile_boxes, wait_limit_cycles, skip_fill)
        return self

    def set_stage_blocks(self, max_blocks=0):
        crisp_set_stage_blocks(self.handle, max_blocks)
        return self

    def reset_status(self, stream=None):
        crisp_reset_status(self.handle, stream)

    def bytes_model(self, ncols, y_dtype=0):
        return crisp_bytes_model(self.handle, ncols, y_dtype)

    def close(self):
        crisp_destroy(self.handle)
        crisp_destroy8(self.handle8)
        crisp_mask_destroy(self.mask)
        self.handle = self.handle8 = 0
        self.mask = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _holds_rows(t, rows, k):
    """Whether `rows` rows of k elements lie at the tensor's address, its first stride apart: a matrix of at least that size whose columns are
    consecutive, or more dimensions where those behind the first are dense in any order (a convolution's weights, channels last or not)."""
    shape, strides = t.shape, t.stride()
    if not shape or shape[0] < rows or 0 in shape:
        return False
    run = 1
    for step, size in sorted((step, size) for step, size in zip(strides[1:], shape[1:]) if size != 1):
        if step != run:
            return k == 1
        run *= size
    return run >= k


class PruningNetwork:
    """One pruning iteration of Algorithm 1 over all layers of a network, without the fine-tuning that follows it:

        network     saliency of Eq. 1 from the caller's gradients, N:M step, block scores   crisp_prune_score
        network     rank-column sums, global order, selection                              crisp_global_rank
        network     keep the selected number of blocks per layer, compress                 crisp_prune_encode

    This class only owns buffers and issues those calls in that order; every number is computed by the library.
    `shapes` is a list of (rows, k); the pattern (n:m, block shape) is shared by the layers.
    """

    def __init__(self, shapes, n, m, block_rows, block_k, min_keep=1, device="cuda"):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        self.n, self.m = n, m
        self.min_keep = min_keep
        self.layers = [HybridLayer(r, k, n, m, block_rows, block_k, 1.0, device=device) for (r, k) in shapes]
        self.sal = [torch.empty((r, k), dtype=torch.float32, device=self.device) for (r, k) in shapes]
        self._acc = None
        self.rank_arr = make_rank_layers([L.rank_layer(min_keep) for L in self.layers])
        self.rank_ws = torch.empty(crisp_global_rank_sizes(self.rank_arr), dtype=torch.uint8, device=self.device)
        self.d_kkeep = torch.zeros(len(shapes), dtype=torch.int32, device=self.device)
        self._h_kkeep = torch.zeros(len(shapes), dtype=torch.int32, pin_memory=True)
        self._blocks = (C.c_int32 * len(shapes))(*[L.nblk for L in self.layers])

    @property
    def acc(self):
        """The running gradient sums of layers whose gradients come in turn (allocated when first used)."""
        if self._acc is None:
            self._acc = [self.torch.empty_like(s) for s in self.sal]
        return self._acc

    def _score_in_turn(self, weights, grads, stream):
        """crisp_prune_score in the calls it replaces, one gradient tensor at a time; the number of layers."""
        count = 0
        for L, w, gs, acc, s in zip(self.layers, weights, grads, self.acc, self.sal):
            rows, k = L.desc.rows, L.desc.k
            for i, g in enumerate(gs):
                self._check_gradient(g, L)
                crisp_saliency_accumulate(g, 0 if g.dtype == self.torch.bfloat16 else 1, g.stride(0), rows, k, acc, k, i == 0,
                                          stream)
            crisp_saliency_finish_max(acc, k, w, w.stride(0), rows, k, len(gs), s, k, L.workspace, stream)
            L.desc.keep_ratio = 1.0
            L.nblk, L.kkeep = crisp_keep_count(L.desc)
            L.build_mask_max_known(s, stream)
            count += 1
        return count

    def _check_gradient(self, g, layer):
        """The library gets an address and a pitch: what is no bf16 or fp32 matrix of the layer's size on a GPU would be read beyond its end, or as
        something else.  (What only has a tensor's methods answers for itself.)"""
        torch = self.torch
        if isinstance(g, torch.Tensor):
            assert g.is_cuda and g.dtype in (torch.bfloat16, torch.float32) and _holds_rows(g, layer.desc.rows, layer.desc.k), \
                "a gradient is a bf16 or fp32 CUDA tensor of its layer's shape"

    def _table(self, arr, layers, weights, grads):
        """Fills in the table of the layers: one host array each for what there is per gradient (returned; the entries point into them),
        and one struct per layer."""
        for L, gs in zip(layers, grads):
            for g in gs:
                self._check_gradient(g, L)
        flat = [g for gs in grads for g in gs]
        ptrs = array("Q", [g.data_ptr() for g in flat])
        lds = array("q", [g.stride()[0] for g in flat])
        dts = array("i", [0 if g.dtype is self.torch.bfloat16 else 1 for g in flat])
        p0, l0, d0, at = ptrs.buffer_info()[0], lds.buffer_info()[0], dts.buffer_info()[0], 0
        for P, L, w, gs, s in zip(arr, layers, weights, grads, self.sal):
            P.desc, P.d_w_bf16, P.ld_w = L.desc, w.data_ptr(), w.stride()[0]
            n = len(gs)
            P.d_grads, P.ld_grads, P.grad_dtypes, P.samples = p0 + 8 * at, l0 + 8 * at, d0 + 4 * at, n
            P.d_saliency, P.ld_s = s.data_ptr(), s.stride()[0]
            P.d_mask_buf, P.d_workspace = L.mask_buf.data_ptr(), L.workspace.data_ptr()
            at += n
        return ptrs, lds, dts, flat

    def step(self, weights, grads, kappa, stream=None):
        """weights[l]: bf16 CUDA tensor [rows, k]; grads[l]: list of H gradient tensors (bf16 or fp32) of that shape;
        kappa: overall sparsity target of this iteration.  Returns the kept-block count of every layer; the layers'
        masks and handles (self.layers[l]) hold the result.

        Lists and tuples (or stacked tensors) of gradients are taken for all layers at once.  Anything else that can be iterated over (a generator
        that makes one layer's gradients after the other, say) is read layer by layer and gradient by gradient, and each
        gradient's kernel is on the stream before the next one is asked for."""
        torch = self.torch
        weights = list(weights)
        # every gradient exists, and none is changed by asking for the next
        held = (list, tuple, torch.Tensor)
        at_once = isinstance(grads, held) and (set(map(type, grads)) <= {list, tuple} or all(isinstance(gs, held) for gs in grads))
        count = min(len(self.layers), len(weights), len(grads) if at_once else len(weights))
        weights, layers = weights[:count], self.layers[:count]
        arr, table = (PruneLayer * count)(), None
        if at_once and _network:
            gradients = [gs if type(gs) in (list, tuple) else list(gs) for gs in grads[:count]]
            table = _network.table(layers, weights, gradients, self.sal, C.addressof(arr))
        if table is None:
            assert all(w.is_cuda and w.element_size() == 2 and w.stride()[1] == 1 and (not isinstance(w, torch.Tensor) or _holds_rows(w, L.desc.rows, L.desc.k))
                       for w, L in zip(weights, layers))
            if not at_once:
                count = self._score_in_turn(weights, grads, stream)
                arr, layers = (PruneLayer * count)(), layers[:count]
            table = self._table(arr, layers, weights, grads[:count] if at_once else [()] * count)
        if at_once:
            crisp_prune_score(arr, stream)
        crisp_global_rank(self.rank_arr, crisp_prune_fraction(kappa, self.n, self.m), self.rank_ws, self.d_kkeep, stream)
        # While the device scores and ranks: what the encodings need whatever the counts are, and the masks and handles that
        # they will take the place of.
        old_masks, old_handles, masks, handles = [(C.c_void_p * count)() for _ in range(4)]
        canonical_bytes, exec_bytes, have_c, have_e = [(C.c_size_t * count)() for _ in range(4)]
        if not (_network and _network.encodings(layers, *map(C.addressof, (arr, have_c, have_e, old_masks, old_handles)))):
            for i, (P, L) in enumerate(zip(arr, layers)):
                if L.canonical_buf is not None:
                    P.d_canonical_buf, P.d_exec_buf = L.canonical_buf.data_ptr(), L.exec_buf.data_ptr()
                    have_c[i], have_e[i] = L.canonical_buf.numel(), L.exec_buf.numel()
                old_masks[i], old_handles[i] = L.mask, L.handle
        # (a copy into pinned memory and a wait for the stream: 10 us less than a copy into pageable memory)
        with _allocating_for(stream):
            self._h_kkeep.copy_(self.d_kkeep, non_blocking=True)
            torch.cuda.current_stream(self.d_kkeep.device).synchronize()
        kk = self._h_kkeep.tolist()
        for P, c in zip(arr, kk):
            P.kkeep = c
        _check(_lib.crisp_prune_encode_sizes(count, arr, canonical_bytes, exec_bytes), "crisp_prune_encode_sizes")
        for i, (cb, eb) in enumerate(zip(canonical_bytes, exec_bytes)):
            if cb > have_c[i] or eb > have_e[i]:
                P, L = arr[i], layers[i]
                L._reserve(cb, eb, stream)
                P.d_canonical_buf, P.d_exec_buf = L.canonical_buf.data_ptr(), L.exec_buf.data_ptr()
        _check(_lib.crisp_prune_encode(count, arr, _stream(stream), masks, handles), "crisp_prune_encode")
        if _network:
            _network.encoded(layers, kk, *map(C.addressof, (self._blocks, masks, handles)))
        else:
            for L, c, mask, handle in zip(layers, kk, masks, handles):
                L.mask, L.handle, L.kkeep = mask, handle, c
                L.desc.keep_ratio = c / L.nblk               # floor(ratio * nblk + 0.5) gives the count back
        crisp_destroy_layers(old_masks, old_handles)
        return kk

    def optimizer(self, weights, **options):
        """AdamW for this network's weights, which are held where the layers' masks have no bit to zero: weights[l] is what `step` prunes
        or, fp32, what it was rounded from (then with copies=: the bf16 tensors that `step` takes).  Options as for AdamW.  The masks are those that the
        layers have when the optimizer's step is called; a layer without one is updated everywhere."""
        return AdamW(weights, masks=self.layers, **options)

    def close(self):
        for L in self.layers:
            L.close()


class Normed:
    """What GroupNorm.forward leaves: y, the statistics [batch, groups, 2] (mean, 1 / standard deviation) that the backward pass takes, and the 8-bit forms of
    x and y that were asked for (Activations8 of k = channels and a column a pixel)."""
    __slots__ = ("y", "statistics", "x8", "y8")

    def __init__(self, y, statistics, x8, y8):
        self.y, self.statistics, self.x8, self.y8 = y, statistics, x8, y8


class GroupNorm:
    """Group norm with an activation over channels-last activations (crisp_group_norm): y = act(weight * (x - mean) / sqrt(var + eps) + bias), mean and variance of
    each sample's groups of channels.

    x is a bf16, fp16 or fp32 CUDA tensor [batch, ..., channels] whose pixels lie a constant pitch apart (an NHWC tensor, or a slice of its channels); weight and
    bias are fp32 CUDA tensors [channels] that this object keeps, or None.  activation: "none", "relu", "relu6" or "silu".
    """
    ACTIVATIONS = {"none": 0, "relu": 1, "relu6": 2, "silu": 3}

    def __init__(self, channels, groups, weight=None, bias=None, eps=1e-5, activation="none"):
        import torch
        self.torch = torch
        self.channels, self.groups, self.eps = channels, groups, float(eps)
        self.activation = self.ACTIVATIONS["none" if activation is None else activation]
        self.weight, self.bias = weight, bias
        self._types = {torch.bfloat16: 0, torch.float32: 1, torch.float16: 2}
        self._native = bool(_network or _bind_network())
        crisp_group_norm_sizes(self._desc(1, 1, 0), False)                   # (channels, groups and eps that the library refuses are refused here)

    def _desc(self, batch, pixels, dtype):
        return GroupNormDesc(batch, pixels, self.channels, self.groups, self.activation, dtype, self.eps)

    def _rows(self, t, what, like=None):
        """Elements from one pixel to the next."""
        shape = t.shape
        assert t.is_cuda and t.dtype in self._types and len(shape) >= 2 and shape[-1] == self.channels, \
            f"{what} is a bf16, fp16 or fp32 CUDA tensor [batch, ..., channels]"
        assert like is None or (t.dtype == like.dtype and t.device == like.device and shape == like.shape), f"{what} has another shape, type or device"
        return _pixel_pitch(t, what)

    def _parameters(self, device):
        for p in (self.weight, self.bias):
            assert p is None or (p.device == device and p.dtype == self.torch.float32 and p.numel() == self.channels and p.is_contiguous()), \
                "weight and bias are fp32 tensors of as many consecutive elements as there are channels, on the activations' device"

    def _shape(self, t):
        """batch, pixels of one sample"""
        pixels = 1
        for size in t.shape[1:-1]:
            pixels *= size
        return t.shape[0], pixels

    def _workspace(self, desc, backward, device, stream):
        size = crisp_group_norm_sizes(desc, backward)
        with _allocating_for(stream):                                        # given back when the call returns: to the stream that uses it
            return self.torch.empty_strided((size,), (1,), dtype=self.torch.uint8, device=device) if size else None

    def forward(self, x, y=None, keep_x=False, keep_y=False, plain_y=True, stream=None):
        """-> Normed.  keep_x, keep_y: x and y also in 8 bits, written in the same pass; plain_y=False: y in 8 bits alone.  y: where to write it (x itself, too)."""
        torch = self.torch
        if y is None and stream is None and self._native and (plain_y or keep_y):
            done = _network.norm(x, self.weight, self.bias, self.eps, self.channels, self.groups, self.activation, keep_x, keep_y, plain_y, _current_device(),
                                 _current_stream())
            if done is not None:
                code, y, statistics, x8, y8, columns = done
                if code:
                    raise CrispError(code, "crisp_group_norm")
                return Normed(y, statistics, x8 if x8 is None else Activations8(self.channels, columns, x8),
                              y8 if y8 is None else Activations8(self.channels, columns, y8))
        ldx = self._rows(x, "x")
        device, (batch, pixels) = x.device, self._shape(x)
        self._parameters(device)
        assert plain_y or (keep_y and y is None), "neither y nor its 8-bit form is asked for"
        desc = self._desc(batch, pixels, self._types[x.dtype])
        with _on(device):
            with _allocating_for(stream):
                statistics = torch.empty_strided((batch, self.groups, 2), (self.groups * 2, 2, 1), dtype=torch.float32, device=device)
                if y is None and plain_y:
                    y = torch.empty(x.shape, dtype=x.dtype, device=device)
            ldy = self._rows(y, "y", x) if y is not None else 0
            x8, y8 = (_buffer8(self.channels, batch * pixels, device, stream) if wanted and batch else None for wanted in (keep_x, keep_y))
            crisp_group_norm(desc, x, ldx, self.weight, self.bias, y, ldy, statistics, x8 and x8.buffer, y8 and y8.buffer,
                             self._workspace(desc, False, device, stream), stream)
        return Normed(y, statistics, x8, y8)

    __call__ = forward

    def backward(self, dy, x, statistics, dx=None, stream=None):
        """-> dx, dweight, dbias (fp32).  x: the forward pass's, as it was or in 8 bits (Normed.x8); statistics: Normed's.  dx: where to write it (dy or x, too)."""
        torch = self.torch
        if dx is None and stream is None and self._native:
            held = type(x) is Activations8
            if not held or x.k == self.channels:
                done = _network.norm_backward(dy, x.buffer if held else x, statistics, self.weight, self.bias, self.eps, self.channels, self.groups, self.activation,
                                              x.ncols if held else -1, _current_device(), _current_stream())
                if done is not None:
                    if done[0]:
                        raise CrispError(done[0], "crisp_group_norm_backward")
                    return done[1:]
        ld_dy = self._rows(dy, "dy")
        device, (batch, pixels) = dy.device, self._shape(dy)
        self._parameters(device)
        held = isinstance(x, Activations8)
        if held:
            assert x.k == self.channels and x.ncols == batch * pixels and x.buffer.device == device, "x in 8 bits of other sizes, or on another device"
        ldx = 0 if held or x is None else self._rows(x, "x", dy)
        assert statistics.device == device and statistics.dtype == torch.float32 and statistics.shape == (batch, self.groups, 2) and statistics.is_contiguous(), \
            "statistics are the forward pass's, [batch, groups, 2]"
        desc = self._desc(batch, pixels, self._types[dy.dtype])
        with _on(device):
            with _allocating_for(stream):
                dweight, dbias = (torch.empty_strided((self.channels,), (1,), dtype=torch.float32, device=device) for _ in range(2))
                if dx is None:
                    dx = torch.empty(dy.shape, dtype=dy.dtype, device=device)
            ld_dx = self._rows(dx, "dx", dy)
            crisp_group_norm_backward(desc, dy, ld_dy, None if held else x, ldx, x.buffer if held else None, statistics, self.weight, self.bias, dx, ld_dx,
                                      dweight, dbias, self._workspace(desc, True, device, stream), stream)
        return dx, dweight, dbias


def _rows_of(t):
    """(rows, k, pitch) of a tensor whose elements lie in rows of consecutive ones, or None."""
    shape, strides = t.shape, t.stride()
    if len(shape) == 0 or 0 in shape:
        return (1, t.numel(), t.numel())
    if t.is_contiguous():
        k = t.numel() // shape[0]
        return (shape[0], k, k) if len(shape) > 1 else (1, shape[0], shape[0])
    if len(shape) == 2 and (strides[1] == 1 or shape[1] == 1) and strides[0] >= shape[1]:
        return (shape[0], shape[1], strides[0])
    return None


def _kept_buffer(name):
    """A buffer whose address the table of a step holds: what is assigned to it is copied into it."""
    def take(self, value):
        buffer = getattr(self, name)
        assert buffer is not None and value.shape == buffer.shape and value.dtype == buffer.dtype, "a state keeps its size and type"
        buffer.copy_(value)
    return property(operator.attrgetter(name), take)


class AdamW:
    """AdamW over many tensors in one call (crisp_adamw): the fine-tuning that follows a pruning step.

    weights   CUDA tensors, fp32 or bf16, contiguous or matrices of consecutive rows; updated in place (bf16 ones are rounded at random)
    copies    bf16 tensors of the same shapes, or None for none: what fp32 weights are rounded to after every step
    masks     for each tensor None, or a HybridLayer of its shape (or a crisp_mask_t): weights without a bit in its mask become and stay 0
    state_bits 32, or 8 with a scale for each 128 elements.  The states of all tensors lie in the flat buffers m and v, each beginning at a multiple
              of 128 elements (`starts`): fp32 m and v, or uint8 codes of m and sqrt(v) with biased exponents in m_exp and v_exp (crisp.h).  They,
              `step_count` and `seed` are all there is to save (and lr, where it is not the constructor's).
              They stay where they are: what is assigned to one is copied into it.
    capturable  the step number is kept in device memory (`d_step`, counted up by every step), and so is lr (`d_lr`): a captured step
              goes on counting when it is replayed, and takes the lr that was assigned last.  Assigning `lr` and `step_count` writes d_lr and d_step on the
              current stream, and reading them waits for the device.
    """

    m, v, m_exp, v_exp, d_step, d_lr = (_kept_buffer(name) for name in ("_m", "_v", "_m_exp", "_v_exp", "_d_step", "_d_lr"))

    def __init__(self, weights, copies=None, masks=None, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2, state_bits=32, seed=0, step=0,
                 capturable=False):
        import torch
        self.torch = torch
        self.weights = list(weights)
        n = len(self.weights)
        self.copies = [None] * n if copies is None else list(copies)
        self.masks = [None] * n if masks is None else list(masks)
        assert len(self.copies) == n and len(self.masks) == n, "a copy and a mask, or None, for each tensor"
        assert state_bits in (8, 32), "states are held in 8 bits or in 32"
        self._lr, self.betas, self.eps, self.weight_decay = lr, betas, eps, weight_decay
        self.state_bits, self.seed, self._step_count = state_bits, seed, step
        self.device = self.weights[0].device if n else torch.device("cuda", torch.cuda.current_device())
        assert all(getattr(mask, "device", self.device) == self.device for mask in self.masks), "a layer and the weights under its mask lie on one device"
        self._table = (AdamwTensor * n)()
        self._address = C.addressof(self._table)
        self.starts, at = [], 0
        for w in self.weights:
            self.starts.append(at)
            at += (w.numel() + 127) // 128 * 128
        self.elements = at
        wide = state_bits == 32
        state = lambda count, dtype: torch.zeros(count, dtype=dtype, device=self.device)  # noqa: E731
        self._m, self._v = [state(at, torch.float32 if wide else torch.uint8) for _ in range(2)]
        self._m_exp, self._v_exp = [None if wide else state(at // 128, torch.uint8) for _ in range(2)]
        spans = []
        for i, (T, w, c) in enumerate(zip(self._table, self.weights, self.copies)):
            rows = _rows_of(w)
            assert rows and w.dtype in (torch.float32, torch.bfloat16), "weights are fp32 or bf16 CUDA tensors, in rows of consecutive elements"
            (T.rows, T.k, _), T.w_dtype = rows, int(w.dtype == torch.float32)
            self._place(T, w, c)
            T.d_m, T.d_v = (b.data_ptr() + self.starts[i] * b.element_size() for b in (self.m, self.v))
            if not wide:
                T.d_m_exp, T.d_v_exp = (b.data_ptr() + self.starts[i] // 128 for b in (self.m_exp, self.v_exp))
            for t in (w, c):
                if t is not None and t.numel():
                    spans.append((t.data_ptr(), t.data_ptr() + (sum((s - 1) * d for s, d in zip(t.shape, t.stride())) + 1) * t.element_size()))
        spans.sort()
        assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:])), "the address ranges of two weights or copies overlap"
        load()
        if _network is None:
            _bind_network()
        self._params = AdamwParams(state_bits=state_bits)
        self.capturable = capturable
        self._d_step = torch.full((1,), step, dtype=torch.int64, device=self.device) if capturable else None
        self._d_lr = torch.full((1,), lr, dtype=torch.float32, device=self.device) if capturable else None
        if capturable:
            self._params.d_step, self._params.d_lr = self.d_step.data_ptr(), self.d_lr.data_ptr()

    @property
    def lr(self):
        return float(self.d_lr) if self.capturable else self._lr

    @lr.setter
    def lr(self, value):
        if self.capturable:
            self.d_lr.fill_(value)
        else:
            self._lr = value

    @property
    def step_count(self):
        """Steps made so far."""
        return int(self.d_step) if self.capturable else self._step_count

    @step_count.setter
    def step_count(self, value):
        if self.capturable:
            self.d_step.fill_(value)
        else:
            self._step_count = value

    def _place(self, T, w, c):
        """Where a tensor's weights and their copy lie."""
        torch, rows = self.torch, _rows_of(w)
        assert w.is_cuda and w.device == self.device and rows and rows[:2] == (T.rows, T.k) and w.dtype == (torch.float32 if T.w_dtype else torch.bfloat16), \
            "weights are CUDA tensors of one device and keep their shape and type"
        T.d_w, T.ld_w, T.d_copy_bf16, T.ld_copy = w.data_ptr(), rows[2], None, 0
        if c is not None:
            rows = _rows_of(c)
            assert c.is_cuda and c.device == self.device and c.dtype == torch.bfloat16 and T.w_dtype and c.shape == w.shape and rows, \
                "a copy is a bf16 CUDA tensor of the shape of its fp32 weights"
            T.d_copy_bf16, T.ld_copy = c.data_ptr(), rows[2]

    def step(self, grads, grad_scale=None, stream=None):
        """One step with grads[i] (bf16 or fp32, of the shape of weights[i], in rows of consecutive elements; None: the tensor is left as it is);
        grad_scale: an fp32 CUDA tensor of one element that the gradients are multiplied by (a clipping factor, say)."""
        assert len(grads) == len(self._table), "a gradient, or None, for each tensor"
        p = self._params
        p.lr, (p.beta1, p.beta2), p.eps, p.weight_decay = self._lr, self.betas, self.eps, self.weight_decay
        p.step, p.seed = self._step_count + 1, self.seed     # (where it is kept on the device the first is not heeded)
        if grad_scale is not None:
            assert grad_scale.is_cuda and grad_scale.device == self.device and grad_scale.dtype is self.torch.float32 and grad_scale.numel() == 1, \
                "grad_scale is an fp32 CUDA tensor of one element"
        p.d_grad_scale = grad_scale.data_ptr() if grad_scale is not None else None
        gpu = self.device.index
        if gpu == _current_device():
            self._launch(grads, stream, gpu)
        else:
            with self.torch.cuda.device(self.device):
                self._launch(grads, stream, gpu)
        if not self.capturable:
            self._step_count += 1
        return self

    def _launch(self, grads, stream, gpu):
        if self.capturable:                                  # (the step's own number, made before it and taken back if it is refused)
            with _allocating_for(stream):
                self._d_step += 1
        try:
            code = None
            if _network and type(grads) is list:
                code = _network.adamw(self._address, self.weights, self.copies, grads, self.masks, C.addressof(self._params), _stream(stream), gpu)
            if code is None:
                self._gradients(grads)
                self.torch.autograd.graph.increment_version([t for ts, g in zip(zip(self.weights, self.copies), grads) for t in ts
                                                             if t is not None and g is not None and not t.is_inference()])
                code = _lib.crisp_adamw(len(self._table), self._table, self._params, _stream(stream))
            if code:
                raise CrispError(code, "crisp_adamw")
        except Exception:
            if self.capturable:
                with _allocating_for(stream):
                    self._d_step -= 1
            raise

    def _gradients(self, grads):
        """Fills in what a step's gradients and masks bring, or says what is wrong with them."""
        torch = self.torch
        for T, g, w, c, mask in zip(self._table, grads, self.weights, self.copies, self.masks):
            if g is None:
                T.d_grad = None
                continue
            self._place(T, w, c)
            assert g.is_cuda and g.device == self.device and g.dtype in (torch.float32, torch.bfloat16) and g.shape == w.shape, \
                "a gradient is a bf16 or fp32 CUDA tensor of its weights' shape"
            rows = _rows_of(g)
            assert rows, "a gradient lies in rows of consecutive elements"
            assert getattr(mask, "device", self.device) == self.device, "a layer and the weights under its mask lie on one device"
            T.d_grad, T.grad_dtype, T.ld_grad = g.data_ptr(), int(g.dtype == torch.float32), rows[2]
            T.mask = getattr(mask, "mask", mask) or None

    def moments(self, stream=None):
        """(m, sqrt(v)) of 8-bit states as flat bf16 tensors, in which they are exact (but for an m below 2^-126)."""
        assert self.state_bits == 8, "32-bit states are their values"
        if stream is not None:
            with self.torch.cuda.device(self.device), _allocating_for(stream):
                return self.moments()
        if _network and self.device.index == _current_device():
            code, *out = _network.moments(self._m, self._m_exp, self._v, self._v_exp, _current_stream())
            if code:
                raise CrispError(code, "crisp_adamw_moments")
            return out
        n = self.elements
        with self.torch.cuda.device(self.device):
            both = self.torch.empty_strided((2, n), (n, 1), dtype=self.torch.bfloat16, device=self.device)
            at = both.data_ptr()
            code = _lib.crisp_adamw_moments(self.m.data_ptr(), self.m_exp.data_ptr(), self.v.data_ptr(), self.v_exp.data_ptr(), n, at, at + 2 * n, _current_stream())
        if code:
            raise CrispError(code, "crisp_adamw_moments")
        return list(both.unbind(0))
