// The parts of a pruning iteration that go over all layers and gradients of a network in Python: the table of the layers, and the tensors that
// decode returns.  They take torch's tensors themselves.  Asking a tensor for its address and pitch from Python takes 0.4 us, a layer's entry of
// the table 3 us and a tensor made by torch.empty_strided 1.6, of an iteration of 35 layers and 140 gradients that waits for all of it.  What they
// cannot do as the Python code beside their callers does (tensor subclasses, other containers, types and shapes) they leave to it by returning None.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty_strided.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <cstdint>
#include <cstring>

#include "crisp.h"

namespace {

decltype(&crisp_decode) lib_decode;
decltype(&crisp_spmm8_sizes) lib_spmm8_sizes;
decltype(&crisp_spmm8) lib_spmm8;
decltype(&crisp_decode8) lib_decode8;
decltype(&crisp_encode8_sizes) lib_encode8_sizes;
decltype(&crisp_encode8) lib_encode8;
decltype(&crisp_destroy8) lib_destroy8;
decltype(&crisp_adamw) lib_adamw;
decltype(&crisp_adamw_moments) lib_moments;

// The names of attributes, made once.
struct {
    PyObject *desc, *mask_buf, *workspace, *canonical_buf, *exec_buf, *mask, *handle, *kkeep;
} names;

struct Ref {                             // an owned reference
    PyObject *p;
    explicit Ref(PyObject *o = nullptr) : p(o) {}
    ~Ref() { Py_XDECREF(p); }
    Ref(const Ref &) = delete;
    Ref &operator=(const Ref &) = delete;
};

// A plain tensor (or parameter) of two dimensions on a GPU, or nullptr.
const at::Tensor *plain(PyObject *o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == at::kStrided && t.dim() == 2 ? &t : nullptr;
}
// The address of a buffer that the object owns; false with an exception, or true and *out null where the attribute is no plain tensor.
bool buffer(PyObject *owner, PyObject *name, void **out, int64_t *numel) {
    Ref o(PyObject_GetAttr(owner, name));
    if (!o.p) return false;
    *out = nullptr;
    if (THPVariable_CheckExact(o.p)) {
        const at::Tensor &t = THPVariable_Unpack(o.p);
        *out = t.data_ptr();
        if (numel) *numel = t.numel();
    }
    return true;
}
// Whether it holds the layer's rows of consecutive elements.
bool holds(const at::Tensor &t, const crisp_layer_desc_t &d) {
    return t.size(0) >= d.rows && t.size(1) >= d.k && (t.stride(1) == 1 || d.k == 1);
}
bool descriptor(PyObject *layer, crisp_layer_desc_t *copy, double *keep_ratio) {        // reads it, or sets its keep ratio
    Ref o(PyObject_GetAttr(layer, names.desc));
    if (!o.p) return false;
    Py_buffer view;
    if (PyObject_GetBuffer(o.p, &view, PyBUF_WRITABLE) != 0) return false;
    const bool ok = view.len == (Py_ssize_t)sizeof(crisp_layer_desc_t);
    if (ok && copy) std::memcpy(copy, view.buf, sizeof *copy);
    if (ok && keep_ratio) static_cast<crisp_layer_desc_t *>(view.buf)->keep_ratio = *keep_ratio;
    PyBuffer_Release(&view);
    if (!ok) PyErr_SetString(PyExc_TypeError, "a layer's descriptor has another size");
    return ok;
}
template <typename T> T *address(PyObject *o) { return reinterpret_cast<T *>(PyLong_AsVoidPtr(o)); }
bool arguments(const char *name, Py_ssize_t given, Py_ssize_t n) {
    if (given == n) return true;
    PyErr_Format(PyExc_TypeError, "%s takes %zd arguments (%zd given)", name, n, given);
    return false;
}

// table(layers, weights, gradients, saliencies, array of crisp_prune_layer_t) -> bytes that the array's entries point into, or None: not filled in.
// All four are lists; an entry of `gradients` is a list or tuple.
PyObject *table(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arguments("table", n, 5)) return nullptr;
    for (int i = 0; i < 4; ++i)
        if (!PyList_CheckExact(args[i])) Py_RETURN_NONE;
    const Py_ssize_t count = PyList_GET_SIZE(args[1]);
    crisp_prune_layer_t *arr = address<crisp_prune_layer_t>(args[4]);
    if (!arr) return PyErr_Occurred() ? nullptr : Py_NewRef(Py_None);
    if (PyList_GET_SIZE(args[0]) < count || PyList_GET_SIZE(args[2]) < count || PyList_GET_SIZE(args[3]) < count) Py_RETURN_NONE;
    Py_ssize_t total = 0;
    for (Py_ssize_t l = 0; l < count; ++l) {
        PyObject *gs = PyList_GET_ITEM(args[2], l);
        if (!PyList_CheckExact(gs) && !PyTuple_CheckExact(gs)) Py_RETURN_NONE;
        total += PySequence_Fast_GET_SIZE(gs);
    }
    Ref held(PyBytes_FromStringAndSize(nullptr, total * (Py_ssize_t)(sizeof(void *) + sizeof(int64_t) + sizeof(int32_t)) + 8));
    if (!held.p) return nullptr;
    uintptr_t at = (reinterpret_cast<uintptr_t>(PyBytes_AS_STRING(held.p)) + 7) & ~(uintptr_t)7;
    const void **ptrs = reinterpret_cast<const void **>(at);
    int64_t *lds = reinterpret_cast<int64_t *>(ptrs + total);
    int32_t *dtypes = reinterpret_cast<int32_t *>(lds + total);
    for (Py_ssize_t l = 0; l < count; ++l) {
        crisp_prune_layer_t &P = arr[l];
        PyObject *layer = PyList_GET_ITEM(args[0], l), *gs = PyList_GET_ITEM(args[2], l);
        const at::Tensor *w = plain(PyList_GET_ITEM(args[1], l)), *s = plain(PyList_GET_ITEM(args[3], l));
        if (!w || !s || w->element_size() != 2 || w->stride(1) != 1) Py_RETURN_NONE;
        if (!descriptor(layer, &P.desc, nullptr) || !buffer(layer, names.mask_buf, &P.d_mask_buf, nullptr) ||
            !buffer(layer, names.workspace, &P.d_workspace, nullptr))
            return nullptr;
        if (!P.d_mask_buf || !P.d_workspace || !holds(*w, P.desc)) Py_RETURN_NONE;
        P.d_w_bf16 = static_cast<const uint16_t *>(w->data_ptr()); P.ld_w = w->stride(0);
        P.d_saliency = static_cast<float *>(s->data_ptr()); P.ld_s = s->stride(0);
        P.d_grads = ptrs; P.ld_grads = lds; P.grad_dtypes = dtypes;
        P.samples = (int32_t)PySequence_Fast_GET_SIZE(gs);
        PyObject **items = PySequence_Fast_ITEMS(gs);
        for (int32_t h = 0; h < P.samples; ++h) {
            const at::Tensor *g = plain(items[h]);
            if (!g || (g->scalar_type() != at::kBFloat16 && g->scalar_type() != at::kFloat) || !holds(*g, P.desc)) Py_RETURN_NONE;
            *ptrs++ = g->data_ptr(); *lds++ = g->stride(0);
            *dtypes++ = g->scalar_type() == at::kBFloat16 ? 0 : 1;
        }
    }
    return Py_NewRef(held.p);
    END_HANDLE_TH_ERRORS
}

// encodings(layers, array of crisp_prune_layer_t, size_t canonical capacities, size_t execution capacities, old masks, old handles): what the encodings
// need whatever the counts are, and the masks and handles that they will take the place of.
PyObject *encodings(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arguments("encodings", n, 6)) return nullptr;
    if (!PyList_CheckExact(args[0])) Py_RETURN_FALSE;
    crisp_prune_layer_t *arr = address<crisp_prune_layer_t>(args[1]);
    size_t *canonical = address<size_t>(args[2]), *execution = address<size_t>(args[3]);
    void **masks = address<void *>(args[4]), **handles = address<void *>(args[5]);
    if (!arr || !canonical || !execution || !masks || !handles) return PyErr_Occurred() ? nullptr : Py_NewRef(Py_False);
    for (Py_ssize_t l = 0; l < PyList_GET_SIZE(args[0]); ++l) {
        PyObject *layer = PyList_GET_ITEM(args[0], l);
        int64_t have_c = 0, have_e = 0;
        if (!buffer(layer, names.canonical_buf, &arr[l].d_canonical_buf, &have_c) || !buffer(layer, names.exec_buf, &arr[l].d_exec_buf, &have_e)) return nullptr;
        canonical[l] = (size_t)have_c; execution[l] = (size_t)have_e;
        Ref mask(PyObject_GetAttr(layer, names.mask)), handle(PyObject_GetAttr(layer, names.handle));
        if (!mask.p || !handle.p) return nullptr;
        masks[l] = PyLong_AsVoidPtr(mask.p); handles[l] = PyLong_AsVoidPtr(handle.p);
        if (PyErr_Occurred()) return nullptr;
    }
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// encoded(layers, counts, blocks, masks, handles): the layers take their new masks and handles; blocks: int32 blocks of a row tile.
PyObject *encoded(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arguments("encoded", n, 5)) return nullptr;
    const int32_t *blocks = address<int32_t>(args[2]);
    void **masks = address<void *>(args[3]), **handles = address<void *>(args[4]);
    if (!PyList_CheckExact(args[0]) || !PyList_CheckExact(args[1]) || PyList_GET_SIZE(args[1]) < PyList_GET_SIZE(args[0]) || !blocks || !masks || !handles) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "encoded(layers, counts, blocks, masks, handles)");
        return nullptr;
    }
    for (Py_ssize_t l = 0; l < PyList_GET_SIZE(args[0]); ++l) {
        PyObject *layer = PyList_GET_ITEM(args[0], l), *c = PyList_GET_ITEM(args[1], l);
        Ref mask(PyLong_FromVoidPtr(masks[l])), handle(PyLong_FromVoidPtr(handles[l]));
        if (!mask.p || !handle.p || PyObject_SetAttr(layer, names.mask, mask.p) || PyObject_SetAttr(layer, names.handle, handle.p) ||
            PyObject_SetAttr(layer, names.kkeep, c))
            return nullptr;
        double ratio = (double)PyLong_AsLong(c) / (double)blocks[l];                // floor(ratio * blocks + 0.5) gives the count back
        if (PyErr_Occurred() || !descriptor(layer, nullptr, &ratio)) return nullptr;
    }
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// decode(handle, rows, k, GPU, stream) and decode8(...) -> (status, bf16 tensor [rows, k])
template <typename Handle>
PyObject *dense(crisp_status_t (*call)(Handle, uint16_t *, int64_t, void *), const char *name, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arguments(name, n, 5)) return nullptr;
    long long v[5];
    for (int i = 0; i < 5; ++i) {
        v[i] = PyLong_AsLongLong(args[i]);
        if (v[i] == -1 && PyErr_Occurred()) return nullptr;
    }
    at::Tensor w = at::empty_strided({v[1], v[2]}, {v[2], 1}, at::TensorOptions().dtype(at::kBFloat16).device(at::Device(at::kCUDA, (at::DeviceIndex)v[3])));
    crisp_status_t s;
    Py_BEGIN_ALLOW_THREADS
    s = call(reinterpret_cast<Handle>((uintptr_t)v[0]), static_cast<uint16_t *>(w.data_ptr()), v[2], reinterpret_cast<void *>((uintptr_t)v[4]));
    Py_END_ALLOW_THREADS
    Ref out(THPVariable_Wrap(std::move(w)));
    return out.p ? Py_BuildValue("lO", (long)s, out.p) : nullptr;
    END_HANDLE_TH_ERRORS
}
PyObject *decode(PyObject *, PyObject *const *args, Py_ssize_t n) { return dense(lib_decode, "decode", args, n); }
PyObject *decode8(PyObject *, PyObject *const *args, Py_ssize_t n) { return dense(lib_decode8, "decode8", args, n); }

// Rows, columns and pitch of a tensor whose elements lie in rows of consecutive ones (as the binding's _rows_of has them); false: it does not.
bool rows_of(const at::Tensor &t, int64_t (&v)[3]) {
    const int64_t n = t.numel();
    if (t.dim() == 0 || n == 0) {
        v[0] = 1; v[1] = v[2] = n;
    } else if (t.is_contiguous()) {
        v[0] = t.dim() > 1 ? t.size(0) : 1;
        v[1] = v[2] = n / v[0];
    } else if (t.dim() == 2 && (t.stride(1) == 1 || t.size(1) == 1) && t.stride(0) >= t.size(1)) {
        v[0] = t.size(0); v[1] = t.size(1); v[2] = t.stride(0);
    } else {
        return false;
    }
    return true;
}

// adamw(array of crisp_adamw_tensor_t, weights, copies, gradients, masks, crisp_adamw_t, stream, GPU) -> status: where the tensors of a step lie, and its masks, and the step;
// or None: not a step that this takes, and nothing done.  The four are lists of one length; an entry of `copies` and `gradients` may be None, one of `masks` a layer or None.  (The shapes and types of weights and copies
// are those that the array was made for, or it is not filled in.)
PyObject *adamw(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arguments("adamw", n, 8)) return nullptr;
    crisp_adamw_tensor_t *arr = address<crisp_adamw_tensor_t>(args[0]);
    const crisp_adamw_t *params = address<const crisp_adamw_t>(args[5]);
    void *stream = PyLong_AsVoidPtr(args[6]);
    const long gpu = PyLong_AsLong(args[7]);                 // of the states: all else has to lie there
    if (PyErr_Occurred()) return nullptr;
    if (!arr || !params) Py_RETURN_NONE;
    for (int i = 1; i < 5; ++i)
        if (!PyList_CheckExact(args[i]) || PyList_GET_SIZE(args[i]) != PyList_GET_SIZE(args[1])) Py_RETURN_NONE;
    for (Py_ssize_t l = 0; l < PyList_GET_SIZE(args[1]); ++l) {
        crisp_adamw_tensor_t &T = arr[l];
        PyObject *wo = PyList_GET_ITEM(args[1], l), *co = PyList_GET_ITEM(args[2], l), *go = PyList_GET_ITEM(args[3], l), *mo = PyList_GET_ITEM(args[4], l);
        T.d_grad = nullptr;
        if (go == Py_None) continue;
        if (!THPVariable_CheckExact(go) || !THPVariable_Check(wo) || (co != Py_None && !THPVariable_Check(co))) Py_RETURN_NONE;
        const at::Tensor &g = THPVariable_Unpack(go), &w = THPVariable_Unpack(wo);
        int64_t rows[3];
        if (!w.is_cuda() || w.get_device() != gpu || w.layout() != at::kStrided || w.scalar_type() != (T.w_dtype ? at::kFloat : at::kBFloat16) || !rows_of(w, rows) || rows[0] != T.rows ||
            rows[1] != T.k)
            Py_RETURN_NONE;
        T.d_w = w.data_ptr(); T.ld_w = rows[2];
        T.d_copy_bf16 = nullptr; T.ld_copy = 0;              // (the table is kept from step to step, and a copy may have been given up)
        if (co != Py_None) {
            const at::Tensor &c = THPVariable_Unpack(co);
            if (!c.is_cuda() || c.layout() != at::kStrided || c.device() != w.device() || c.scalar_type() != at::kBFloat16 || !c.sizes().equals(w.sizes()) ||
                !rows_of(c, rows))
                Py_RETURN_NONE;
            T.d_copy_bf16 = static_cast<uint16_t *>(c.data_ptr()); T.ld_copy = rows[2];
        }
        if (!g.is_cuda() || g.layout() != at::kStrided || g.device() != w.device() || (g.scalar_type() != at::kBFloat16 && g.scalar_type() != at::kFloat) ||
            !g.sizes().equals(w.sizes()) || !rows_of(g, rows))
            Py_RETURN_NONE;
        void *mask = nullptr;
        if (mo != Py_None) {
            Ref m(PyObject_GetAttr(mo, names.mask));
            if (!m.p) { PyErr_Clear(); Py_RETURN_NONE; }
            mask = PyLong_AsVoidPtr(m.p);
            if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
        }
        T.d_grad = g.data_ptr(); T.ld_grad = rows[2]; T.grad_dtype = g.scalar_type() == at::kFloat;
        T.mask = static_cast<crisp_mask_t>(mask);
    }
    // (autograd is told that they change, as by any operation in place)
    for (int i = 1; i < 3; ++i)
        for (Py_ssize_t l = 0; l < PyList_GET_SIZE(args[1]); ++l)
            if (PyList_GET_ITEM(args[i], l) != Py_None && PyList_GET_ITEM(args[3], l) != Py_None) {
                const at::Tensor &t = THPVariable_Unpack(PyList_GET_ITEM(args[i], l));
                if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
            }
    crisp_status_t s;
    Py_BEGIN_ALLOW_THREADS
    s = lib_adamw((int32_t)PyList_GET_SIZE(args[1]), arr, params, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(s);
    END_HANDLE_TH_ERRORS
}

// moments(m, m's exponents, sqrt(v), its exponents, stream) -> (status, m, sqrt(v)): the buffers of 8-bit states as flat bf16 tensors
PyObject *moments(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arguments("moments", n, 5)) return nullptr;
    const uint8_t *p[4];
    int64_t count = 0;
    int gpu = 0;
    for (int i = 0; i < 4; ++i) {
        if (!THPVariable_CheckExact(args[i])) { PyErr_SetString(PyExc_TypeError, "moments takes plain tensors"); return nullptr; }
        const at::Tensor &t = THPVariable_Unpack(args[i]);
        p[i] = static_cast<const uint8_t *>(t.data_ptr());
        if (i == 0) { count = t.numel(); gpu = t.get_device(); }
    }
    void *stream = PyLong_AsVoidPtr(args[4]);
    if (PyErr_Occurred()) return nullptr;
    const at::TensorOptions on = at::TensorOptions().dtype(at::kBFloat16).device(at::Device(at::kCUDA, (at::DeviceIndex)gpu));
    at::Tensor m = at::empty_strided({count}, {1}, on), root = at::empty_strided({count}, {1}, on);
    crisp_status_t s;
    Py_BEGIN_ALLOW_THREADS
    s = lib_moments(p[0], p[1], p[2], p[3], count, static_cast<uint16_t *>(m.data_ptr()), static_cast<uint16_t *>(root.data_ptr()), stream);
    Py_END_ALLOW_THREADS
    Ref a(THPVariable_Wrap(std::move(m))), b(THPVariable_Wrap(std::move(root)));
    return a.p && b.p ? Py_BuildValue("lOO", (long)s, a.p, b.p) : nullptr;
    END_HANDLE_TH_ERRORS
}

// encode8(mask, W, rows, k, GPU, buffer, handle that is replaced, stream) -> (status, handle, bytes that the buffer would need), or None: not a plain matrix that
// the call takes.  Where the buffer is too small nothing is done, and the handle is the old one.
PyObject *encode8(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arguments("encode8", n, 8)) return nullptr;
    long long v[8] = {};
    for (int i = 0; i < 8; ++i)
        if (i != 1 && i != 5) {
            v[i] = PyLong_AsLongLong(args[i]);
            if (v[i] == -1 && PyErr_Occurred()) return nullptr;
        }
    const at::Tensor *w = plain(args[1]);
    if (!w || w->scalar_type() != at::kBFloat16 || w->get_device() != v[4] || (w->stride(1) != 1 && w->size(1) != 1) || w->size(0) != v[2] || w->size(1) != v[3])
        Py_RETURN_NONE;
    const crisp_mask_t mask = reinterpret_cast<crisp_mask_t>((uintptr_t)v[0]);
    size_t bytes = 0;
    crisp_status_t s = lib_encode8_sizes(mask, &bytes);
    crisp_handle8_t h = reinterpret_cast<crisp_handle8_t>((uintptr_t)v[6]);          // (kept where nothing is done)
    const at::Tensor *buffer = args[5] != Py_None && THPVariable_CheckExact(args[5]) ? &THPVariable_Unpack(args[5]) : nullptr;
    if (s == CRISP_OK && buffer && (size_t)buffer->numel() >= bytes) {
        const int64_t ld = w->size(0) > 1 ? w->stride(0) : w->size(1);
        Py_BEGIN_ALLOW_THREADS
        lib_destroy8(h);
        h = nullptr;
        s = lib_encode8(static_cast<const uint16_t *>(w->data_ptr()), ld, mask, buffer->data_ptr(), reinterpret_cast<void *>((uintptr_t)v[7]), &h);
        Py_END_ALLOW_THREADS
        bytes = 0;
    }
    return Py_BuildValue("lKK", (long)s, (unsigned long long)(uintptr_t)h, (unsigned long long)bytes);
    END_HANDLE_TH_ERRORS
}

// product8(handle, X, rows, k, GPU, tokens, y_dtype, stream) -> (status, Y), or None: not a plain matrix that the call takes.  Workspace and Y are allocated for the
// current stream, which `stream` has to be.
PyObject *product8(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!arguments("product8", n, 8)) return nullptr;
    long long v[8] = {};
    for (int i = 0; i < 8; ++i)
        if (i != 1) {
            v[i] = PyLong_AsLongLong(args[i]);
            if (v[i] == -1 && PyErr_Occurred()) return nullptr;
        }
    const at::Tensor *x = plain(args[1]);
    const bool tokens = v[5] != 0;
    if (!x || x->scalar_type() != at::kBFloat16 || x->get_device() != v[4] || (x->stride(1) != 1 && x->size(1) != 1) || x->size(tokens ? 1 : 0) != v[3])
        Py_RETURN_NONE;
    const int64_t ncols = x->size(tokens ? 0 : 1), ldx = x->size(0) > 1 ? x->stride(0) : x->size(1), ldy = tokens ? v[2] : ncols;
    const crisp_handle8_t h = reinterpret_cast<crisp_handle8_t>((uintptr_t)v[0]);
    size_t bytes = 0;
    crisp_status_t s = lib_spmm8_sizes(h, ncols, &bytes);
    const at::TensorOptions on = at::TensorOptions().device(at::Device(at::kCUDA, (at::DeviceIndex)v[4]));
    at::Tensor y, act;
    if (s == CRISP_OK) {
        y = at::empty_strided({tokens ? ncols : v[2], ldy}, {ldy, 1}, on.dtype(v[6] ? at::kFloat : at::kBFloat16));
        if (bytes) act = at::empty_strided({(int64_t)bytes}, {1}, on.dtype(at::kByte));
        Py_BEGIN_ALLOW_THREADS
        s = lib_spmm8(h, static_cast<const uint16_t *>(x->data_ptr()), ldx, (int32_t)tokens, ncols, bytes ? act.data_ptr() : nullptr, y.data_ptr(), ldy, (int32_t)tokens,
                      (int32_t)v[6], reinterpret_cast<void *>((uintptr_t)v[7]));
        Py_END_ALLOW_THREADS
    }
    if (s != CRISP_OK) return Py_BuildValue("lO", (long)s, Py_None);
    Ref out(THPVariable_Wrap(std::move(y)));
    return out.p ? Py_BuildValue("lO", (long)s, out.p) : nullptr;
    END_HANDLE_TH_ERRORS
}

// bind(addresses of crisp_decode, crisp_spmm8_sizes, crisp_spmm8, crisp_decode8, crisp_encode8_sizes, crisp_encode8, crisp_destroy8, crisp_adamw and
// crisp_adamw_moments)
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (!arguments("bind", n, 9)) return nullptr;
    lib_adamw = reinterpret_cast<decltype(&crisp_adamw)>(PyLong_AsVoidPtr(args[7]));
    lib_moments = reinterpret_cast<decltype(&crisp_adamw_moments)>(PyLong_AsVoidPtr(args[8]));
    lib_decode8 = reinterpret_cast<decltype(&crisp_decode8)>(PyLong_AsVoidPtr(args[3]));
    lib_encode8_sizes = reinterpret_cast<decltype(&crisp_encode8_sizes)>(PyLong_AsVoidPtr(args[4]));
    lib_encode8 = reinterpret_cast<decltype(&crisp_encode8)>(PyLong_AsVoidPtr(args[5]));
    lib_destroy8 = reinterpret_cast<decltype(&crisp_destroy8)>(PyLong_AsVoidPtr(args[6]));
    lib_decode = reinterpret_cast<decltype(&crisp_decode)>(PyLong_AsVoidPtr(args[0]));
    lib_spmm8_sizes = reinterpret_cast<decltype(&crisp_spmm8_sizes)>(PyLong_AsVoidPtr(args[1]));
    lib_spmm8 = reinterpret_cast<decltype(&crisp_spmm8)>(PyLong_AsVoidPtr(args[2]));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

#define CRISP_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CRISP_METHOD(bind), CRISP_METHOD(table), CRISP_METHOD(encodings), CRISP_METHOD(encoded), CRISP_METHOD(decode), CRISP_METHOD(adamw), CRISP_METHOD(moments), CRISP_METHOD(product8), CRISP_METHOD(encode8), CRISP_METHOD(decode8), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_network", nullptr, 0, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__network(void) {
    names = {PyUnicode_InternFromString("desc"), PyUnicode_InternFromString("mask_buf"), PyUnicode_InternFromString("workspace"),
             PyUnicode_InternFromString("canonical_buf"), PyUnicode_InternFromString("exec_buf"), PyUnicode_InternFromString("mask"),
             PyUnicode_InternFromString("handle"), PyUnicode_InternFromString("kkeep")};
    PyObject *m = PyModule_Create(&module);
    // what the binding compares: the layout of torch's tensors and of Python's objects is that of the headers
#define CRISP_TEXT2(x) #x
#define CRISP_TEXT(x) CRISP_TEXT2(x)
    if (m && PyModule_AddStringConstant(m, "built_for", CRISP_TEXT(TORCH_VERSION_MAJOR) "." CRISP_TEXT(TORCH_VERSION_MINOR) "." CRISP_TEXT(TORCH_VERSION_PATCH)
                                        " " CRISP_TEXT(PY_MAJOR_VERSION) "." CRISP_TEXT(PY_MINOR_VERSION)) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
