// The per-iteration calls from Python, for the ordinary case: checks the tensors, makes the output and
// calls the C entry point, without a Python object in between.  What this leaves (subclasses and wrapped
// tensors, anything that is not as the call wants it, modes that watch torch's functions) returns None, and
// the caller goes through binding.py's own checks, which say what is wrong.
//
// A minibatch of a small graph is two kernels of 4 us; through ctypes a call took 7.2 and 8.2 us of the host,
// of which the launch is 3: 1.7 for torch.empty from Python, 1.0 for ctypes, the rest attributes and checks.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/autograd/generated/variable_factories.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include <cstdint>
#include <string>

#include "bifeat.h"

namespace {

using DequantFn = int (*)(void *, const uint8_t *, int64_t, const int64_t *, int64_t, float *, void *);
using CacheWriteFn = decltype(&bifeat_cache_write);
using CacheReadFn = decltype(&bifeat_cache_read);
using CacheAttendFn = decltype(&bifeat_cache_attend);
using AggregateFn = int (*)(void *, const uint8_t *, int64_t, const int64_t *, const void *, int64_t, int64_t, float *,
                            void *);

PyObject *g_device = nullptr, *g_stream = nullptr;  // torch._C._cuda_getDevice, ._cuda_getCurrentRawStream

// `with`: of whose device it has to be
const at::Tensor *tensor(PyObject *o, at::ScalarType a, at::ScalarType b, const at::Tensor *with = nullptr) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.dim() < 1 || t.layout() != at::kStrided) return nullptr;
    if (!t.unsafeGetTensorImpl()->has_storage() || !t.is_contiguous()) return nullptr;
    if (with && t.device() != with->device()) return nullptr;
    return t.scalar_type() == a || t.scalar_type() == b ? &t : nullptr;
}

bool watched() {
    return at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set() ||
           torch::jit::tracer::isTracing();
}

// the current stream's handle, as binding.py asks for it; false with a Python error set, or where `on` is not on the current device
bool stream(void **out, const at::Tensor *on = nullptr) {
    PyObject *device = PyObject_CallNoArgs(g_device);
    if (!device) return false;
    if (on && PyLong_AsLong(device) != on->device().index()) {
        Py_DECREF(device);
        return false;
    }
    PyObject *handle = PyObject_CallOneArg(g_stream, device);
    Py_DECREF(device);
    if (!handle) return false;
    *out = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    return !(*out == nullptr && PyErr_Occurred());
}

// The interpreter runs other threads while this lives: an allocation may wait for the device, or for a lock that
// another thread holds.
struct Released {
    PyThreadState *state = PyEval_SaveThread();
    ~Released() { PyEval_RestoreThread(state); }
    Released() = default;
    Released(const Released &) = delete;
};

at::Tensor rows(const at::Tensor &like, int64_t n, int64_t D) {
    return torch::empty({n, D}, at::TensorOptions().dtype(at::kFloat).device(like.device()));
}

// Returns the output tensor, an error status as an integer, or None (see the top).
PyObject *finish(int status, const at::Tensor &out) {
    return status == 0 ? THPVariable_Wrap(out) : PyLong_FromLong(status);
}

// gather_dequant(address of the entry point, handle, codes, idx, D)
PyObject *gather_dequant(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 5) Py_RETURN_NONE;
    try {
        const at::Tensor *codes = tensor(a[2], at::kByte, at::kByte), *idx = tensor(a[3], at::kLong, at::kLong);
        if (!codes || !idx || watched()) Py_RETURN_NONE;
        auto fn = reinterpret_cast<DequantFn>(PyLong_AsVoidPtr(a[0]));
        void *handle = PyLong_AsVoidPtr(a[1]), *s = nullptr;
        const int64_t D = PyLong_AsLongLong(a[4]);
        if (!fn || !handle || D <= 0 || PyErr_Occurred() || !stream(&s)) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        const int64_t M = idx->size(0), N = codes->size(0);
        const auto *pc = static_cast<const uint8_t *>(codes->data_ptr());
        const auto *pi = static_cast<const int64_t *>(idx->data_ptr());
        at::Tensor out;
        int status;
        {
            Released interpreter;
            out = rows(*codes, M, D);
            status = fn(handle, pc, N, pi, M, static_cast<float *>(out.data_ptr()), s);
        }
        return finish(status, out);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// aggregate(address for 64-bit entries, for 32-bit ones, handle, codes, indptr, indices, D)
PyObject *aggregate(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 7) Py_RETURN_NONE;
    try {
        const at::Tensor *codes = tensor(a[3], at::kByte, at::kByte), *indptr = tensor(a[4], at::kLong, at::kLong),
                         *indices = tensor(a[5], at::kLong, at::kInt);
        if (!codes || !indptr || !indices || indptr->size(0) < 1 || watched()) Py_RETURN_NONE;
        auto fn = reinterpret_cast<AggregateFn>(PyLong_AsVoidPtr(a[indices->scalar_type() == at::kInt ? 1 : 0]));
        void *handle = PyLong_AsVoidPtr(a[2]), *s = nullptr;
        const int64_t D = PyLong_AsLongLong(a[6]);
        if (!fn || !handle || D <= 0 || PyErr_Occurred() || !stream(&s)) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        const int64_t V = indptr->size(0) - 1, E = indices->size(0), N = codes->size(0);
        const auto *pc = static_cast<const uint8_t *>(codes->data_ptr());
        const auto *pp = static_cast<const int64_t *>(indptr->data_ptr());
        const void *pi = indices->data_ptr();
        at::Tensor out;
        int status;
        {
            Released interpreter;
            out = rows(*codes, V, D);
            status = fn(handle, pc, N, pp, pi, V, E, static_cast<float *>(out.data_ptr()), s);
        }
        return finish(status, out);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// ---- the paged cache.  Each call begins with (address of the entry point, handle, page bytes, heads, head_dim), then pages,
// and has tables, lengths, indptr (or None) in a row.  All tensors are of the pages' device, and that is current.

struct Cache {
    void *fn, *handle;
    int64_t page_bytes, heads, d;
    const at::Tensor *pages;
};

bool cache_of(PyObject *const *a, Cache *c) {
    c->fn = PyLong_AsVoidPtr(a[0]);
    c->handle = PyLong_AsVoidPtr(a[1]);
    c->page_bytes = PyLong_AsLongLong(a[2]);
    c->heads = PyLong_AsLongLong(a[3]);
    c->d = PyLong_AsLongLong(a[4]);
    c->pages = tensor(a[5], at::kByte, at::kByte);
    return !PyErr_Occurred() && c->fn && c->handle && c->pages && c->pages->dim() == 2 && c->pages->size(1) == c->page_bytes &&
           !watched();
}

bool batch_of(PyObject *const *a, const Cache &c, int64_t tokens, bifeat_cache_batch *b) {
    const at::Tensor *tables = tensor(a[0], at::kInt, at::kInt, c.pages), *lengths = tensor(a[1], at::kLong, at::kLong, c.pages), *indptr = nullptr;
    if (!tables || !lengths || tables->dim() != 2 || lengths->dim() != 1 || lengths->size(0) != tables->size(0)) return false;
    const int64_t B = tables->size(0);
    if (a[2] != Py_None) {
        indptr = tensor(a[2], at::kLong, at::kLong, c.pages);
        if (!indptr || indptr->dim() != 1 || indptr->size(0) != B + 1) return false;
    }
    *b = {static_cast<const int32_t *>(tables->data_ptr()), tables->size(1), static_cast<const int64_t *>(lengths->data_ptr()),
          indptr ? static_cast<const int64_t *>(indptr->data_ptr()) : nullptr, B, tokens};
    return true;
}

// [tokens, heads, head_dim] of one of the three types, columns next to each other
const at::Tensor *head_rows(PyObject *o, const Cache &c, bifeat_head_rows *r, int32_t *dtype) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.dim() != 3 || t.layout() != at::kStrided || !t.unsafeGetTensorImpl()->has_storage() ||
        t.size(2) != c.d || t.stride(2) != 1 || t.device() != c.pages->device())
        return nullptr;
    const auto type = t.scalar_type();
    if (type != at::kFloat && type != at::kHalf && type != at::kBFloat16) return nullptr;
    *dtype = type == at::kFloat ? BIFEAT_F32 : type == at::kHalf ? BIFEAT_F16 : BIFEAT_BF16;
    *r = {t.data_ptr(), t.stride(0), t.stride(1)};
    return &t;
}

// cache_write(..., pages, k, v, tables, lengths, indptr): the status, or None
PyObject *cache_write(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 11) Py_RETURN_NONE;
    try {
        Cache c;
        bifeat_head_rows k, v;
        bifeat_cache_batch b;
        int32_t dtype, other;
        void *s = nullptr;
        const at::Tensor *tk, *tv;
        if (!cache_of(a, &c) || !(tk = head_rows(a[6], c, &k, &dtype)) || !(tv = head_rows(a[7], c, &v, &other)) || dtype != other ||
            tk->size(1) != c.heads || tv->size(1) != c.heads || tk->size(0) != tv->size(0) || !batch_of(a + 8, c, tk->size(0), &b) ||
            !stream(&s, c.pages)) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        const int64_t count = c.pages->size(0);
        auto *p = static_cast<uint8_t *>(c.pages->data_ptr());
        int status;
        {
            Released interpreter;
            status = reinterpret_cast<CacheWriteFn>(c.fn)(static_cast<bifeat_cache *>(c.handle), p, count, &b, &k, &v, dtype, s);
        }
        return PyLong_FromLong(status);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// cache_read(..., pages, tokens, dtype, tables, lengths, indptr): (k, v), an error status, or None
PyObject *cache_read(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 11) Py_RETURN_NONE;
    try {
        Cache c;
        bifeat_cache_batch b;
        void *s = nullptr;
        const int64_t tokens = PyLong_AsLongLong(a[6]), dtype = PyLong_AsLongLong(a[7]);
        if (PyErr_Occurred() || tokens < 0 || !cache_of(a, &c) || !batch_of(a + 8, c, tokens, &b) || !stream(&s, c.pages)) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        const int64_t count = c.pages->size(0);
        const auto *p = static_cast<const uint8_t *>(c.pages->data_ptr());
        const auto options = at::TensorOptions()
                                 .dtype(dtype == BIFEAT_F32 ? at::kFloat : dtype == BIFEAT_F16 ? at::kHalf : at::kBFloat16)
                                 .device(c.pages->device());
        at::Tensor k, v;
        int status;
        {
            Released interpreter;
            k = torch::empty({tokens, c.heads, c.d}, options);
            v = torch::empty({tokens, c.heads, c.d}, options);
            status = reinterpret_cast<CacheReadFn>(c.fn)(static_cast<bifeat_cache *>(c.handle), p, count, &b, k.data_ptr(), v.data_ptr(),
                                                         (int32_t)dtype, s);
        }
        if (status != 0) return PyLong_FromLong(status);
        PyObject *pk = THPVariable_Wrap(k), *pv = pk ? THPVariable_Wrap(v) : nullptr, *both = pv ? PyTuple_Pack(2, pk, pv) : nullptr;
        Py_XDECREF(pk);
        Py_XDECREF(pv);
        return both;
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// cache_attend(..., pages, q, scale, softcap, window, prefix, slopes, tables, lengths, indptr): the output, an error status, or None
PyObject *cache_attend(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 15) Py_RETURN_NONE;
    try {
        Cache c;
        bifeat_head_rows q;
        bifeat_cache_batch b;
        bifeat_attend_options o{};
        int32_t dtype;
        void *s = nullptr;
        const at::Tensor *tq, *prefix = nullptr, *slopes = nullptr;
        o.scale = (float)PyFloat_AsDouble(a[7]);
        o.softcap = (float)PyFloat_AsDouble(a[8]);
        o.window = PyLong_AsLongLong(a[9]);
        if (PyErr_Occurred() || !cache_of(a, &c) || !(tq = head_rows(a[6], c, &q, &dtype)) || !batch_of(a + 12, c, tq->size(0), &b) ||
            (a[10] != Py_None && (!(prefix = tensor(a[10], at::kLong, at::kLong, c.pages)) || prefix->dim() != 1 || prefix->size(0) != b.sequences)) ||
            (a[11] != Py_None && (!(slopes = tensor(a[11], at::kFloat, at::kFloat, c.pages)) || slopes->dim() != 1 || slopes->size(0) != tq->size(1))) ||
            tq->size(1) > INT32_MAX || (tq->requires_grad() && c10::GradMode::is_enabled()) || !stream(&s, c.pages)) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        if (prefix) o.prefix = static_cast<const int64_t *>(prefix->data_ptr());
        if (slopes) o.slopes = static_cast<const float *>(slopes->data_ptr());
        const int64_t count = c.pages->size(0);
        const auto *p = static_cast<const uint8_t *>(c.pages->data_ptr());
        at::Tensor out;
        int status;
        {
            Released interpreter;
            out = torch::empty(tq->sizes(), at::TensorOptions().dtype(tq->scalar_type()).device(tq->device()));
            status = reinterpret_cast<CacheAttendFn>(c.fn)(static_cast<bifeat_cache *>(c.handle), p, count, &b, &q, (int32_t)tq->size(1), dtype,
                                                           &o, out.data_ptr(), s);
        }
        return finish(status, out);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

PyMethodDef methods[] = {
    {"gather_dequant", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gather_dequant)), METH_FASTCALL, nullptr},
    {"aggregate", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(aggregate)), METH_FASTCALL, nullptr},
    {"cache_write", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_write)), METH_FASTCALL, nullptr},
    {"cache_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_read)), METH_FASTCALL, nullptr},
    {"cache_attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_attend)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
    PyObject *c = PyImport_ImportModule("torch._C");
    if (!c) return nullptr;
    g_device = PyObject_GetAttrString(c, "_cuda_getDevice");
    g_stream = g_device ? PyObject_GetAttrString(c, "_cuda_getCurrentRawStream") : nullptr;
    Py_DECREF(c);
    // (tensors are taken apart by their layout in the torch that this was compiled against)
    PyObject *torch = PyImport_ImportModule("torch");
    PyObject *version = torch ? PyObject_GetAttrString(torch, "__version__") : nullptr;
    PyObject *text = version ? PyObject_Str(version) : nullptr;
    const char *now = text ? PyUnicode_AsUTF8(text) : nullptr;
    const std::string python = std::to_string(PY_MAJOR_VERSION) + "." + std::to_string(PY_MINOR_VERSION) + ".";
    if (now && (std::string(now) != BF_TORCH_VERSION || std::string(Py_GetVersion()).rfind(python, 0) != 0))
        PyErr_Format(PyExc_ImportError, "_calls.so was built for torch %s and Python %sx", BF_TORCH_VERSION, python.c_str());
    Py_XDECREF(text);
    Py_XDECREF(version);
    Py_XDECREF(torch);
    if (PyErr_Occurred()) return nullptr;
    return g_stream ? PyModule_Create(&module) : nullptr;
}
