// CPython module `_native`: what a step call does on the host between Python and the C ABI, in one native call.
//
// A program that hands over nested lists of gradient tensors pays per tensor and step: dtype, size, layout and
// address read through Python attributes cost 0.37 us a tensor (95 us for 256 workers with one tensor each, where
// the GPU's part of the step is 5 us), here about 0.02 us.  Arguments, torch's current stream and the call itself add 1 us
// instead of 3.  No arithmetic, no checks beyond those of module.py, nothing kept from one call for the next but the
// buffer that the pointers are written to.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>
#include <exception>
#include <new>
#include <vector>

#include "../../include/desloc.h"

namespace {

// The library is loaded by the ctypes binding; its entry points arrive as addresses.
struct Entry {
    decltype(&desloc_step) step = nullptr;
    decltype(&desloc_step_masked) step_masked = nullptr;
    decltype(&desloc_step_normclip) step_normclip = nullptr;
    decltype(&desloc_step_diag) step_diag = nullptr;
    decltype(&desloc_rel_change) rel_change = nullptr;
    decltype(&desloc_get_diag_norms) diag_norms = nullptr;
    decltype(&desloc_step_host) step_host = nullptr;
    decltype(&desloc_embed) embed = nullptr;
    decltype(&desloc_embed_grad) embed_grad = nullptr;
    decltype(&desloc_embed_grad_bytes) embed_grad_bytes = nullptr;
    decltype(&desloc_clip_grads) clip_grads = nullptr;
    decltype(&desloc_clip_grads_bytes) clip_grads_bytes = nullptr;
    decltype(&desloc_token_logprobs) token_logprobs = nullptr;
    decltype(&desloc_token_logprobs_grad) token_logprobs_grad = nullptr;
} g_entry;

struct Table {
    PyObject_HEAD
    std::vector<int64_t> *numel;
    std::vector<void *> *ptrs;
    Py_ssize_t workers;
};

PyObject *table_new(PyTypeObject *type, PyObject *args, PyObject *) {
    PyObject *numel = nullptr;
    Py_ssize_t workers = 0;
    if (!PyArg_ParseTuple(args, "On", &numel, &workers)) return nullptr;
    PyObject *seq = PySequence_Fast(numel, "numel must be a sequence");
    if (!seq) return nullptr;
    Table *self = reinterpret_cast<Table *>(type->tp_alloc(type, 0));
    bool ok = self != nullptr;
    if (ok) {
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
        self->workers = workers;
        self->numel = new (std::nothrow) std::vector<int64_t>();
        self->ptrs = new (std::nothrow) std::vector<void *>();
        try {
            if (!self->numel || !self->ptrs || workers < 0) throw std::bad_alloc();
            self->ptrs->resize(static_cast<size_t>(n) * workers);
            for (Py_ssize_t i = 0; ok && i < n; ++i) {
                const long long v = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(seq, i));
                ok = !(v == -1 && PyErr_Occurred());
                self->numel->push_back(v);
            }
        } catch (const std::bad_alloc &) {
            PyErr_NoMemory();
            ok = false;
        }
    }
    Py_DECREF(seq);
    if (!ok) {
        Py_XDECREF(reinterpret_cast<PyObject *>(self));
        return nullptr;
    }
    return reinterpret_cast<PyObject *>(self);
}

void table_dealloc(PyObject *o) {
    Table *self = reinterpret_cast<Table *>(o);
    delete self->numel;
    delete self->ptrs;
    Py_TYPE(o)->tp_free(o);
}

bool as_pointer(PyObject *o, void **out) {
    *out = o == Py_None ? nullptr : PyLong_AsVoidPtr(o);
    return !(*out == nullptr && PyErr_Occurred());
}

// fill(nested, kind, where, message) -> address of the pointer array [workers * tensors], row m = worker m.
// kind: 0 = fp32, 1 = bf16.  where: 0 = any device, 1 = host only, 2 + d = CUDA device d only.  A tensor that does not fit raises
// ValueError(message).  Returns None at the first element that is no torch.Tensor: the caller marshals the lists then.
PyObject *table_fill(PyObject *o, PyObject *const *args, Py_ssize_t nargs) {
    Table *self = reinterpret_cast<Table *>(o);
    if (nargs != 4) {
        PyErr_SetString(PyExc_TypeError, "fill(nested, kind, where, message)");
        return nullptr;
    }
    const long kind = PyLong_AsLong(args[1]), where = PyLong_AsLong(args[2]);
    if (PyErr_Occurred()) return nullptr;
    const at::ScalarType want = kind == 1 ? at::kBFloat16 : at::kFloat;
    const Py_ssize_t nt = static_cast<Py_ssize_t>(self->numel->size());
    const size_t room = self->ptrs->size();
    PyObject *rows = PySequence_Fast(args[0], "need one tensor list per worker");
    if (!rows) return nullptr;
    size_t count = 0;
    enum { OK, UNFIT, FOREIGN, FAILED } state = OK;
    try {
        for (Py_ssize_t m = 0; state == OK && m < PySequence_Fast_GET_SIZE(rows); ++m) {
            PyObject *row = PySequence_Fast(PySequence_Fast_GET_ITEM(rows, m), "need one tensor list per worker");
            if (!row) {
                state = FAILED;
                break;
            }
            for (Py_ssize_t k = 0; state == OK && k < nt && k < PySequence_Fast_GET_SIZE(row); ++k) {
                PyObject *item = PySequence_Fast_GET_ITEM(row, k);
                if (!THPVariable_Check(item)) {
                    state = FOREIGN;
                    break;
                }
                const at::Tensor &t = THPVariable_Unpack(item);
                if (t.scalar_type() != want || t.numel() != (*self->numel)[k] || !t.is_contiguous() ||
                    (where == 1 && t.is_cuda()) || (where >= 2 && !(t.is_cuda() && t.get_device() == where - 2))) {
                    state = UNFIT;
                    break;
                }
                if (count < room) (*self->ptrs)[count] = t.data_ptr();
                ++count;
            }
            Py_DECREF(row);
        }
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        state = FAILED;
    }
    Py_DECREF(rows);
    if (state == FAILED) return nullptr;
    if (state == FOREIGN) Py_RETURN_NONE;
    if (state == UNFIT) {
        PyErr_SetObject(PyExc_ValueError, args[3]);
        return nullptr;
    }
    if (count != room) {
        PyErr_SetString(PyExc_ValueError, "need one gradient list per worker");
        return nullptr;
    }
    return PyLong_FromVoidPtr(self->ptrs->data());
}

// set(addresses) -> address of the pointer array, which holds them now: for what fill() leaves to the caller.
PyObject *table_set(PyObject *o, PyObject *list) {
    Table *self = reinterpret_cast<Table *>(o);
    PyObject *seq = PySequence_Fast(list, "addresses must be a sequence");
    if (!seq) return nullptr;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
    bool ok = static_cast<size_t>(n) == self->ptrs->size();
    if (!ok) PyErr_SetString(PyExc_ValueError, "need one address per worker and tensor");
    for (Py_ssize_t i = 0; ok && i < n; ++i) ok = as_pointer(PySequence_Fast_GET_ITEM(seq, i), &(*self->ptrs)[i]);
    Py_DECREF(seq);
    return ok ? PyLong_FromVoidPtr(self->ptrs->data()) : nullptr;
}

PyMethodDef table_methods[] = {
    {"set", table_set, METH_O, nullptr},
    {"fill", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(table_fill)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject table_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

// ---- step calls -----------------------------------------------------------------------------------
bool as_int64(PyObject *o, int64_t *out) {
    PyObject *n = PyNumber_Long(o);
    if (!n) return false;
    *out = PyLong_AsLongLong(n);
    Py_DECREF(n);
    return !(*out == -1 && PyErr_Occurred());
}
bool as_float(PyObject *o, float *out) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) return false;
    *out = static_cast<float>(v);
    return true;
}

// (context, t, lr, clip bound, max_norm, pointer array, device, which) -> sync mask, or a negative status.
// which: 0 = step, 1 = step_normclip, 2 = step_diag.  Runs on torch's current stream of the device.
PyObject *call_step(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    void *ctx = nullptr, *ptrs = nullptr;
    int64_t t = 0, device = 0, which = 0;
    float lr = 0.f, bound = 0.f, max_norm = 0.f;
    if (nargs != 8) {
        PyErr_SetString(PyExc_TypeError, "step(ctx, t, lr, clip_bound, max_norm, grads, device, which)");
        return nullptr;
    }
    if (!as_pointer(args[0], &ctx) || !as_int64(args[1], &t) || !as_float(args[2], &lr) || !as_float(args[3], &bound) ||
        !as_float(args[4], &max_norm) || !as_pointer(args[5], &ptrs) || !as_int64(args[6], &device) ||
        !as_int64(args[7], &which))
        return nullptr;
    const void *const *g = static_cast<const void *const *>(ptrs);
    desloc_ctx *c = static_cast<desloc_ctx *>(ctx);
    uint32_t mask = 0;
    int rc = 0;
    try {
        void *stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
        Py_BEGIN_ALLOW_THREADS
        if (which == 0) rc = g_entry.step(c, t, lr, bound, g, stream, &mask);
        else if (which == 1) rc = g_entry.step_normclip(c, t, lr, bound, max_norm, g, stream, &mask);
        else rc = g_entry.step_diag(c, t, lr, bound, max_norm, g, stream, &mask);
        Py_END_ALLOW_THREADS
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    return PyLong_FromLong(rc == DESLOC_OK ? static_cast<long>(mask) : rc);
}

// (context, mask, lr, clip bound, pointer array, device) -> status
PyObject *call_step_masked(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    void *ctx = nullptr, *ptrs = nullptr;
    int64_t mask = 0, device = 0;
    float lr = 0.f, bound = 0.f;
    if (nargs != 6) {
        PyErr_SetString(PyExc_TypeError, "step_masked(ctx, mask, lr, clip_bound, grads, device)");
        return nullptr;
    }
    if (!as_pointer(args[0], &ctx) || !as_int64(args[1], &mask) || !as_float(args[2], &lr) || !as_float(args[3], &bound) ||
        !as_pointer(args[4], &ptrs) || !as_int64(args[5], &device))
        return nullptr;
    int rc = 0;
    try {
        void *stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
        Py_BEGIN_ALLOW_THREADS
        rc = g_entry.step_masked(static_cast<desloc_ctx *>(ctx), static_cast<uint32_t>(mask), lr, bound,
                                 static_cast<const void *const *>(ptrs), stream);
        Py_END_ALLOW_THREADS
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    return PyLong_FromLong(rc);
}

// (context, t, lr, clip bound, host pointer array, device pointer array, device) -> sync mask, or a negative status
PyObject *call_step_host(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    void *ctx = nullptr, *from = nullptr, *to = nullptr;
    int64_t t = 0, device = 0;
    float lr = 0.f, bound = 0.f;
    if (nargs != 7) {
        PyErr_SetString(PyExc_TypeError, "step_host(ctx, t, lr, clip_bound, host_grads, dev_grads, device)");
        return nullptr;
    }
    if (!as_pointer(args[0], &ctx) || !as_int64(args[1], &t) || !as_float(args[2], &lr) || !as_float(args[3], &bound) ||
        !as_pointer(args[4], &from) || !as_pointer(args[5], &to) || !as_int64(args[6], &device))
        return nullptr;
    uint32_t mask = 0;
    int rc = 0;
    try {
        void *stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
        Py_BEGIN_ALLOW_THREADS
        rc = g_entry.step_host(static_cast<desloc_ctx *>(ctx), t, lr, bound, static_cast<const void *const *>(from),
                               static_cast<void *const *>(to), stream, &mask);
        Py_END_ALLOW_THREADS
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    return PyLong_FromLong(rc == DESLOC_OK ? static_cast<long>(mask) : rc);
}

// A list of n floats.
PyObject *float_list(const float *v, size_t n) {
    PyObject *list = PyList_New(static_cast<Py_ssize_t>(n));
    for (size_t i = 0; list && i < n; ++i) {
        PyObject *f = PyFloat_FromDouble(v[i]);
        if (!f) {
            Py_CLEAR(list);
            break;
        }
        PyList_SET_ITEM(list, static_cast<Py_ssize_t>(i), f);
    }
    return list;
}

// (context, array, pointer array, device, workers) -> list of floats, or a negative status
PyObject *call_rel_change(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    void *ctx = nullptr, *ptrs = nullptr;
    int64_t array = 0, device = 0, workers = 0;
    if (nargs != 5) {
        PyErr_SetString(PyExc_TypeError, "rel_change(ctx, array, then, device, workers)");
        return nullptr;
    }
    if (!as_pointer(args[0], &ctx) || !as_int64(args[1], &array) || !as_pointer(args[2], &ptrs) ||
        !as_int64(args[3], &device) || !as_int64(args[4], &workers))
        return nullptr;
    int rc = 0;
    std::vector<float> out;
    try {
        out.resize(static_cast<size_t>(workers));
        void *stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
        Py_BEGIN_ALLOW_THREADS
        rc = g_entry.rel_change(static_cast<desloc_ctx *>(ctx), static_cast<int32_t>(array),
                                static_cast<const float *const *>(ptrs), out.data(), stream);
        Py_END_ALLOW_THREADS
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    if (rc != DESLOC_OK) return PyLong_FromLong(rc);
    return float_list(out.data(), out.size());
}

// (context, workers, tensors, device) -> ([3][workers][tensors], [3][workers]) as nested lists, or a negative status
PyObject *call_diag_norms(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    void *ctx = nullptr;
    int64_t workers = 0, tensors = 0, device = 0;
    if (nargs != 4) {
        PyErr_SetString(PyExc_TypeError, "diag_norms(ctx, workers, tensors, device)");
        return nullptr;
    }
    if (!as_pointer(args[0], &ctx) || !as_int64(args[1], &workers) || !as_int64(args[2], &tensors) ||
        !as_int64(args[3], &device))
        return nullptr;
    int rc = 0;
    std::vector<float> per, tot;
    try {
        per.resize(static_cast<size_t>(3 * workers * tensors));
        tot.resize(static_cast<size_t>(3 * workers));
        void *stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
        Py_BEGIN_ALLOW_THREADS
        rc = g_entry.diag_norms(static_cast<desloc_ctx *>(ctx), per.data(), tot.data(), stream);
        Py_END_ALLOW_THREADS
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    if (rc != DESLOC_OK) return PyLong_FromLong(rc);
    PyObject *a = PyList_New(3), *b = PyList_New(3);
    bool ok = a && b;
    for (int k = 0; ok && k < 3; ++k) {
        PyObject *rows = PyList_New(static_cast<Py_ssize_t>(workers)), *t = float_list(tot.data() + k * workers, workers);
        ok = rows && t;
        for (int64_t m = 0; ok && m < workers; ++m) {
            PyObject *row = float_list(per.data() + (k * workers + m) * tensors, tensors);
            ok = row != nullptr;
            if (ok) PyList_SET_ITEM(rows, static_cast<Py_ssize_t>(m), row);
        }
        if (ok) {
            PyList_SET_ITEM(a, k, rows);
            PyList_SET_ITEM(b, k, t);
        } else {
            Py_XDECREF(rows);
            Py_XDECREF(t);
        }
    }
    PyObject *both = ok ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    return both;
}

// ---- operators around the step --------------------------------------------------------------------
// Through ctypes these calls cost 18 to 24 us of the host's time, here 4 to 7, the launch included.
// These take what most programs hand over: tensors on the right device, of a known type, in the usual layouts.  For everything else they return
// None, and module.py, which copies, splits or refuses, goes its own way.  A status below 0 comes back as a number.
int value_type(at::ScalarType t) { return t == at::kFloat ? DESLOC_F32 : t == at::kBFloat16 ? DESLOC_BF16 : -1; }
int token_type(at::ScalarType t) { return t == at::kInt ? DESLOC_I32 : t == at::kLong ? DESLOC_I64 : -1; }

const at::Tensor *tensor_on(PyObject *o, int64_t device) {
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.is_cuda() && t.get_device() == device ? &t : nullptr;
}
at::Tensor new_tensor(at::IntArrayRef shape, at::ScalarType type, int64_t device) {
    return at::empty(shape, at::TensorOptions().dtype(type).device(at::Device(at::kCUDA, static_cast<c10::DeviceIndex>(device))));
}
void *stream_of(int64_t device) { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream(); }

// Calls `body`, which returns a new reference (or null with an error set).
template <typename F>
PyObject *guarded(const F &body) {
    try {
        return body();
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// Written behind torch's back: a tensor that autograd has saved is refused in backward() from here on, as after any operation in place.  (Tensors of
// inference mode count no versions.)
void wrote(const at::Tensor &t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// Views of one tensor hold one counter: of some in a row the first one is enough.
bool same_counter(const at::Tensor &a, const at::Tensor &b) {
    const c10::VariableVersion &u = a.unsafeGetTensorImpl()->version_counter(), &v = b.unsafeGetTensorImpl()->version_counter();
    const void *at[2];
    static_assert(sizeof u == sizeof at[0]);   // (a reference to the counter)
    std::memcpy(&at[0], &u, sizeof u);
    std::memcpy(&at[1], &v, sizeof v);
    return at[0] && at[0] == at[1];
}
// The same for a tensor or for those in sequences of sequences, whatever kind of sequence fill() takes.  `last`: the one before, which `o` keeps alive.
void wrote_all(PyObject *o, const at::Tensor *&last, int depth) {
    const bool list = PyList_Check(o) || PyTuple_Check(o);   // (first: torch's check of what is no tensor is slow)
    if (!list && THPVariable_Check(o)) {
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!last || !same_counter(*last, t)) wrote(t);
        last = &t;
        return;
    }
    if (depth == 0 || (!list && !PySequence_Check(o))) return;
    PyObject *items = PySequence_Fast(o, "");
    if (!items) return PyErr_Clear();
    for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(items); ++i) wrote_all(PySequence_Fast_GET_ITEM(items, i), last, depth - 1);
    if (!list) last = nullptr;   // (its items may go with it)
    Py_DECREF(items);
}
void wrote_all(PyObject *o) {
    const at::Tensor *last = nullptr;
    wrote_all(o, last, 2);
}
PyObject *call_wrote(PyObject *, PyObject *o) {
    return guarded([&]() -> PyObject * {
        wrote_all(o);
        Py_RETURN_NONE;
    });
}

// Tokens [workers, ...], dense.
bool worker_tokens(const at::Tensor *t, int64_t workers, desloc_rows *rows, int64_t *n) {
    if (!t || t->dim() < 1 || t->size(0) != workers || token_type(t->scalar_type()) < 0 || !t->is_contiguous()) return false;
    *n = workers ? t->numel() / workers : 0;
    *rows = {t->data_ptr(), token_type(t->scalar_type()), {*n, 1}};
    return true;
}

// (context, tensor, width, workers, tokens, scale, type, device) -> tensor [*tokens, width]
PyObject *call_embed(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    void *ctx = nullptr;
    int64_t tensor = 0, width = 0, workers = 0, type = 0, device = 0, n = 0;
    float scale = 0.f;
    if (nargs != 8) {
        PyErr_SetString(PyExc_TypeError, "embed(ctx, tensor, width, workers, tokens, scale, type, device)");
        return nullptr;
    }
    if (!as_pointer(args[0], &ctx) || !as_int64(args[1], &tensor) || !as_int64(args[2], &width) || !as_int64(args[3], &workers) ||
        !as_float(args[5], &scale) || !as_int64(args[6], &type) || !as_int64(args[7], &device))
        return nullptr;
    return guarded([&]() -> PyObject * {
        const at::Tensor *t = tensor_on(args[4], device);
        desloc_rows tokens;
        if (!worker_tokens(t, workers, &tokens, &n) || (type != DESLOC_F32 && type != DESLOC_BF16) || width < 1) Py_RETURN_NONE;
        c10::SmallVector<int64_t, 4> shape(t->sizes().begin(), t->sizes().end());
        shape.push_back(width);
        const at::Tensor out = new_tensor(shape, type == DESLOC_BF16 ? at::kBFloat16 : at::kFloat, device);
        const desloc_rows rows{out.data_ptr(), static_cast<int32_t>(type), {n * width, width}};
        void *stream = stream_of(device);
        int rc = 0;
        Py_BEGIN_ALLOW_THREADS
        rc = g_entry.embed(static_cast<desloc_ctx *>(ctx), static_cast<int32_t>(tensor), width, &tokens, n, scale, &rows, stream);
        Py_END_ALLOW_THREADS
        return rc == DESLOC_OK ? THPVariable_Wrap(out) : PyLong_FromLong(rc);
    });
}

// (context, tensor, width, workers, tokens, dout, pointers or nested lists, tensors, elements, type, scale, accumulate, device) -> 0
PyObject *call_embed_grad(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    void *ctx = nullptr;
    int64_t tensor = 0, width = 0, workers = 0, tensors = 0, numel = 0, type = 0, accumulate = 0, device = 0, n = 0;
    float scale = 0.f;
    if (nargs != 13) {
        PyErr_SetString(PyExc_TypeError, "embed_grad(ctx, tensor, width, workers, tokens, dout, grads, tensors, elements, type, scale, accumulate, device)");
        return nullptr;
    }
    if (!as_pointer(args[0], &ctx) || !as_int64(args[1], &tensor) || !as_int64(args[2], &width) || !as_int64(args[3], &workers) ||
        !as_int64(args[7], &tensors) || !as_int64(args[8], &numel) || !as_int64(args[9], &type) || !as_float(args[10], &scale) ||
        !as_int64(args[11], &accumulate) || !as_int64(args[12], &device))
        return nullptr;
    return guarded([&]() -> PyObject * {
        desloc_rows tokens;
        const at::Tensor *t = tensor_on(args[4], device), *d = tensor_on(args[5], device);
        if (!worker_tokens(t, workers, &tokens, &n) || !d || value_type(d->scalar_type()) < 0 || !d->is_contiguous() || d->dim() != t->dim() + 1 ||
            d->size(-1) != width || d->sizes().slice(0, t->dim()) != t->sizes())
            Py_RETURN_NONE;
        const desloc_rows rows{d->data_ptr(), value_type(d->scalar_type()), {n * width, width}};
        std::vector<void *> own;
        std::vector<at::Tensor> written;
        void *const *grads = nullptr;
        if (PyLong_Check(args[6])) {
            grads = static_cast<void *const *>(PyLong_AsVoidPtr(args[6]));
        } else {
            if (!PyList_Check(args[6]) || PyList_GET_SIZE(args[6]) != workers) Py_RETURN_NONE;
            own.resize(static_cast<size_t>(workers * tensors), nullptr);
            for (int64_t m = 0; m < workers; ++m) {
                PyObject *row = PyList_GET_ITEM(args[6], m);
                if (!PyList_Check(row) || PyList_GET_SIZE(row) <= tensor) Py_RETURN_NONE;
                const at::Tensor *g = tensor_on(PyList_GET_ITEM(row, tensor), device);
                if (!g || value_type(g->scalar_type()) != type || g->numel() != numel || !g->is_contiguous()) Py_RETURN_NONE;
                own[static_cast<size_t>(m * tensors + tensor)] = g->data_ptr();
                written.push_back(*g);
            }
            grads = own.data();
        }
        const int64_t bytes = g_entry.embed_grad_bytes(static_cast<desloc_ctx *>(ctx), static_cast<int32_t>(tensor), width, n);
        if (bytes < 0) return PyLong_FromLong(static_cast<long>(bytes));
        const at::Tensor work = new_tensor({bytes}, at::kByte, device);
        void *stream = stream_of(device), *at_work = work.data_ptr();
        int rc = 0;
        Py_BEGIN_ALLOW_THREADS
        rc = g_entry.embed_grad(static_cast<desloc_ctx *>(ctx), static_cast<int32_t>(tensor), width, &tokens, n, &rows, scale,
                                static_cast<int32_t>(accumulate), grads, at_work, bytes, stream);
        Py_END_ALLOW_THREADS
        if (rc == DESLOC_OK)
            for (const at::Tensor &g : written) wrote(g);
        return PyLong_FromLong(rc);
    });
}

// (context, max_norm, type, pointers, type of out, pointers of out, workers, device, tensors of out) -> (norms, factors)
PyObject *call_clip_grads(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    void *ctx = nullptr, *from = nullptr, *to = nullptr;
    int64_t type = 0, out_type = 0, workers = 0, device = 0;
    float max_norm = 0.f;
    if (nargs != 9) {
        PyErr_SetString(PyExc_TypeError, "clip_grads(ctx, max_norm, type, grads, out_type, out, workers, device, written)");
        return nullptr;
    }
    if (!as_pointer(args[0], &ctx) || !as_float(args[1], &max_norm) || !as_int64(args[2], &type) || !as_pointer(args[3], &from) ||
        !as_int64(args[4], &out_type) || !as_pointer(args[5], &to) || !as_int64(args[6], &workers) || !as_int64(args[7], &device))
        return nullptr;
    return guarded([&]() -> PyObject * {
        const int64_t bytes = g_entry.clip_grads_bytes(static_cast<desloc_ctx *>(ctx));
        if (bytes < 0) return PyLong_FromLong(static_cast<long>(bytes));
        const at::Tensor norms = new_tensor({workers}, at::kFloat, device), factors = new_tensor({workers}, at::kFloat, device),
                         work = new_tensor({bytes}, at::kByte, device);
        void *stream = stream_of(device), *at_work = work.data_ptr();
        float *at_norms = static_cast<float *>(norms.data_ptr()), *at_factors = static_cast<float *>(factors.data_ptr());
        int rc = 0;
        Py_BEGIN_ALLOW_THREADS
        rc = g_entry.clip_grads(static_cast<desloc_ctx *>(ctx), max_norm, static_cast<int32_t>(type), static_cast<const void *const *>(from),
                                static_cast<int32_t>(out_type), static_cast<void *const *>(to), at_norms, at_factors, at_work, bytes, stream);
        Py_END_ALLOW_THREADS
        if (rc != DESLOC_OK) return PyLong_FromLong(rc);
        wrote_all(args[8]);
        PyObject *n = THPVariable_Wrap(norms), *f = n ? THPVariable_Wrap(factors) : nullptr, *both = f ? PyTuple_Pack(2, n, f) : nullptr;
        Py_XDECREF(n);
        Py_XDECREF(f);
        return both;
    });
}

// Rows of up to two dimensions in front of `last` dimensions.
struct Lead {
    int64_t n[2] = {1, 1};
    bool of(const at::Tensor &t, int64_t last) {
        const int64_t lead = t.dim() - last;
        if (lead < 0 || lead > 2) return false;
        for (int64_t k = 0; k < lead; ++k) n[2 - lead + k] = t.size(k);
        return true;
    }
};
desloc_rows rows_of(const at::Tensor &t, int64_t last, int type) {
    desloc_rows r{t.data_ptr(), type, {0, 0}};
    const int64_t lead = t.dim() - last;
    for (int64_t k = 0; k < lead; ++k) r.stride[2 - lead + k] = t.stride(k);
    return r;
}
bool logit_rows(const at::Tensor *x, const at::Tensor *t, Lead *lead) {
    return x && t && x->dim() >= 1 && value_type(x->scalar_type()) >= 0 && token_type(t->scalar_type()) >= 0 && lead->of(*x, 1) &&
           x->sizes().slice(0, x->dim() - 1) == t->sizes() && x->size(-1) >= 1 && (x->stride(-1) == 1 || x->size(-1) == 1);
}
// A tensor's device where it has one that these calls take.
int64_t cuda_device_of(PyObject *o) {
    if (!THPVariable_Check(o)) return -1;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.is_cuda() ? t.get_device() : -1;
}

// (logits, tokens, entropy, top) -> (logp, lse, entropy, top_ids, top_logp)
PyObject *call_logprobs(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    int64_t top = 0;
    if (nargs != 4) {
        PyErr_SetString(PyExc_TypeError, "token_logprobs(logits, tokens, entropy, top)");
        return nullptr;
    }
    const int with_entropy = PyObject_IsTrue(args[2]);
    if (with_entropy < 0 || !as_int64(args[3], &top)) return nullptr;
    return guarded([&]() -> PyObject * {
        const int64_t device = cuda_device_of(args[0]);
        const at::Tensor *x = device < 0 ? nullptr : tensor_on(args[0], device), *t = device < 0 ? nullptr : tensor_on(args[1], device);
        Lead lead;
        if (!logit_rows(x, t, &lead) || top < 0 || top > DESLOC_MAX_TOP) Py_RETURN_NONE;
        at::Tensor r[5];
        r[0] = new_tensor(t->sizes(), at::kFloat, device);
        r[1] = new_tensor(t->sizes(), at::kFloat, device);
        if (with_entropy) r[2] = new_tensor(t->sizes(), at::kFloat, device);
        if (top > 0) {
            c10::SmallVector<int64_t, 4> shape(t->sizes().begin(), t->sizes().end());
            shape.push_back(top);
            r[3] = new_tensor(shape, at::kLong, device);
            r[4] = new_tensor(shape, at::kFloat, device);
        }
        void *p[5];
        for (int k = 0; k < 5; ++k) p[k] = r[k].defined() ? r[k].data_ptr() : nullptr;
        const desloc_rows logits = rows_of(*x, 1, value_type(x->scalar_type())), tokens = rows_of(*t, 0, token_type(t->scalar_type()));
        void *stream = stream_of(device);
        const int64_t vocab = x->size(-1);
        int rc = 0;
        Py_BEGIN_ALLOW_THREADS
        rc = g_entry.token_logprobs(lead.n[0], lead.n[1], vocab, &logits, &tokens, static_cast<int32_t>(top), static_cast<float *>(p[0]),
                                    static_cast<float *>(p[1]), static_cast<float *>(p[2]), static_cast<int64_t *>(p[3]), static_cast<float *>(p[4]),
                                    static_cast<int>(device), stream);
        Py_END_ALLOW_THREADS
        if (rc != DESLOC_OK) return PyLong_FromLong(rc);
        PyObject *tuple = PyTuple_New(5);
        for (int k = 0; tuple && k < 5; ++k) {
            PyObject *o = r[k].defined() ? THPVariable_Wrap(r[k]) : Py_NewRef(Py_None);
            if (!o) {
                Py_CLEAR(tuple);
                break;
            }
            PyTuple_SET_ITEM(tuple, k, o);
        }
        return tuple;
    });
}

// (logits, tokens, lse, dlogp, entropy, dentropy, out or None) -> out
PyObject *call_logprobs_grad(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    if (nargs != 7) {
        PyErr_SetString(PyExc_TypeError, "token_logprobs_grad(logits, tokens, lse, dlogp, entropy, dentropy, out)");
        return nullptr;
    }
    return guarded([&]() -> PyObject * {
        const int64_t device = cuda_device_of(args[0]);
        const at::Tensor *x = device < 0 ? nullptr : tensor_on(args[0], device), *t = device < 0 ? nullptr : tensor_on(args[1], device);
        Lead lead;
        if (!logit_rows(x, t, &lead)) Py_RETURN_NONE;
        const float *dense[4] = {};
        for (int k = 0; k < 4; ++k) {
            if (k >= 2 && args[2 + k] == Py_None) continue;
            const at::Tensor *d = tensor_on(args[2 + k], device);
            if (!d || d->scalar_type() != at::kFloat || d->sizes() != t->sizes() || !d->is_contiguous()) Py_RETURN_NONE;
            dense[k] = static_cast<const float *>(d->data_ptr());
        }
        if (dense[3] && !dense[2] && t->numel() > 0) Py_RETURN_NONE;
        at::Tensor out;
        if (args[6] == Py_None) {
            out = at::empty_like(*x, at::MemoryFormat::Contiguous);
        } else {
            const at::Tensor *o = tensor_on(args[6], device);
            if (!o || o->scalar_type() != x->scalar_type() || o->sizes() != x->sizes() || (o->stride(-1) != 1 && o->size(-1) > 1)) Py_RETURN_NONE;
            out = *o;
        }
        const desloc_rows logits = rows_of(*x, 1, value_type(x->scalar_type())), tokens = rows_of(*t, 0, token_type(t->scalar_type())),
                          to = rows_of(out, 1, value_type(out.scalar_type()));
        void *stream = stream_of(device);
        const int64_t vocab = x->size(-1);
        int rc = 0;
        Py_BEGIN_ALLOW_THREADS
        rc = g_entry.token_logprobs_grad(lead.n[0], lead.n[1], vocab, &logits, &tokens, dense[0], dense[1], dense[2], dense[3], &to,
                                         static_cast<int>(device), stream);
        Py_END_ALLOW_THREADS
        if (rc == DESLOC_OK && args[6] != Py_None) wrote(out);
        return rc == DESLOC_OK ? THPVariable_Wrap(out) : PyLong_FromLong(rc);
    });
}

// bind(addresses of desloc_step, _step_masked, _step_normclip, _step_diag, _rel_change, _get_diag_norms, _step_host, and of the operators around the
// step: _embed, _embed_grad, _embed_grad_bytes, _clip_grads, _clip_grads_bytes, _token_logprobs, _token_logprobs_grad)
PyObject *bind_entries(PyObject *, PyObject *args) {
    unsigned long long a[14];
    if (!PyArg_ParseTuple(args, "KKKKKKKKKKKKKK", &a[0], &a[1], &a[2], &a[3], &a[4], &a[5], &a[6], &a[7], &a[8], &a[9], &a[10], &a[11], &a[12], &a[13]))
        return nullptr;
    g_entry.step = reinterpret_cast<decltype(g_entry.step)>(a[0]);
    g_entry.step_masked = reinterpret_cast<decltype(g_entry.step_masked)>(a[1]);
    g_entry.step_normclip = reinterpret_cast<decltype(g_entry.step_normclip)>(a[2]);
    g_entry.step_diag = reinterpret_cast<decltype(g_entry.step_diag)>(a[3]);
    g_entry.rel_change = reinterpret_cast<decltype(g_entry.rel_change)>(a[4]);
    g_entry.diag_norms = reinterpret_cast<decltype(g_entry.diag_norms)>(a[5]);
    g_entry.step_host = reinterpret_cast<decltype(g_entry.step_host)>(a[6]);
    g_entry.embed = reinterpret_cast<decltype(g_entry.embed)>(a[7]);
    g_entry.embed_grad = reinterpret_cast<decltype(g_entry.embed_grad)>(a[8]);
    g_entry.embed_grad_bytes = reinterpret_cast<decltype(g_entry.embed_grad_bytes)>(a[9]);
    g_entry.clip_grads = reinterpret_cast<decltype(g_entry.clip_grads)>(a[10]);
    g_entry.clip_grads_bytes = reinterpret_cast<decltype(g_entry.clip_grads_bytes)>(a[11]);
    g_entry.token_logprobs = reinterpret_cast<decltype(g_entry.token_logprobs)>(a[12]);
    g_entry.token_logprobs_grad = reinterpret_cast<decltype(g_entry.token_logprobs_grad)>(a[13]);
    Py_RETURN_NONE;
}

template <typename F>
PyCFunction fast(F f) {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(f));
}

PyMethodDef methods[] = {{"bind", bind_entries, METH_VARARGS, nullptr},
                         {"step", fast(call_step), METH_FASTCALL, nullptr},
                         {"step_masked", fast(call_step_masked), METH_FASTCALL, nullptr},
                         {"step_host", fast(call_step_host), METH_FASTCALL, nullptr},
                         {"diag_norms", fast(call_diag_norms), METH_FASTCALL, nullptr},
                         {"rel_change", fast(call_rel_change), METH_FASTCALL, nullptr},
                         {"wrote", call_wrote, METH_O, nullptr},
                         {"embed", fast(call_embed), METH_FASTCALL, nullptr},
                         {"embed_grad", fast(call_embed_grad), METH_FASTCALL, nullptr},
                         {"clip_grads", fast(call_clip_grads), METH_FASTCALL, nullptr},
                         {"token_logprobs", fast(call_logprobs), METH_FASTCALL, nullptr},
                         {"token_logprobs_grad", fast(call_logprobs_grad), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) {
    table_type.tp_name = "_native.Table";
    table_type.tp_basicsize = sizeof(Table);
    table_type.tp_flags = Py_TPFLAGS_DEFAULT;
    table_type.tp_new = table_new;
    table_type.tp_dealloc = table_dealloc;
    table_type.tp_methods = table_methods;
    if (PyType_Ready(&table_type) < 0) return nullptr;
    PyObject *m = PyModule_Create(&module_def);
    if (!m) return nullptr;
    if (PyModule_AddObjectRef(m, "Table", reinterpret_cast<PyObject *>(&table_type)) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    // This module reads torch's own objects, whose layout is that of one build: module.py compares.
    if (PyModule_AddStringConstant(m, "torch_version", DESLOC_TORCH_VERSION) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
