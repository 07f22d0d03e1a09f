// The decoder's calls on torch tensors (paper_2601_20309_amd/decode.py): each tensor's type, shape, strides and
// device are looked at here and go into the C ABI's arguments.  In C++ because a step of a model makes two
// such calls per layer: taking eight tensors apart in Python costs 8 us, here 0.3.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <c10/core/AutogradState.h>
#include <c10/hip/HIPStream.h>
#include <hip/hip_runtime_api.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstring>
#include <exception>
#include <initializer_list>
#include <new>

#include "../../include/duplexkv.h"

namespace {

// What a decoder was made for, as decode.py hands it over with every call.
struct Spec {
    kv_decoder *decoder;
    int64_t n_heads, n_kv_heads, dim, max_blocks;
    at::ScalarType x;
    float scale;
    int device;
};

// One call's arguments.  ok falls when something does not fit.
struct Call {
    bool ok = true;
    int device;  // the decoder's: tensors lie there
    explicit Call(const Spec *d) : device(d->device) {}

    const at::Tensor *tensor(PyObject *o)
    {
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) {
            ok = false;
            return nullptr;
        }
        const at::Tensor *t = &THPVariable_Unpack(o);
        if (!t->defined() || !t->is_cuda() || t->layout() != at::kStrided || t->device().index() != device || t->is_neg() ||
            !t->has_storage() || differentiated(*t)) {
            ok = false;
            return nullptr;
        }
        return t;
    }

    // A gradient is asked for, backward or forward (torch.no_grad() leaves the latter).
    static bool differentiated(const at::Tensor &t)
    {
        return (t.requires_grad() && at::GradMode::is_enabled()) ||
               (c10::AutogradState::get_tls_state().get_fw_grad_mode() && t._fw_grad(0).defined());
    }

    // [row, head, dim] of the 16-bit type, the last dimension contiguous
    kv_rows rows(PyObject *o, at::ScalarType x, int64_t n, int64_t heads, int64_t dim)
    {
        kv_rows r = {nullptr, 0, 0};
        const at::Tensor *t = tensor(o);
        if (!t) return r;
        if (t->scalar_type() != x || t->dim() != 3 || t->size(0) != n || t->size(1) != heads || t->size(2) != dim ||
            (dim > 1 && t->stride(2) != 1)) {
            ok = false;
            return r;
        }
        return kv_rows{t->data_ptr(), n > 1 ? t->stride(0) : 0, heads > 1 ? t->stride(1) : 0};
    }

    // [n] or, with m >= 0, [n][m], contiguous
    template <typename T>
    T *plain(PyObject *o, at::ScalarType type, int64_t n, int64_t m = -1)
    {
        const at::Tensor *t = tensor(o);
        if (!t) return nullptr;
        if (t->scalar_type() != type || t->dim() != (m < 0 ? 1 : 2) || t->size(0) != n || (m >= 0 && t->size(1) != m) ||
            !t->is_contiguous()) {
            ok = false;
            return nullptr;
        }
        return (T *)t->data_ptr();
    }

    // [request][max_blocks], rows any distance apart
    const int32_t *table(PyObject *o, int64_t n, int64_t max_blocks, int32_t &stride)
    {
        const at::Tensor *t = tensor(o);
        if (!t || t->scalar_type() != at::kInt || t->dim() != 2 || t->size(0) != n || t->size(1) != max_blocks ||
            (max_blocks > 1 && t->stride(1) != 1) || (n > 1 && (t->stride(0) < max_blocks || t->stride(0) > INT32_MAX))) {
            ok = false;
            return nullptr;
        }
        stride = (int32_t)(n > 1 ? t->stride(0) : max_blocks);
        return (const int32_t *)t->data_ptr();
    }

    int64_t length(PyObject *o, int dims)
    {
        const at::Tensor *t = tensor(o);
        if (!t || t->dim() != dims || t->size(0) > INT32_MAX) {
            ok = false;
            return 0;
        }
        return t->size(0);
    }

    int64_t number(PyObject *o, int64_t lo, int64_t hi)
    {
        const int64_t v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) {
            ok = false;
            return 0;
        }
        if (v < lo || v > hi) ok = false;
        return v;
    }

    // What a call has written has another version, so that a backward pass that saved it says so.  (Inference tensors
    // have no versions.)
    static int written(int rc, std::initializer_list<PyObject *> outputs)
    {
        for (PyObject *o : outputs)
            if (rc == KV_OK && o != Py_None && !THPVariable_Unpack(o).is_inference()) THPVariable_Unpack(o).unsafeGetTensorImpl()->bump_version();
        return rc;
    }

    // None: the current stream of the decoder's device
    void *stream(PyObject *o)
    {
        if (o == Py_None) return (void *)c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream();
        return PyLong_AsVoidPtr(o);
    }
};

template <typename F>
PyObject *result(F &&f)
{
    try {
        const int rc = f();
        if (PyErr_Occurred()) return nullptr;
        return PyLong_FromLong(rc);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "decoder call failed");
    }
    return nullptr;
}

const Spec *spec_of(PyObject *o) { return (const Spec *)PyCapsule_GetPointer(o, "duplexkv.decoder"); }

bool count_is(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) PyErr_Format(PyExc_TypeError, "takes %zd arguments, got %zd", want, n);
    return n == want;
}

void free_spec(PyObject *o) { delete spec_of(o); }

// spec(handle, cache address, n_heads, n_kv_heads, head_dim, max_blocks, x_type, scale)
PyObject *spec(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count_is(n, 8)) return nullptr;
    void *handle = PyLong_AsVoidPtr(a[0]);
    void *cache = PyLong_AsVoidPtr(a[1]);
    const int64_t v[5] = {PyLong_AsLongLong(a[2]), PyLong_AsLongLong(a[3]), PyLong_AsLongLong(a[4]), PyLong_AsLongLong(a[5]),
                          PyLong_AsLongLong(a[6])};
    const double scale = PyFloat_AsDouble(a[7]);
    if (PyErr_Occurred()) return nullptr;
    hipPointerAttribute_t at;
    if (hipPointerGetAttributes(&at, cache) != hipSuccess) {
        PyErr_SetString(PyExc_RuntimeError, "the cache's device is not known");
        return nullptr;
    }
    Spec *s = new (std::nothrow)
        Spec{(kv_decoder *)handle, v[0], v[1], v[2], v[3], v[4] == KV_FP16 ? at::kHalf : at::kBFloat16, (float)scale,
             at.device};
    if (!s) return PyErr_NoMemory();
    PyObject *capsule = PyCapsule_New(s, "duplexkv.decoder", free_spec);
    if (!capsule) delete s;
    return capsule;
}

// put(spec, layer, k, v, table, lens, q, q_out, starts, inv_freq, interleaved, sections, positions, q_norm, k_norm, eps, stream)
PyObject *put(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    if (!count_is(n_args, 17)) return nullptr;
    const Spec *d = spec_of(a[0]);
    if (!d) return nullptr;
    return result([&] {
        Call c(d);
        kv_put_args p;
        memset(&p, 0, sizeof p);
        p.layer = (int32_t)c.number(a[1], INT32_MIN, INT32_MAX);
        const int64_t n = c.length(a[5], 1), rows = c.length(a[2], 3);
        p.n_seqs = (int32_t)n;
        p.n_rows = (int32_t)rows;
        p.k = c.rows(a[2], d->x, rows, d->n_kv_heads, d->dim);
        p.v = c.rows(a[3], d->x, rows, d->n_kv_heads, d->dim);
        p.table = c.table(a[4], n, d->max_blocks, p.table_stride);
        p.lens = c.plain<int32_t>(a[5], at::kInt, n);
        p.q = c.rows(a[6], d->x, rows, d->n_heads, d->dim);
        p.q_out = c.rows(a[7], d->x, rows, d->n_heads, d->dim);
        if ((a[6] == Py_None) != (a[7] == Py_None) || a[3] == Py_None) return KV_EINVAL;
        p.starts = c.plain<int32_t>(a[8], at::kInt, n + 1);
        if (a[9] != Py_None) {
            const int64_t pairs = c.length(a[9], 1);
            p.inv_freq = c.plain<float>(a[9], at::kFloat, pairs);
            p.rot_dim = (int32_t)std::min<int64_t>(2 * pairs, INT32_MAX);
            p.interleaved = PyObject_IsTrue(a[10]);
            p.n_axes = (int32_t)PyTuple_Size(a[11]);
            for (int32_t i = 0; i < p.n_axes && i < 3; i++) p.sections[i] = (int32_t)PyLong_AsLong(PyTuple_GetItem(a[11], i));
            if (const at::Tensor *t = c.tensor(a[12])) {
                if (t->scalar_type() != at::kInt || t->dim() != 2 || t->size(0) != p.n_axes || t->size(1) != rows ||
                    (rows > 1 && t->stride(1) != 1))
                    return KV_EINVAL;
                p.positions = (const int32_t *)t->data_ptr();
                p.position_stride = p.n_axes > 1 ? t->stride(0) : rows;
            }
        } else if (a[12] != Py_None) {
            return KV_EINVAL;
        }
        p.q_norm = c.plain<float>(a[13], at::kFloat, d->dim);
        p.k_norm = c.plain<float>(a[14], at::kFloat, d->dim);
        p.norm_eps = (float)PyFloat_AsDouble(a[15]);
        void *const stream = c.stream(a[16]);
        if (!c.ok || PyErr_Occurred()) return KV_EINVAL;
        return c.written(kv_put(d->decoder, &p, stream), {a[7]});
    });
}

// attend(spec, layer, q, table, lens, out, scale, lse, mass, mass_out, stream)
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    if (!count_is(n_args, 11)) return nullptr;
    const Spec *d = spec_of(a[0]);
    if (!d) return nullptr;
    return result([&] {
        Call c(d);
        kv_attend_args p;
        memset(&p, 0, sizeof p);
        p.layer = (int32_t)c.number(a[1], INT32_MIN, INT32_MAX);
        const int64_t n = c.length(a[4], 1);
        p.n_seqs = (int32_t)n;
        p.q = c.rows(a[2], d->x, n, d->n_heads, d->dim);
        p.table = c.table(a[3], n, d->max_blocks, p.table_stride);
        p.lens = c.plain<int32_t>(a[4], at::kInt, n);
        p.out = c.rows(a[5], d->x, n, d->n_heads, d->dim);
        p.scale = a[6] == Py_None ? d->scale : (float)PyFloat_AsDouble(a[6]);
        p.lse = c.plain<float>(a[7], at::kFloat, n, d->n_heads);
        p.mass = c.plain<float>(a[8], at::kFloat, n, d->max_blocks);
        p.mass_out = a[9] == Py_None ? const_cast<float *>(p.mass) : c.plain<float>(a[9], at::kFloat, n, d->max_blocks);
        p.mass_stride = d->max_blocks;
        void *const stream = c.stream(a[10]);
        if (!c.ok || a[2] == Py_None || a[5] == Py_None || PyErr_Occurred()) return KV_EINVAL;
        return c.written(kv_attend(d->decoder, &p, stream), {a[5], a[7], a[9] == Py_None ? a[8] : a[9]});
    });
}

// attend_rows(spec, layer, q, table, lens, out, starts, causal, scale, lse, stream)
PyObject *attend_rows(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    if (!count_is(n_args, 11)) return nullptr;
    const Spec *d = spec_of(a[0]);
    if (!d) return nullptr;
    return result([&] {
        Call c(d);
        kv_attend_rows_args p;
        memset(&p, 0, sizeof p);
        p.layer = (int32_t)c.number(a[1], INT32_MIN, INT32_MAX);
        const int64_t n = c.length(a[4], 1), rows = c.length(a[2], 3);
        p.n_seqs = (int32_t)n;
        p.n_rows = (int32_t)rows;
        p.q = c.rows(a[2], d->x, rows, d->n_heads, d->dim);
        p.table = c.table(a[3], n, d->max_blocks, p.table_stride);
        p.lens = c.plain<int32_t>(a[4], at::kInt, n);
        p.out = c.rows(a[5], d->x, rows, d->n_heads, d->dim);
        p.starts = c.plain<int32_t>(a[6], at::kInt, n + 1);
        p.causal = PyObject_IsTrue(a[7]);
        p.scale = a[8] == Py_None ? d->scale : (float)PyFloat_AsDouble(a[8]);
        p.lse = c.plain<float>(a[9], at::kFloat, rows, d->n_heads);
        void *const stream = c.stream(a[10]);
        if (!c.ok || a[5] == Py_None || PyErr_Occurred()) return KV_EINVAL;
        return c.written(kv_attend_rows(d->decoder, &p, stream), {a[5], a[9]});
    });
}

// evict(spec, table, lens, mass, budget, n_first, n_last, ids, at, count, table_out, lens_out, mass_out, stream)
PyObject *evict(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    if (!count_is(n_args, 14)) return nullptr;
    const Spec *d = spec_of(a[0]);
    if (!d) return nullptr;
    return result([&] {
        Call c(d);
        kv_evict_args p;
        memset(&p, 0, sizeof p);
        const int64_t n = c.length(a[2], 1);
        p.n_seqs = (int32_t)n;
        p.budget = (int32_t)c.number(a[4], 0, INT32_MAX);
        p.n_first = (int32_t)c.number(a[5], 0, INT32_MAX);
        p.n_last = (int32_t)c.number(a[6], 1, INT32_MAX);
        p.table = c.plain<int32_t>(a[1], at::kInt, n, d->max_blocks);
        p.lens = c.plain<int32_t>(a[2], at::kInt, n);
        p.mass = c.plain<float>(a[3], at::kFloat, n, d->max_blocks);
        const at::Tensor *ids = c.tensor(a[7]);
        if (!ids || ids->dim() != 2 || ids->size(1) > INT32_MAX) return KV_EINVAL;
        p.max_evict = (int32_t)ids->size(1);
        p.evicted_ids = c.plain<int32_t>(a[7], at::kInt, n, p.max_evict);
        p.evicted_at = c.plain<int32_t>(a[8], at::kInt, n, p.max_evict);
        p.n_evicted = c.plain<int32_t>(a[9], at::kInt, n);
        p.table_out = c.plain<int32_t>(a[10] == Py_None ? a[1] : a[10], at::kInt, n, d->max_blocks);
        p.lens_out = c.plain<int32_t>(a[11] == Py_None ? a[2] : a[11], at::kInt, n);
        p.mass_out = c.plain<float>(a[12] == Py_None ? a[3] : a[12], at::kFloat, n, d->max_blocks);
        p.table_stride = (int32_t)d->max_blocks;
        p.mass_stride = d->max_blocks;
        for (int i : {1, 3, 8, 9})
            if (a[i] == Py_None) return KV_EINVAL;
        void *const stream = c.stream(a[13]);
        if (!c.ok || PyErr_Occurred()) return KV_EINVAL;
        return c.written(kv_evict(d->decoder, &p, stream), {a[7], a[8], a[9], a[10] == Py_None ? a[1] : a[10],
                                                            a[11] == Py_None ? a[2] : a[11], a[12] == Py_None ? a[3] : a[12]});
    });
}

PyMethodDef methods[] = {{"spec", (PyCFunction)(void *)spec, METH_FASTCALL, nullptr},
                         {"put", (PyCFunction)(void *)put, METH_FASTCALL, nullptr},
                         {"attend", (PyCFunction)(void *)attend, METH_FASTCALL, nullptr},
                         {"attend_rows", (PyCFunction)(void *)attend_rows, METH_FASTCALL, nullptr},
                         {"evict", (PyCFunction)(void *)evict, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_decode_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__decode_tensors(void) { return PyModule_Create(&module); }
