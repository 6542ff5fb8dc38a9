// The shortest calls for Python.
//
// alch_capture_pack: reads its tensors, makes the three small outputs and calls the library, in one call from Python.
// A short prompt's capture is 4 us on the GPU; from Python, seven attributes of each of its 14 tensors, three allocations and a
// ctypes call of eleven arguments took twice as long (one prompt of 317 tokens, six streams: 10.9 us a pass, with this 7.0).
//
// alch_embed_forward: the rows of one token are 1.7 us on the GPU and a launch of 3 to 4 from the host; marshalled in Python the call took
// 6.0 with X given and 7.1 without, with this 4.2 and 5.0.
//
// Records in 8 bits: the entries of their calls, from 18 tensors for six streams, and alch_capture_pack_q8 as a whole (one prompt of 317 tokens: 9.3 us a pass, with this 7.2).
// alch_policy_loss: a few rows are two launches of 3 us each (three of 18953 logits: 9.2 us a pass, with this 7.5).
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stddef.h>
#include <string.h>

#include <cmath>

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>

#include "alch.h"

namespace {

typedef int (*PackFn)(const alch_batch*, const uint8_t*, int32_t, const alch_stream*, int64_t, int32_t*, int32_t*, int32_t*, void*, size_t,
                      void*);
constexpr Py_ssize_t kMost = 64;  // streams of a call that this takes

// A plain tensor in device memory, as strided storage; null: something else, which is the caller's own business.
const at::Tensor* plain(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.layout() == at::kStrided && t.is_cuda() && !t.is_quantized() ? &t : nullptr;
}

// (function, batch, mask, streams, dsts, capacity, sequences, workspace, stream) -> (status, kept_index, cu_kept, n_kept_and_status),
// or None for arguments that it leaves to the caller: other kinds of sequences and tensors, and whatever an error is due for.
PyObject* capture_pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 9, "capture_pack takes nine arguments");
    const at::Tensor *mask = plain(a[2]), *ws = plain(a[7]);
    const bool lists = (PyList_CheckExact(a[3]) || PyTuple_CheckExact(a[3])) && (PyList_CheckExact(a[4]) || PyTuple_CheckExact(a[4]));
    const Py_ssize_t count = lists ? PySequence_Fast_GET_SIZE(a[3]) : 0;
    if (!mask || !ws || !lists || count > kMost || PySequence_Fast_GET_SIZE(a[4]) < count) Py_RETURN_NONE;
    alch_stream words[kMost];
    for (Py_ssize_t k = 0; k < count; ++k) {
        const at::Tensor *s = plain(PySequence_Fast_GET_ITEM(a[3], k)), *d = plain(PySequence_Fast_GET_ITEM(a[4], k));
        if (!s || !d || s->dim() != 2 || s->numel() == 0 || s->stride(1) != 1 || s->stride(0) < 0 || !d->is_contiguous()) Py_RETURN_NONE;
        const size_t size = s->element_size();
        words[k] = alch_stream{s->data_ptr(), d->data_ptr(), (size_t)s->size(1) * size, (size_t)s->stride(0) * size};
    }
    const PackFn fn = reinterpret_cast<PackFn>(PyLong_AsVoidPtr(a[0]));
    const alch_batch* batch = static_cast<const alch_batch*>(PyLong_AsVoidPtr(a[1]));
    const long long capacity = PyLong_AsLongLong(a[5]), n_seqs = PyLong_AsLongLong(a[6]);
    void* stream = PyLong_AsVoidPtr(a[8]);
    if (PyErr_Occurred()) return nullptr;
    const at::TensorOptions ints = at::TensorOptions().dtype(at::kInt).device(mask->device());
    const at::Tensor kept = at::empty({capacity > 1 ? capacity : 1}, ints), cu = at::empty({n_seqs + 1}, ints), status = at::empty({2}, ints);
    const void* m = mask->data_ptr();
    void *p[4] = {kept.data_ptr(), cu.data_ptr(), status.data_ptr(), ws->data_ptr()};
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(batch, static_cast<const uint8_t*>(m), (int32_t)count, words, capacity, static_cast<int32_t*>(p[0]), static_cast<int32_t*>(p[1]),
            static_cast<int32_t*>(p[2]), p[3], (size_t)ws->numel(), stream);
    Py_END_ALLOW_THREADS
    PyObject* out = PyTuple_New(4);
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, PyLong_FromLong(rc));
    PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(kept));
    PyTuple_SET_ITEM(out, 2, THPVariable_Wrap(cu));
    PyTuple_SET_ITEM(out, 3, THPVariable_Wrap(status));
    return out;
    END_HANDLE_TH_ERRORS
}

typedef int (*EmbedFn)(alch_dtype, int32_t, int32_t, int32_t, const int32_t*, const void*, float, void*, void*);

// (function, token_ids, W_embed, scale, X or None, current device, its current stream) -> (status, X), or None as above.
PyObject* embed_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 7, "embed_forward takes seven arguments");
    const at::Tensor *ids = plain(a[1]), *W = plain(a[2]), *given = a[4] == Py_None ? nullptr : plain(a[4]);
    if (!ids || !W || (!given && a[4] != Py_None) || !(PyFloat_CheckExact(a[3]) || PyLong_CheckExact(a[3]))) Py_RETURN_NONE;
    const EmbedFn fn = reinterpret_cast<EmbedFn>(PyLong_AsVoidPtr(a[0]));
    const double scale = PyFloat_AsDouble(a[3]);
    const long long device = PyLong_AsLongLong(a[5]);
    void* stream = PyLong_AsVoidPtr(a[6]);
    if (PyErr_Occurred()) return nullptr;
    const auto type = W->scalar_type();
    if (ids->dim() != 1 || W->dim() != 2 || ids->scalar_type() != at::kInt || (type != at::kBFloat16 && type != at::kFloat)) Py_RETURN_NONE;
    const int64_t tokens = ids->size(0), vocab = W->size(0), hidden = W->size(1);
    const auto fits = [&](const at::Tensor& t) { return t.get_device() == device && t.is_contiguous(); };
    if (!fits(*ids) || !fits(*W) || tokens > INT32_MAX || vocab > INT32_MAX || hidden > INT32_MAX) Py_RETURN_NONE;
    if (given && !(fits(*given) && given->scalar_type() == type && given->dim() == 2 && given->size(0) == tokens && given->size(1) == hidden)) Py_RETURN_NONE;
    const at::Tensor X = given ? *given : at::empty({tokens, hidden}, at::TensorOptions().dtype(type).device(W->device()));
    const int32_t* p = static_cast<const int32_t*>(ids->data_ptr());
    const void* w = W->data_ptr();
    void* x = X.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(type == at::kFloat ? ALCH_F32 : ALCH_BF16, (int32_t)vocab, (int32_t)hidden, (int32_t)tokens, p, w, (float)scale, x, stream);
    Py_END_ALLOW_THREADS
    PyObject* out = PyTuple_New(2);
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, PyLong_FromLong(rc));
    if (given) Py_INCREF(a[4]);
    PyTuple_SET_ITEM(out, 1, given ? a[4] : THPVariable_Wrap(X));
    return out;
    END_HANDLE_TH_ERRORS
}

bool list(PyObject* o) { return PyList_CheckExact(o) || PyTuple_CheckExact(o); }

// The entries of a call on records in 8 bits for tensors of so many rows, 0 < their number <= kMost; false: for the caller to look at.
static_assert(sizeof(alch_q8_stream) == sizeof(alch_q8_tensor), "one layout");
bool read_q8(PyObject* tensors, PyObject* pairs, long long rows, long long device, alch_q8_tensor* of, Py_ssize_t* count, int64_t* held) {
    if (!list(tensors) || !list(pairs)) return false;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(tensors);
    if (n == 0 || n > kMost || PySequence_Fast_GET_SIZE(pairs) != n) return false;
    *count = n;
    *held = -1;
    for (Py_ssize_t k = 0; k < n; ++k) {
        PyObject* pair = PySequence_Fast_GET_ITEM(pairs, k);
        if (!list(pair) || PySequence_Fast_GET_SIZE(pair) != 2) return false;
        const at::Tensor *t = plain(PySequence_Fast_GET_ITEM(tensors, k)), *c = plain(PySequence_Fast_GET_ITEM(pair, 0)), *s = plain(PySequence_Fast_GET_ITEM(pair, 1));
        if (!t || !c || !s || t->dim() != 2 || c->dim() != 2 || s->dim() != 2) return false;
        const int64_t width = c->size(1), groups = (width + ALCH_Q8_GROUP - 1) / ALCH_Q8_GROUP;
        const auto type = t->scalar_type();
        if (*held < 0) *held = c->size(0);
        if (t->size(0) != rows || t->size(1) != width || (width > 1 && t->stride(1) != 1) || (type != at::kBFloat16 && type != at::kFloat) ||
            t->get_device() != device || c->get_device() != device || s->get_device() != device || c->size(0) != *held || c->scalar_type() != at::kChar ||
            !c->is_contiguous() || s->size(0) != *held || s->size(1) != groups || s->scalar_type() != at::kFloat || !s->is_contiguous())
            return false;
        of[k] = alch_q8_tensor{t->data_ptr(), static_cast<const int8_t*>(c->data_ptr()), static_cast<const float*>(s->data_ptr()), width,
                               (size_t)(rows > 1 ? t->stride(0) : width) * t->element_size(), type == at::kFloat ? ALCH_F32 : ALCH_BF16, 0};
    }
    return true;
}

// (tensors, pairs of codes and scales, rows of each tensor, device) -> (the entries of alch_capture_gather_q8 or alch_record_expand, rows of the codes), or
// None as above, where the pairs have different numbers of rows, too.
PyObject* q8_entries(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 4, "q8_entries takes four arguments");
    const long long rows = PyLong_AsLongLong(a[2]), device = PyLong_AsLongLong(a[3]);
    if (PyErr_Occurred()) return nullptr;
    alch_q8_tensor of[kMost];
    Py_ssize_t count;
    int64_t held;
    if (!read_q8(a[0], a[1], rows, device, of, &count, &held)) Py_RETURN_NONE;
    return Py_BuildValue("(y#L)", reinterpret_cast<const char*>(of), (Py_ssize_t)(count * sizeof(of[0])), (long long)held);
    END_HANDLE_TH_ERRORS
}

typedef int (*PackQ8Fn)(const alch_batch*, const uint8_t*, int32_t, const alch_q8_stream*, int64_t, int32_t*, int32_t*, int32_t*, void*, size_t, void*);

// (function, batch, its tokens, its sequences, mask, streams, pairs of codes and scales, capacity or None, workspace, current device, its current stream) ->
// (status, kept_index, cu_kept, n_kept_and_status), or None as above.
PyObject* capture_pack_q8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 11, "capture_pack_q8 takes eleven arguments");
    const PackQ8Fn fn = reinterpret_cast<PackQ8Fn>(PyLong_AsVoidPtr(a[0]));
    const alch_batch* batch = static_cast<const alch_batch*>(PyLong_AsVoidPtr(a[1]));
    const long long tokens = PyLong_AsLongLong(a[2]), n_seqs = PyLong_AsLongLong(a[3]), device = PyLong_AsLongLong(a[9]);
    void* stream = PyLong_AsVoidPtr(a[10]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor *mask = plain(a[4]), *ws = plain(a[8]);
    if (!mask || !ws || mask->get_device() != device || mask->element_size() != 1 || mask->numel() != tokens || !mask->is_contiguous()) Py_RETURN_NONE;
    if (ws->get_device() != device || ws->scalar_type() != at::kByte || !ws->is_contiguous()) Py_RETURN_NONE;
    alch_q8_tensor of[kMost];
    Py_ssize_t count;
    int64_t held;
    if (!read_q8(a[5], a[6], tokens, device, of, &count, &held)) Py_RETURN_NONE;
    if (a[7] != Py_None && !PyLong_CheckExact(a[7])) Py_RETURN_NONE;
    const long long capacity = a[7] == Py_None ? held : PyLong_AsLongLong(a[7]);
    if (PyErr_Occurred()) return nullptr;
    if (capacity < 0 || capacity > held) Py_RETURN_NONE;
    const int64_t rows = capacity > 1 ? capacity : 1, bounds = n_seqs + 1;
    // one allocation: the index, the sequences' counts behind it, then the status
    const at::Tensor out = at::empty({rows + bounds + 2}, at::TensorOptions().dtype(at::kInt).device(mask->device()));
    int32_t* p = static_cast<int32_t*>(out.data_ptr());
    const void *m = mask->data_ptr();
    void* w = ws->data_ptr();
    const size_t bytes = (size_t)ws->numel();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(batch, static_cast<const uint8_t*>(m), (int32_t)count, reinterpret_cast<const alch_q8_stream*>(of), capacity, p, p + rows, p + rows + bounds, w, bytes, stream);
    Py_END_ALLOW_THREADS
    PyObject* result = PyTuple_New(4);
    if (!result) return nullptr;
    PyTuple_SET_ITEM(result, 0, PyLong_FromLong(rc));
    PyTuple_SET_ITEM(result, 1, THPVariable_Wrap(out.narrow(0, 0, rows)));
    PyTuple_SET_ITEM(result, 2, THPVariable_Wrap(out.narrow(0, rows, bounds)));
    PyTuple_SET_ITEM(result, 3, THPVariable_Wrap(out.narrow(0, rows + bounds, 2)));
    return result;
    END_HANDLE_TH_ERRORS
}

typedef int (*PolicyFn)(alch_dtype, int32_t, const void*, int64_t, const alch_policy*, void*, int64_t, float*, void*, size_t, void*);

// (function, logits, items, their device, the pointers of an alch_policy from label on, clip_low, clip_high, kl_coef, whether a gradient is wanted, dlogits,
// logp, loss (each None: a new one), workspace, current device, its current stream) -> (status, loss, logp, dlogits), or None as above.
PyObject* policy_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 15, "policy_loss takes fifteen arguments");
    constexpr Py_ssize_t kPointers = offsetof(alch_policy, logp_out) - offsetof(alch_policy, label);
    const PolicyFn fn = reinterpret_cast<PolicyFn>(PyLong_AsVoidPtr(a[0]));
    const long long items = PyLong_AsLongLong(a[2]), of = PyLong_AsLongLong(a[3]), device = PyLong_AsLongLong(a[13]);
    void* stream = PyLong_AsVoidPtr(a[14]);
    if (PyErr_Occurred()) return nullptr;
    for (int i = 5; i < 8; ++i)
        if (!PyFloat_CheckExact(a[i]) && !PyLong_CheckExact(a[i])) Py_RETURN_NONE;
    const double low = PyFloat_AsDouble(a[5]), high = PyFloat_AsDouble(a[6]), kl = PyFloat_AsDouble(a[7]);
    const int want = PyObject_IsTrue(a[8]);
    if (PyErr_Occurred()) return nullptr;
    for (const double v : {low, high, kl})
        if (std::isinf((float)v) && !std::isinf(v)) Py_RETURN_NONE;  // (no number of 32 bits)
    const at::Tensor *x = plain(a[1]), *ws = plain(a[12]), *given[3];
    for (int i = 0; i < 3; ++i) {
        given[i] = a[9 + i] == Py_None ? nullptr : plain(a[9 + i]);
        if (!given[i] && a[9 + i] != Py_None) Py_RETURN_NONE;
    }
    if (!x || !ws || of != device || !PyBytes_CheckExact(a[4]) || PyBytes_GET_SIZE(a[4]) != kPointers) Py_RETURN_NONE;
    const auto type = x->scalar_type();
    if (x->dim() != 2 || (type != at::kBFloat16 && type != at::kFloat)) Py_RETURN_NONE;
    const int64_t rows = x->size(0), vocab = x->size(1);
    if (rows != items || rows > INT32_MAX || vocab > INT32_MAX || vocab < 1) Py_RETURN_NONE;
    const auto fits = [&](const at::Tensor& t) {
        return t.dim() == 2 && t.get_device() == device && t.scalar_type() == type && t.size(0) == rows && t.size(1) == vocab && (vocab == 1 || t.stride(1) == 1);
    };
    const auto dense = [&](const at::Tensor& t, int64_t size) {
        return t.dim() == 1 && t.size(0) == size && t.scalar_type() == at::kFloat && t.get_device() == device && t.is_contiguous();
    };
    if (!fits(*x) || (given[0] && !fits(*given[0])) || (given[1] && !dense(*given[1], rows)) || (given[2] && !dense(*given[2], 4))) Py_RETURN_NONE;
    if (ws->get_device() != device || ws->scalar_type() != at::kByte || !ws->is_contiguous()) Py_RETURN_NONE;
    const at::TensorOptions options = at::TensorOptions().dtype(at::kFloat).device(x->device());
    at::Tensor grad;
    if (given[0]) grad = *given[0];
    else if (want) grad = at::empty({rows, vocab}, options.dtype(type));
    const at::Tensor logp = given[1] ? *given[1] : at::empty({rows}, options), loss = given[2] ? *given[2] : at::empty({4}, options);
    alch_policy p;
    p.n_items = (int32_t)rows;
    p.clip_low = (float)low;
    p.clip_high = (float)high;
    p.kl_coef = (float)kl;
    memcpy(&p.label, PyBytes_AS_STRING(a[4]), kPointers);
    p.logp_out = static_cast<float*>(logp.data_ptr());
    const void* logits = x->data_ptr();
    void *to = grad.defined() ? grad.data_ptr() : nullptr, *w = ws->data_ptr();
    float* sums = static_cast<float*>(loss.data_ptr());
    const int64_t ld = rows > 1 ? x->stride(0) : vocab, ld_grad = !to ? 0 : rows > 1 ? grad.stride(0) : vocab;
    const size_t bytes = (size_t)ws->numel();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(type == at::kFloat ? ALCH_F32 : ALCH_BF16, (int32_t)vocab, logits, ld, &p, to, ld_grad, sums, w, bytes, stream);
    Py_END_ALLOW_THREADS
    PyObject* result = PyTuple_New(4);
    if (!result) return nullptr;
    const auto out = [&](int i, const at::Tensor& t) {
        if (given[i]) Py_INCREF(a[9 + i]);
        return given[i] ? a[9 + i] : THPVariable_Wrap(t);
    };
    PyTuple_SET_ITEM(result, 0, PyLong_FromLong(rc));
    PyTuple_SET_ITEM(result, 1, out(2, loss));
    PyTuple_SET_ITEM(result, 2, out(1, logp));
    if (grad.defined()) {
        PyTuple_SET_ITEM(result, 3, out(0, grad));
    } else {
        Py_INCREF(Py_None);
        PyTuple_SET_ITEM(result, 3, Py_None);
    }
    return result;
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"capture_pack_q8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(capture_pack_q8)), METH_FASTCALL, nullptr},
                         {"policy_loss", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(policy_loss)), METH_FASTCALL, nullptr},
                         {"q8_entries", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(q8_entries)), METH_FASTCALL, nullptr},
                         {"embed_forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(embed_forward)), METH_FASTCALL, nullptr},
                         {"capture_pack", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(capture_pack)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The layout of at::Tensor is compiled in, and another torch may export the same names: the binding compares torch_build with its own.
PyMODINIT_FUNC PyInit__marshal(void) {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_build", ALCH_TORCH_BUILD) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
