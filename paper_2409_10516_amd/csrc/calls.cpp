// The calls around a cache in pages from Python, as short as they can be made: they are made once per token and layer, and with few rows the
// device is done before an interpreter has looked at a dozen tensors (a call of ra_attend_paged, us: checks and arguments in Python 5.5, here 0.9,
// the two launches 6.4).
//
// Each function takes the arguments of its namesake in binding.py, all of them, by position, and asks of them what that asks. It makes the call
// and returns what that returns; a status that is not RA_OK it returns as a number. Where anything is not as it should be or out of the ordinary
// (a stream, partial results), it returns None, having done nothing, and the caller goes through the checks in Python, which say what is wrong.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>

#include "ra.h"

namespace {

struct Cache {
    at::Tensor t[3];                // K, V (one may be undefined) and the table, as they were when the cache was checked
    const void* at[3];
    ra_paged_cache c;
    int device;
    at::ScalarType type;
};

PyObject* raw_stream = nullptr;     // device -> handle of its current stream
PyObject* device_number[64];
decltype(&ra_append_tokens_paged) append_call = nullptr;
decltype(&ra_gather_paged) gather_call = nullptr;
decltype(&ra_full_attention_paged) full_call = nullptr;
decltype(&ra_full_attention_paged_workspace_bytes) full_room = nullptr;
decltype(&ra_attend_paged) attend_call = nullptr;
decltype(&ra_attend_paged_workspace_bytes) attend_room = nullptr;

int current_device() { return c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice().index(); }

void drop(PyObject* capsule) { delete static_cast<Cache*>(PyCapsule_GetPointer(capsule, "paged")); }

// what is asked of a call's cache: tensors that are where they were, on the current device. (Tensors that share their memory until they are written to
// get their own here, as they do where Python asks for an address, and are somewhere else then.)
const Cache* cache_of(PyObject* o) {
    const Cache* c = static_cast<const Cache*>(PyCapsule_GetPointer(o, "paged"));
    if (!c || current_device() != c->device) return nullptr;
    for (int i = 0; i < 3; ++i)
        if (c->t[i].defined() && c->t[i].mutable_data_ptr() != c->at[i]) return nullptr;
    return c;
}
bool is(const Cache& c, const at::Tensor& t, at::ScalarType type, at::IntArrayRef shape) {
    return t.is_cuda() && t.device().index() == c.device && t.scalar_type() == type && t.sizes() == shape && t.is_contiguous();
}
// the address of a contiguous tensor of a type and shape on the cache's device, null if it is not one
const void* data(const Cache& c, PyObject* o, at::ScalarType type, at::IntArrayRef shape) {
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return is(c, t, type, shape) ? t.const_data_ptr() : nullptr;
}
// the same of one that is written to, whose memory is its own then
void* place(const Cache& c, PyObject* o, at::ScalarType type, at::IntArrayRef shape) {
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return is(c, t, type, shape) ? t.mutable_data_ptr() : nullptr;
}
// the same, where None will do: false if it is neither
bool maybe(const Cache& c, PyObject* o, at::ScalarType type, at::IntArrayRef shape, const void** at) {
    *at = nullptr;
    return o == Py_None || (*at = data(c, o, type, shape)) != nullptr;
}
at::Tensor make(const Cache& c, at::IntArrayRef shape, at::ScalarType type) {
    return at::empty(shape, at::TensorOptions().dtype(type).device(at::kCUDA, c.device));
}
bool stream_of(const Cache& c, void** st) {
    PyObject* h = PyObject_CallOneArg(raw_stream, device_number[c.device]);
    if (!h) return false;
    *st = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    return !PyErr_Occurred();
}
bool number(PyObject* o, int64_t* v) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &over);
    return over == 0;
}
bool number(PyObject* o, int* v) {
    int64_t x;
    if (!number(o, &x) || x != (int)x) return false;
    *v = (int)x;
    return true;
}

// the workspace: the caller's, or a new one of `need` bytes, which `own` keeps
bool room(const Cache& c, PyObject* o, size_t need, at::Tensor* own, void** at, size_t* have) {
    if (o == Py_None) {
        if (!need) return false;
        *own = make(c, {(int64_t)need}, at::kByte);
        *at = own->mutable_data_ptr();
        *have = need;
        return true;
    }
    if (!THPVariable_Check(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.device().index() != c.device || !t.is_contiguous()) return false;
    *at = t.mutable_data_ptr();
    *have = t.nbytes();
    return true;
}
// out and lse: given or new
struct Results {
    PyObject* given[2];
    at::Tensor made[2];
    float* at[2];
    bool take(const Cache& c, PyObject* out, PyObject* lse, int64_t n_seq, int64_t n_q, int64_t d) {
        given[0] = out;
        given[1] = lse;
        const int64_t shape[3] = {n_seq, n_q, d};
        for (int i = 0; i < 2; ++i) {
            const at::IntArrayRef s(shape, 3 - i);
            if (given[i] == Py_None) made[i] = make(c, s, at::kFloat);
            at[i] = given[i] == Py_None ? made[i].data_ptr<float>() : static_cast<float*>(place(c, given[i], at::kFloat, s));
            if (!at[i]) return false;
        }
        return true;
    }
    PyObject* pair() {
        PyObject* o[2];
        for (int i = 0; i < 2; ++i) o[i] = given[i] == Py_None ? THPVariable_Wrap(made[i]) : Py_NewRef(given[i]);
        PyObject* t = o[0] && o[1] ? PyTuple_Pack(2, o[0], o[1]) : nullptr;
        Py_XDECREF(o[0]);
        Py_XDECREF(o[1]);
        return t;
    }
};
// q [n_seq][n_q][d]: its address, or null
const void* query(const Cache& c, PyObject* o, int64_t* n_q, int64_t* d) {
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.dim() != 3 || t.size(0) != c.c.n_seq) return nullptr;
    *n_q = t.size(1);
    *d = t.size(2);
    return *n_q > 0x7fffffff || *d > 0x7fffffff ? nullptr : data(c, o, c.type, t.sizes());
}

// f, with whatever it throws left to the checks in Python
template <class F>
PyObject* careful(F f) {
    try {
        PyObject* got = f();
        if (got || PyErr_Occurred()) return got;
    } catch (...) {
    }
    PyErr_Clear();
    Py_RETURN_NONE;
}

// (q, cache, n_tokens, N, workspace, out, lse)
PyObject* full(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return careful([&]() -> PyObject* {
        const Cache* c = n == 7 ? cache_of(a[1]) : nullptr;
        int64_t n_q = 0, d = 0, N = 0;
        const void *q, *n_tokens;
        if (!c || !(q = query(*c, a[0], &n_q, &d)) || !maybe(*c, a[2], at::kInt, {c->c.n_seq}, &n_tokens)) return nullptr;
        if (a[3] == Py_None) N = (int64_t)c->c.table_pages * c->c.page;
        else if (!number(a[3], &N)) return nullptr;
        at::Tensor own;
        void *ws, *st;
        size_t have;
        Results r;
        if (!room(*c, a[4], a[4] == Py_None ? full_room((ra_dtype)c->c.dt, c->c.n_seq, (int)n_q, c->c.n_kv_heads, N) : 0, &own, &ws, &have) ||
            !r.take(*c, a[5], a[6], c->c.n_seq, n_q, d) || !stream_of(*c, &st))
            return nullptr;
        ra_status rc;
        Py_BEGIN_ALLOW_THREADS
        rc = full_call(q, &c->c, (int)n_q, N, (int)d, (const int32_t*)n_tokens, ws, have, st, r.at[0], r.at[1]);
        Py_END_ALLOW_THREADS
        return rc == RA_OK ? r.pair() : PyLong_FromLong(rc);
    });
}

// (q, cache, sink, window, ids, n_tokens, n_indexed, N, workspace, out, lse)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return careful([&]() -> PyObject* {
        const Cache* c = n == 11 ? cache_of(a[1]) : nullptr;
        int64_t n_q = 0, d = 0, N = 0;
        int sink, window;
        const void *q, *ids, *n_tokens, *n_indexed;
        if (!c || !(q = query(*c, a[0], &n_q, &d)) || !number(a[2], &sink) || !number(a[3], &window) || !THPVariable_Check(a[4])) return nullptr;
        const at::Tensor& list = THPVariable_Unpack(a[4]);
        if (list.dim() != 3 || list.size(2) > 0x7fffffff) return nullptr;
        const int topk = (int)list.size(2);
        if (!(ids = data(*c, a[4], at::kInt, {c->c.n_seq, n_q, topk})) || !maybe(*c, a[5], at::kInt, {c->c.n_seq}, &n_tokens) ||
            !maybe(*c, a[6], at::kInt, {c->c.n_seq}, &n_indexed))
            return nullptr;
        if (a[7] == Py_None) N = (int64_t)c->c.table_pages * c->c.page;
        else if (!number(a[7], &N)) return nullptr;
        at::Tensor own;
        void *ws, *st;
        size_t have;
        Results r;
        const size_t need = a[8] == Py_None ? attend_room((ra_dtype)c->c.dt, c->c.n_seq, (int)n_q, c->c.n_kv_heads, N, sink, window, topk) : 0;
        if (!room(*c, a[8], need, &own, &ws, &have) || !r.take(*c, a[9], a[10], c->c.n_seq, n_q, d) || !stream_of(*c, &st)) return nullptr;
        ra_status rc;
        Py_BEGIN_ALLOW_THREADS
        rc = attend_call(q, &c->c, (int)n_q, N, (int)d, (const int32_t*)n_tokens, (const int32_t*)n_indexed, sink, window, topk, (const int32_t*)ids, ws,
                         have, st, r.at[0], r.at[1], nullptr, nullptr, nullptr, nullptr);
        Py_END_ALLOW_THREADS
        return rc == RA_OK ? r.pair() : PyLong_FromLong(rc);
    });
}

// heads of tokens [n_seq][T][heads][128], the heads of a token side by side, all tokens equally far apart
struct Tokens {
    const void* at = nullptr;
    int64_t heads = 0, row = 0;
    bool take(const Cache& c, PyObject* o, int64_t* T) {
        if (o == Py_None) return true;
        if (!THPVariable_Check(o)) return false;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.device().index() != c.device || t.scalar_type() != c.type || t.dim() != 4 || t.size(0) != c.c.n_seq || t.size(3) != RA_DIM ||
            (*T >= 0 && t.size(1) != *T))
            return false;
        *T = t.size(1);
        heads = t.size(2);
        // (the stride of a dimension of one element says nothing)
        row = *T > 1 ? t.stride(1) : t.size(0) > 1 ? t.stride(0) : heads * RA_DIM;
        if (t.stride(3) != 1 || (heads > 1 && t.stride(2) != RA_DIM) || (t.size(0) > 1 && t.stride(0) != *T * row)) return false;
        return (at = t.const_data_ptr()) != nullptr;
    }
    static constexpr int64_t RA_DIM = 128;
};

// (q, k, v, first, cache, n_new, q_weight, k_weight, eps, inv_freq, interleaved, rot_scale, q_out)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return careful([&]() -> PyObject* {
        const Cache* c = n == 13 ? cache_of(a[4]) : nullptr;
        if (!c) return nullptr;
        const int64_t n_seq = c->c.n_seq, n_kv = c->c.n_kv_heads;
        Tokens t[3];
        int64_t T = -1;
        for (int i = 0; i < 3; ++i)
            if (!t[i].take(*c, a[i], &T)) return nullptr;
        if (T < 0 || (t[1].at && t[1].heads != n_kv) || (t[2].at && t[2].heads != n_kv) || t[0].heads > 0x7fffffff) return nullptr;
        const void *first, *n_new, *qw, *kw, *freq = nullptr;
        if (!maybe(*c, a[3], at::kInt, {n_seq}, &first) || !maybe(*c, a[5], at::kInt, {n_seq}, &n_new) || !maybe(*c, a[6], c->type, {128}, &qw) ||
            !maybe(*c, a[7], c->type, {128}, &kw))
            return nullptr;
        int64_t rot = 0;
        if (a[9] != Py_None) {
            if (!THPVariable_Check(a[9])) return nullptr;
            rot = 2 * THPVariable_Unpack(a[9]).numel();
            if (rot > 128 || !(freq = data(*c, a[9], at::kFloat, {rot / 2}))) return nullptr;
        }
        if (!PyFloat_CheckExact(a[8]) || !PyFloat_CheckExact(a[11]) || !PyBool_Check(a[10])) return nullptr;
        at::Tensor made;
        void *out = nullptr, *st;
        if (t[0].at) {
            if (a[12] == Py_None) {
                made = make(*c, {n_seq, t[0].heads, T, 128}, c->type);
                if (n_new) made.zero_();
                out = made.mutable_data_ptr();
            } else if (!(out = place(*c, a[12], c->type, {n_seq, t[0].heads, T, 128}))) {
                return nullptr;
            }
        } else if (a[12] != Py_None) {
            return nullptr;
        }
        if (!stream_of(*c, &st)) return nullptr;
        ra_status rc;
        Py_BEGIN_ALLOW_THREADS
        rc = append_call(t[0].at, t[1].at, t[2].at, &c->c, (int)(t[0].at ? t[0].heads : n_kv), T, 128, t[0].row, t[1].row, t[2].row, qw, kw,
                         PyFloat_AS_DOUBLE(a[8]), (const float*)freq, (int)rot, a[10] == Py_True, PyFloat_AS_DOUBLE(a[11]),
                         (const int32_t*)first, (const int32_t*)n_new, st, out);
        Py_END_ALLOW_THREADS
        if (rc != RA_OK) return PyLong_FromLong(rc);
        PyObject* o = made.defined() ? THPVariable_Wrap(made) : Py_NewRef(a[12]);
        PyObject* t1 = o ? PyTuple_Pack(1, o) : nullptr;
        Py_XDECREF(o);
        return t1;
    });
}

// (cache, values, first, rows, out)
PyObject* gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return careful([&]() -> PyObject* {
        const Cache* c = n == 5 ? cache_of(a[0]) : nullptr;
        const void* first;
        int64_t rows = 0;
        if (!c || !PyBool_Check(a[1]) || !maybe(*c, a[2], at::kInt, {c->c.n_seq}, &first)) return nullptr;
        if (a[3] == Py_None) rows = (int64_t)c->c.table_pages * c->c.page;
        else if (!number(a[3], &rows)) return nullptr;
        if (rows < 0) return nullptr;
        const int64_t shape[4] = {c->c.n_seq, c->c.n_kv_heads, rows, 128};
        at::Tensor made;
        void *out, *st;
        if (a[4] == Py_None) out = (made = make(*c, shape, c->type)).mutable_data_ptr();
        else out = place(*c, a[4], c->type, shape);
        if (!out || !stream_of(*c, &st)) return nullptr;
        ra_status rc;
        Py_BEGIN_ALLOW_THREADS
        rc = gather_call(&c->c, a[1] == Py_True, rows, 128, (const int32_t*)first, st, out);
        Py_END_ALLOW_THREADS
        if (rc != RA_OK) return PyLong_FromLong(rc);
        PyObject* o = made.defined() ? THPVariable_Wrap(made) : Py_NewRef(a[4]);
        PyObject* t = o ? PyTuple_Pack(1, o) : nullptr;
        Py_XDECREF(o);
        return t;
    });
}

// (K, V, table, address of the ra_paged_cache, which is copied, device) -> what the calls take as their cache
PyObject* cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) return PyErr_Format(PyExc_TypeError, "cache takes 5 arguments");
    Cache* c = new Cache;
    for (int i = 0; i < 3; ++i) {
        if (THPVariable_Check(a[i])) c->t[i] = THPVariable_Unpack(a[i]);
        c->at[i] = c->t[i].defined() ? c->t[i].mutable_data_ptr() : nullptr;
    }
    if (const void* from = PyLong_AsVoidPtr(a[3])) c->c = *static_cast<const ra_paged_cache*>(from);
    c->device = (int)PyLong_AsLong(a[4]);
    c->type = (c->t[0].defined() ? c->t[0] : c->t[1]).scalar_type();
    if (PyErr_Occurred() || c->device < 0 || c->device >= 64) {
        delete c;
        return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "device out of range");
    }
    return PyCapsule_New(c, "paged", drop);
}

// (a device's current stream, addresses of the six functions)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7) return PyErr_Format(PyExc_TypeError, "bind takes 7 arguments");
    void* at[6];
    for (int i = 0; i < 6; ++i) at[i] = PyLong_AsVoidPtr(a[i + 1]);
    if (PyErr_Occurred()) return nullptr;
    append_call = reinterpret_cast<decltype(append_call)>(at[0]);
    gather_call = reinterpret_cast<decltype(gather_call)>(at[1]);
    full_call = reinterpret_cast<decltype(full_call)>(at[2]);
    full_room = reinterpret_cast<decltype(full_room)>(at[3]);
    attend_call = reinterpret_cast<decltype(attend_call)>(at[4]);
    attend_room = reinterpret_cast<decltype(attend_room)>(at[5]);
    for (int i = 0; i < 64; ++i)
        if (!device_number[i] && !(device_number[i] = PyLong_FromLong(i))) return nullptr;
    Py_XSETREF(raw_stream, Py_NewRef(a[0]));
    Py_RETURN_NONE;
}

#define RA_METHOD(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(NAME)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {RA_METHOD(bind), RA_METHOD(cache), RA_METHOD(append), RA_METHOD(gather), RA_METHOD(full), RA_METHOD(attend), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
