// The checks of torch tensors and the calls of the KV-cache operators behind kv.py's KV, as a Python extension module.
//
// The C entry points see addresses only, so what the tensors are (device, type, shape, strides) is checked before each
// call: nine tensors of an attention call, which lasts 8 us on the GPU for one token. Read from Python the properties
// took 8 to 10 us a call on the host of a GB300, before the 3 to 5 us of the launches; here about one.
//
// Nothing here links against libjpi.so: kv.py passes the entry points of the library that it has loaded.

#include <Python.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <exception>
#include <stdexcept>
#include <string>

#include "jpi_kv.h"

namespace {

struct Calls {
    int H, K, D, device;
    at::ScalarType dtype;
    decltype(&jpi_kv_append) append;
    decltype(&jpi_kv_attend) attend;
    decltype(&jpi_kv_weigh) weigh;
    decltype(&jpi_kv_evict) evict;
};

// A refused argument: a Python ValueError or TypeError.
struct Refused : std::runtime_error {
    using std::runtime_error::runtime_error;
};
struct Mistyped : std::runtime_error {
    using std::runtime_error::runtime_error;
};

std::string str(at::IntArrayRef s) {
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + ")";
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) throw Mistyped(std::string(name) + " must be a tensor, not " + Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}

int to_int(int64_t n, const char* what) {
    if (n > INT_MAX || n < INT_MIN) throw Refused(std::string(what) + " does not fit 32 bits");
    return (int)n;
}

int int_of(PyObject* o, const char* name) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Mistyped(std::string(name) + " must be an int of 32 bits");
    }
    return to_int(v, name);
}

void check_data(const Calls& c, const char* name, const at::Tensor& t, at::ScalarType dtype) {
    if (!t.is_cuda() || t.get_device() != c.device || t.layout() != at::kStrided)
        throw Refused(std::string(name) + " is a " + c10::str(t.layout()) + " tensor on " + t.device().str() + ", the handle on cuda:" +
                      std::to_string(c.device));
    if (t.scalar_type() != dtype) throw Refused(std::string(name) + " is " + c10::toString(t.scalar_type()) + ", not " + c10::toString(dtype));
}

// The address of a tensor that is taken (and written) as one contiguous block.
template <typename T>
T* whole(const Calls& c, const char* name, PyObject* o, at::IntArrayRef shape, at::ScalarType dtype) {
    const at::Tensor& t = tensor(o, name);
    check_data(c, name, t, dtype);
    if (t.sizes() != shape) throw Refused(std::string(name) + " has shape " + str(t.sizes()) + ", not " + str(shape));
    if (!t.is_contiguous()) throw Refused(std::string(name) + " must be contiguous");
    return static_cast<T*>(t.data_ptr());
}

// New tokens [batch][tokens][heads][D], one row of `stride` elements each; others are copied to such rows.
struct Tokens {
    at::Tensor copy;
    const void* at = nullptr;
    long long stride = 0;
    int64_t B = 0, T = 0;
};
Tokens tokens(const Calls& c, const char* name, PyObject* o, int heads) {
    const at::Tensor& t = tensor(o, name);
    check_data(c, name, t, c.dtype);
    if (t.dim() != 4 || t.size(2) != heads || t.size(3) != c.D)
        throw Refused(std::string(name) + " has shape " + str(t.sizes()) + ", not [batch][tokens][" + std::to_string(heads) + "][" +
                      std::to_string(c.D) + "]");
    Tokens r;
    r.B = t.size(0);
    r.T = t.size(1);
    to_int(r.B, "the batch");
    to_int(r.T, "the number of tokens");
    const at::IntArrayRef s = t.strides();
    const int64_t row = (int64_t)heads * c.D;
    r.stride = r.T > 1 ? s[1] : r.B > 1 ? s[0] : row;
    r.at = t.data_ptr();
    if (s[3] != 1 || (s[2] != c.D && heads > 1) || (r.B > 1 && r.T > 1 && s[0] != r.T * s[1]) || r.stride < row ||
        r.stride * (int64_t)t.element_size() % 16 != 0 || reinterpret_cast<uintptr_t>(r.at) % 16 != 0) {
        r.copy = t.is_contiguous() ? t.clone() : t.contiguous();
        r.at = r.copy.data_ptr();
        r.stride = row;
    }
    return r;
}

// Caches [n][rows][KV heads][D], with `layers` >= 0 [layers] before that; v may be NULL.
jpi_kv_cache cache(const Calls& c, const char* name, PyObject* ok, PyObject* ov, int64_t n, int64_t layers = -1) {
    const at::Tensor& k = tensor(ok, name);
    check_data(c, name, k, c.dtype);
    const at::IntArrayRef s = k.strides(), z = k.sizes();
    jpi_kv_cache r = {};
    r.k = k.data_ptr();
    if (ov) {
        const at::Tensor& v = tensor(ov, name);
        check_data(c, name, v, c.dtype);
        if (v.sizes() != z || v.strides() != s) throw Refused(std::string(name) + ": k and v must be caches of one shape, type and strides");
        r.v = v.data_ptr();
    }
    const size_t d = layers >= 0;
    if (z.size() != 4 + d || z[d] != n || z[d + 2] != c.K || z[d + 3] != c.D || (d && z[0] != layers))
        throw Refused(std::string(name) + " has shape " + str(z) + ", not " + (d ? "[" + std::to_string(layers) + "]" : "") + "[" +
                      std::to_string(n) + "][rows][" + std::to_string(c.K) + "][" + std::to_string(c.D) + "]");
    if (s[d + 3] != 1) throw Refused(std::string(name) + ": a head's elements must be contiguous");
    r.cache_stride = s[d];
    r.row_stride = s[d + 1];
    r.head_stride = s[d + 2];
    r.layer_stride = d ? s[0] : 0;
    r.rows = to_int(z[d + 1], "the number of rows");
    return r;
}

// A cache argument of one tensor (its keys) or of a pair (k, v).
struct Side {
    jpi_kv_cache c = {};
    const jpi_kv_cache* p = nullptr;
    const int* len = nullptr;
    int64_t n = 1;
};
Side side(const Calls& c, const char* name, PyObject* o, const char* len_name, PyObject* len, bool values, int64_t B, int64_t T) {
    Side r;
    if ((o == Py_None) != (len == Py_None)) throw Refused(std::string(name) + " goes with " + len_name);
    if (o == Py_None) return r;
    PyObject *k = o, *v = nullptr;
    if (values) {
        if (!(PyTuple_Check(o) || PyList_Check(o)) || PySequence_Fast_GET_SIZE(o) != 2) throw Mistyped(std::string(name) + " must be a pair (k, v)");
        k = PySequence_Fast_GET_ITEM(o, 0);
        v = PySequence_Fast_GET_ITEM(o, 1);
    }
    const at::Tensor& t = tensor(k, name);
    r.n = T >= 0 ? B : t.dim() > 0 ? t.size(0) : 0;
    to_int(r.n, "the number of caches");
    r.c = cache(c, name, k, v, r.n);
    r.p = &r.c;
    const int64_t own_shape[2] = {B, T};
    r.len = T >= 0 ? whole<int>(c, len_name, len, own_shape, at::kInt) : whole<int>(c, len_name, len, {r.n}, at::kInt);
    return r;
}

// The call itself runs without the interpreter's lock. Its status, or where that is JPI_OK and `result` is given, the result.
template <typename F>
PyObject* status_of(F&& call, const at::Tensor* result = nullptr) {
    jpi_status s;
    Py_BEGIN_ALLOW_THREADS;
    s = call();
    Py_END_ALLOW_THREADS;
    return s == JPI_OK && result ? THPVariable_Wrap(*result) : PyLong_FromLong(s);
}

// Arguments are counted, and no C++ exception leaves an entry.
template <typename F>
PyObject* entry(PyObject* const* a, Py_ssize_t n, Py_ssize_t want, F&& body) {
    try {
        if (n != want) throw Mistyped("takes " + std::to_string(want) + " arguments, not " + std::to_string(n));
        const auto* c = static_cast<const Calls*>(PyCapsule_GetPointer(a[0], "jpi.kv"));
        if (!c) return nullptr;
        jpi_kv_handle* h = a[1] == Py_None ? nullptr : static_cast<jpi_kv_handle*>(PyLong_AsVoidPtr(a[1]));
        void* st = PyLong_AsVoidPtr(a[2]);
        if (PyErr_Occurred()) return nullptr;
        return body(*c, h, st);
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const Mistyped& e) {
        PyErr_SetString(PyExc_TypeError, e.what());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "an unknown C++ exception");
    }
    return nullptr;
}

// (calls, handle, stream, q, k, v, positions, rows, cache_k, cache_v, q_out)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(a, n, 11, [&](const Calls& c, jpi_kv_handle* h, void* st) {
        if (a[3] == Py_None && a[4] == Py_None) throw Refused("neither q nor k is given");
        Tokens t[3];
        const char* const names[3] = {"q", "k", "v"};
        int64_t B = -1, T = -1;
        for (int i = 0; i < 3; ++i) {
            if (a[3 + i] == Py_None) continue;
            t[i] = tokens(c, names[i], a[3 + i], i == 0 ? c.H : c.K);
            if (B < 0) B = t[i].B, T = t[i].T;
            if (t[i].B != B || t[i].T != T)
                throw Refused(std::string(names[i]) + " holds " + std::to_string(t[i].B) + " x " + std::to_string(t[i].T) + " tokens, not " +
                              std::to_string(B) + " x " + std::to_string(T));
        }
        const int64_t lead[2] = {B, T}, heads[4] = {B, T, c.H, c.D};
        const int* pos = whole<int>(c, "positions", a[6], lead, at::kInt);
        const int* row = whole<int>(c, "rows", a[7], lead, at::kInt);
        void* out = a[3] == Py_None ? nullptr : whole<void>(c, "q_out", a[10], heads, c.dtype);
        jpi_kv_cache ca = {};
        const bool k = a[4] != Py_None, v = a[5] != Py_None;
        if (k) {
            if (a[8] == Py_None || (v && a[9] == Py_None)) throw Refused("k and v need the caches they go to");
            ca = cache(c, "the cache", a[8], v ? a[9] : nullptr, B);
        }
        return status_of([&] {
            return c.append(h, t[0].at, t[0].stride, t[1].at, t[1].stride, t[2].at, t[2].stride, pos, row, (int)B, (int)T, out,
                            k ? &ca : nullptr, st);
        });
    });
}

// (calls, handle, stream, q, prefix, prefix_len, own, seen, out, lse)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(a, n, 10, [&](const Calls& c, jpi_kv_handle* h, void* st) {
        const Tokens q = tokens(c, "q", a[3], c.H);
        const Side p = side(c, "prefix", a[4], "prefix_len", a[5], true, q.B, -1), o = side(c, "own", a[6], "seen", a[7], true, q.B, q.T);
        const int64_t heads[4] = {q.B, q.T, c.H, c.D};
        void* out = whole<void>(c, "out", a[8], heads, c.dtype);
        float* lse = whole<float>(c, "lse", a[9], at::IntArrayRef(heads, 3), at::kFloat);
        return status_of([&] { return c.attend(h, q.at, q.stride, (int)q.B, (int)q.T, p.p, (int)p.n, p.len, o.p, o.len, out, lse, st); });
    });
}

// (calls, handle, stream, q, lse, prefix, prefix_len, own, seen, decay, w_prefix, out_prefix, w_own, out_own)
PyObject* weigh(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(a, n, 14, [&](const Calls& c, jpi_kv_handle* h, void* st) -> PyObject* {
        const Tokens q = tokens(c, "q", a[3], c.H);
        const int64_t heads[3] = {q.B, q.T, c.H};
        const float* lse = whole<float>(c, "lse", a[4], heads, at::kFloat);
        const Side s[2] = {side(c, "prefix", a[5], "prefix_len", a[6], false, q.B, -1), side(c, "own", a[7], "seen", a[8], false, q.B, q.T)};
        const double decay = PyFloat_AsDouble(a[9]);
        if (decay == -1.0 && PyErr_Occurred()) return nullptr;
        const float* in[2] = {};
        float* out[2] = {};
        for (int i = 0; i < 2; ++i) {
            PyObject *w = a[10 + 2 * i], *x = a[11 + 2 * i];
            const char* name = i ? "own" : "prefix";
            if (!s[i].p) {
                if (w != Py_None || x != Py_None) throw Refused(std::string("weights of ") + name + " without " + name);
                continue;
            }
            const int64_t shape[3] = {s[i].n, c.K, s[i].c.rows};
            if (w != Py_None) in[i] = whole<float>(c, i ? "w_own" : "w_prefix", w, shape, at::kFloat);
            out[i] = whole<float>(c, i ? "out_own" : "out_prefix", x, shape, at::kFloat);
        }
        return status_of([&] {
            return c.weigh(h, q.at, q.stride, lse, (int)q.B, (int)q.T, s[0].p, (int)s[0].n, s[0].len, s[1].p, s[1].len, (float)decay, in[0],
                           out[0], in[1], out[1], st);
        });
    });
}

// (calls, handle, stream, k, v, w, length, keep, sink, recent, out_k, out_v, out_w, out_length); returns the rows kept
PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(a, n, 14, [&](const Calls& c, jpi_kv_handle* h, void* st) {
        const at::Tensor& k = tensor(a[3], "k");
        if (k.dim() != 5) throw Refused("k has shape " + str(k.sizes()) + ", not [layers][caches][rows][KV heads][head dim]");
        const int64_t L = k.size(0), N = k.size(1);
        const int layers = to_int(L, "the number of layers"), caches = to_int(N, "the number of caches");
        const jpi_kv_cache src = cache(c, "k, v", a[3], a[4], N, L), dst = cache(c, "out_k, out_v", a[10], a[11], N, L);
        const int64_t w_shape[4] = {L, N, c.K, src.rows}, o_shape[4] = {L, N, c.K, dst.rows};
        const float* w = whole<float>(c, "w", a[5], w_shape, at::kFloat);
        const int* length = whole<int>(c, "length", a[6], {N}, at::kInt);
        const int keep = int_of(a[7], "keep"), sink = int_of(a[8], "sink"), recent = int_of(a[9], "recent");
        if (keep < 0 || (keep > src.rows && keep > dst.rows)) throw Refused("keep is " + std::to_string(keep) + " of " + std::to_string(src.rows) + " rows");
        float* w_out = whole<float>(c, "out_w", a[12], o_shape, at::kFloat);
        int* len_out = whole<int>(c, "out_length", a[13], {N}, at::kInt);
        const at::Tensor kept = at::empty({L, N, c.K, keep}, k.options().dtype(at::kInt));
        return status_of(
            [&] {
                return c.evict(h, &src, w, length, layers, caches, keep, sink, recent, &dst, w_out, len_out, static_cast<int*>(kept.data_ptr()), st);
            },
            &kept);
    });
}

// The geometry that calls are checked against: (heads, KV heads, head dim, bf16, device, the four entry points)
PyObject* calls(PyObject*, PyObject* args) {
    int bf16;
    unsigned long long f[4];
    Calls c = {};
    if (!PyArg_ParseTuple(args, "iiipiKKKK", &c.H, &c.K, &c.D, &bf16, &c.device, &f[0], &f[1], &f[2], &f[3])) return nullptr;
    c.dtype = bf16 ? at::kBFloat16 : at::kFloat;
    c.append = reinterpret_cast<decltype(c.append)>(f[0]);
    c.attend = reinterpret_cast<decltype(c.attend)>(f[1]);
    c.weigh = reinterpret_cast<decltype(c.weigh)>(f[2]);
    c.evict = reinterpret_cast<decltype(c.evict)>(f[3]);
    return PyCapsule_New(new Calls(c), "jpi.kv", [](PyObject* o) { delete static_cast<Calls*>(PyCapsule_GetPointer(o, "jpi.kv")); });
}

template <typename F>
PyCFunction fast(F f) {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f));
}
PyMethodDef methods[] = {{"calls", calls, METH_VARARGS, nullptr},
                         {"append", fast(append), METH_FASTCALL, nullptr},
                         {"attend", fast(attend), METH_FASTCALL, nullptr},
                         {"weigh", fast(weigh), METH_FASTCALL, nullptr},
                         {"evict", fast(evict), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__kv() { return PyModule_Create(&module); }
