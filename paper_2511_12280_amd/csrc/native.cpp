// The Python side of the device entry points: turns tensors into device pointers and calls libd3tom.so.  Marshalling only, no
// arithmetic.  A merge-layer step of a short sequence is half a dozen launches of a few microseconds each, and looking up the
// attributes of some thirty tensors in Python and converting sixty arguments took a good part of the time of its kernels: the
// five calls on one crop of 729 tokens took 38.3 us on the host, 33.3 us here (most of what is left are the launches); a first
// pass over new inputs 105 us with its kernels, 79 us here.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/autograd/python_variable.h>
#include <exception>
#include <tuple>
#include <type_traits>
#include <utility>
#include "../../include/d3tom.h"

namespace {

struct PythonError {};         // a Python exception is set

PyObject* refuse() {
    PyErr_SetString(PyExc_ValueError, "device entry points take contiguous tensors on the GPU");
    throw PythonError();
}

// None or a tensor
void* pointer(PyObject* o) {
    if (o == Py_None) return nullptr;
    if (THPVariable_CheckExact(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) refuse();
        return t.data_ptr();
    }
    // subclasses of Tensor: by their own attributes, whatever those do
    auto take = [](PyObject* r) { if (!r) throw PythonError(); return r; };
    auto truth = [&](PyObject* r) { take(r); const int v = PyObject_IsTrue(r); Py_DECREF(r); if (v < 0) throw PythonError(); return v != 0; };
    if (!truth(PyObject_GetAttrString(o, "is_cuda")) || !truth(PyObject_CallMethod(o, "is_contiguous", nullptr))) refuse();
    PyObject* a = take(PyObject_CallMethod(o, "data_ptr", nullptr));
    void* p = PyLong_AsVoidPtr(a);
    Py_DECREF(a);
    if (!p && PyErr_Occurred()) throw PythonError();
    return p;
}

// a stream's handle: None or an integer; the last argument of every entry point, and the only address taken as it is
void* stream(PyObject* o) {
    if (o == Py_None) return nullptr;
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw PythonError();
    return p;
}

template <typename T> struct Arg;
template <typename T> struct Arg<T*> { static T* get(PyObject* o) { return static_cast<T*>(pointer(o)); } };
template <> struct Arg<int> {
    static int get(PyObject* o) {
        const unsigned long v = PyLong_AsUnsignedLongMask(o);  // the low 32 bits, as ctypes takes a C int
        if (v == (unsigned long)-1 && PyErr_Occurred()) throw PythonError();
        return (int)(unsigned)v;
    }
};
template <> struct Arg<size_t> {
    static size_t get(PyObject* o) {
        const size_t v = PyLong_AsSize_t(o);
        if (v == (size_t)-1 && PyErr_Occurred()) throw PythonError();
        return v;
    }
};
template <> struct Arg<float> {
    static float get(PyObject* o) {
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) throw PythonError();
        return (float)v;
    }
};

// None, or a host struct by its buffer (ctypes structures have one)
template <typename S>
struct HostStruct {
    static const S* get(PyObject* o) {
        if (o == Py_None) return nullptr;
        Py_buffer view;
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw PythonError();
        const void* p = view.buf;
        const bool fits = view.len == (Py_ssize_t)sizeof(S);
        PyBuffer_Release(&view);                               // the caller holds the object while the call runs
        if (!fits) { PyErr_SetString(PyExc_ValueError, "a host struct of another size"); throw PythonError(); }
        return static_cast<const S*>(p);
    }
};

template <typename T> struct Type { using type = T; };

template <typename... A, size_t... I>
int call(int (*fn)(A...), PyObject* const* args, std::index_sequence<I...>) {
    constexpr size_t last = sizeof...(A) - 1;
    auto take = [&](auto type, size_t i) {
        using T = typename decltype(type)::type;
        if constexpr (std::is_same_v<T, void*>) { if (i == last) return stream(args[i]); }
        return Arg<T>::get(args[i]);
    };
    const std::tuple<A...> a{take(Type<A>{}, I)...};           // in order
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = fn(std::get<I>(a)...);
    Py_END_ALLOW_THREADS
    return status;
}

// the entry point's status as a Python int
template <typename... A>
PyObject* enter(int (*fn)(A...), PyObject* const* args, Py_ssize_t n) {
    if (n != (Py_ssize_t)sizeof...(A)) return PyErr_Format(PyExc_TypeError, "%zd arguments, the entry point takes %zd", n, (Py_ssize_t)sizeof...(A));
    try {
        return PyLong_FromLong(call(fn, args, std::index_sequence_for<A...>()));
    } catch (const PythonError&) {
        return nullptr;
    } catch (const std::exception& e) {                        // a tensor without storage
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define D3TOM_ENTRY(NAME) \
    PyObject* py_##NAME(PyObject*, PyObject* const* args, Py_ssize_t n) { return enter(&NAME, args, n); }
D3TOM_ENTRY(d3tom_importance)
D3TOM_ENTRY(d3tom_importance_static)
D3TOM_ENTRY(d3tom_select_topk)
D3TOM_ENTRY(d3tom_merge)
D3TOM_ENTRY(d3tom_merge_kv)
D3TOM_ENTRY(d3tom_merge_layer)
D3TOM_ENTRY(d3tom_attend)
D3TOM_ENTRY(d3tom_attend_weighted)
D3TOM_ENTRY(d3tom_update_deciders)
D3TOM_ENTRY(d3tom_rmsnorm)
D3TOM_ENTRY(d3tom_rope)
D3TOM_ENTRY(d3tom_linear)
D3TOM_ENTRY(d3tom_linear_tile)
#undef D3TOM_ENTRY


// ---- the paged cache: tensors whose sizes and types are looked up and checked here (a step of one token is launches of 3 us; checked in Python, the rotation and the
// appending took 5.0 and 6.5 us on the host, 3.9 so) ----
struct Checked {
    PyObject* const* args;
    Py_ssize_t n, next = 0;
    int device = -1;
    static void need(bool ok, const char* what) {
        if (!ok) { PyErr_SetString(PyExc_ValueError, what); throw PythonError(); }
    }
    PyObject* arg() { return args[next++]; }
    bool none() const { return args[next] == Py_None; }
    // a tensor, on the device of those before it
    const at::Tensor& tensor() {
        PyObject* o = arg();
        need(THPVariable_Check(o), "a tensor is missing");
        const at::Tensor& t = THPVariable_Unpack(o);
        need(t.is_cuda(), "device entry points take contiguous tensors on the GPU");
        const int d = t.get_device();
        need(device < 0 || d == device, "the tensors of a call lie on different devices");
        device = d;
        return t;
    }
    struct Rows { const void* p = nullptr; int64_t stride = 0, rows = 0, heads = 1, dh = 0; at::ScalarType type = at::kFloat; };
    // [rows, heads, dh]: rows may lie apart unless `packed`; or None
    Rows rows(bool packed) {
        Rows r;
        if (none()) { ++next; return r; }
        const at::Tensor& t = tensor();
        need(t.dim() == 3 && (t.size(2) <= 1 || t.stride(2) == 1) && (t.size(1) <= 1 || t.stride(1) == t.size(2)), "rows of heads on the GPU, contiguous inside a row");
        r.p = t.data_ptr(); r.rows = t.size(0); r.heads = t.size(1); r.dh = t.size(2); r.type = t.scalar_type();
        r.stride = r.rows > 1 ? t.stride(0) : r.heads * r.dh;
        need(!packed || r.stride == r.heads * r.dh, "the output's rows have to be contiguous");
        need(r.rows < (1ll << 31) && r.heads < (1ll << 31) && r.dh < (1ll << 31), "sizes beyond 32 bits");
        need(r.type == at::kFloat || r.type == at::kBFloat16, "unsupported element type");
        return r;
    }
    Rows like(const Rows& x) {                                 // a packed output of x's shape and type
        const Rows r = rows(true);
        need(r.p && r.rows == x.rows && r.heads == x.heads && r.dh == x.dh && r.type == x.type, "an output has another shape or type than its input");
        return r;
    }
    // at least `count` entries of a type, contiguous; or None
    template <typename P> P* list(at::ScalarType type, int64_t count) {
        if (none()) { ++next; return nullptr; }
        const at::Tensor& t = tensor();
        need(t.is_contiguous() && t.scalar_type() == type && t.numel() >= count, "an array has another type or too few entries");
        return static_cast<P*>(t.data_ptr());
    }
    // [B, slots]; all of a call have as many slots
    template <typename P> P* slots(at::ScalarType type, int64_t B, int64_t& stride) {
        if (none()) { ++next; return nullptr; }
        const at::Tensor& t = tensor();
        need(t.is_contiguous() && t.scalar_type() == type && t.dim() == 2 && t.size(0) == B && (stride == 0 || t.size(1) == stride) && t.size(1) < (1ll << 31),
             "arrays of slots are [samples, slots], all with as many slots");
        stride = t.size(1);
        return static_cast<P*>(t.data_ptr());
    }
    template <typename S> const S* host() { return HostStruct<S>::get(arg()); }
    int integer() { return Arg<int>::get(arg()); }
    void* workspace(size_t& bytes) {
        const at::Tensor& t = tensor();
        need(t.is_contiguous(), "device entry points take contiguous tensors on the GPU");
        bytes = (size_t)t.numel() * t.element_size();
        return t.data_ptr();
    }
    // the stream's handle and its device
    void* on_stream() {
        void* s = stream(arg());
        need(integer() == device, "the tensors of a call do not lie on its stream's device");
        return s;
    }
    static int dt(at::ScalarType t) { return t == at::kBFloat16 ? D3TOM_BF16 : D3TOM_F32; }
};
template <typename F>
PyObject* checked(PyObject* const* args, Py_ssize_t n, Py_ssize_t takes, F&& body) {
    if (n != takes) return PyErr_Format(PyExc_TypeError, "%zd arguments, the entry point takes %zd", n, takes);
    try {
        Checked c{args, n};
        return PyLong_FromLong(body(c));
    } catch (const PythonError&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}
#define D3TOM_CALL(STATUS, ...) \
    int STATUS; Py_BEGIN_ALLOW_THREADS STATUS = __VA_ARGS__; Py_END_ALLOW_THREADS

// q, k, axes, rows and device of their positions, q_out, k_out, stream, its device
PyObject* py_d3tom_rope_axes(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return checked(args, n, 9, [](Checked& c) {
        const Checked::Rows q = c.rows(false), k = c.rows(false), &t = q.p ? q : k;
        const d3tom_axes* axes = c.host<d3tom_axes>();
        const int pos_rows = c.integer(), pos_device = c.integer();
        Checked::need(!t.p || (pos_rows >= t.rows && pos_device == c.device), "the positions are fewer than the rows, or lie on another device");
        Checked::need(!q.p || !k.p || (q.rows == k.rows && q.dh == k.dh && q.type == k.type), "queries and keys differ in rows, channels or type");
        Checked::Rows qo, ko;
        if (q.p) qo = c.like(q); else ++c.next;
        if (k.p) ko = c.like(k); else ++c.next;
        void* st = t.p ? c.on_stream() : nullptr;
        D3TOM_CALL(status, d3tom_rope_axes(q.p, q.stride, k.p, k.stride, Checked::dt(t.type), (int)t.rows, (int)q.heads, (int)k.heads, (int)t.dh, axes, (void*)qo.p, (void*)ko.p, st));
        return status;
    });
}
// cache, its device, k, v, new_off, max_new, axes, rows and device of their positions, q, q_out, tokens, slot_token, slot_weight, stream, its device
PyObject* py_d3tom_cache_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return checked(args, n, 16, [](Checked& c) {
        const d3tom_paged_cache* cache = c.host<d3tom_paged_cache>();
        Checked::need(cache != nullptr, "a cache is missing");
        c.device = c.integer();
        const Checked::Rows k = c.rows(false), v = c.rows(false);
        Checked::need(k.p && v.p && k.rows == v.rows && k.heads == cache->Hkv && v.heads == cache->Hkv && k.dh == cache->dh && v.dh == cache->dh &&
                      Checked::dt(k.type) == cache->dt && Checked::dt(v.type) == cache->dt, "keys and values are [rows, Hkv, dh] of the cache's type");
        const int32_t* off = c.list<int32_t>(at::kInt, (int64_t)cache->B + 1);
        const int max_new = c.integer();
        const d3tom_axes* axes = c.host<d3tom_axes>();
        const int pos_rows = c.integer(), pos_device = c.integer();
        Checked::need(!axes || (pos_rows >= k.rows && pos_device == c.device), "the positions are fewer than the rows, or lie on another device");
        const Checked::Rows q = c.rows(false);
        Checked::need(!q.p || (q.rows == k.rows && q.dh == k.dh && q.type == k.type), "queries and keys differ in rows, channels or type");
        Checked::Rows qo;
        if (q.p) qo = c.like(q); else ++c.next;
        const int32_t* tokens = c.list<int32_t>(at::kInt, k.rows);
        int64_t stride = 0;
        int32_t* slot_token = c.slots<int32_t>(at::kInt, cache->B, stride);
        float* slot_weight = c.slots<float>(at::kFloat, cache->B, stride);
        void* st = c.on_stream();
        D3TOM_CALL(status, d3tom_cache_append(cache, k.p, k.stride, v.p, v.stride, off, (int)k.rows, max_new, axes, q.p, q.stride, (int)q.heads, (void*)qo.p, tokens, slot_token,
                                              slot_weight, (int)stride, st));
        return status;
    });
}
// q, cache, its device, q_off, max_q, max_len, scale, causal, o, lse, weight_in, weight_out, ws, stream, its device
PyObject* py_d3tom_attend_cache(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return checked(args, n, 15, [](Checked& c) {
        const Checked::Rows q = c.rows(false);
        const d3tom_paged_cache* cache = c.host<d3tom_paged_cache>();
        Checked::need(cache != nullptr, "a cache is missing");
        Checked::need(c.integer() == c.device, "the tensors of a call lie on different devices");
        Checked::need(q.p && q.dh == cache->dh && Checked::dt(q.type) == cache->dt, "queries are [rows, H, dh] of the cache's type");
        const int32_t* off = c.list<int32_t>(at::kInt, (int64_t)cache->B + 1);
        const int max_q = c.integer(), max_len = c.integer();
        const float scale = Arg<float>::get(c.arg());
        const int causal = c.integer();
        const Checked::Rows o = c.like(q);
        float* lse = c.list<float>(at::kFloat, q.rows * q.heads);
        int64_t stride = 0;
        const float* w_in = c.slots<float>(at::kFloat, cache->B, stride);
        float* w_out = c.slots<float>(at::kFloat, cache->B, stride);
        size_t ws_bytes;
        void* ws = c.workspace(ws_bytes);
        void* st = c.on_stream();
        D3TOM_CALL(status, d3tom_attend_cache(q.p, q.stride, cache, off, (int)q.rows, max_q, max_len, (int)q.heads, scale, causal, (void*)o.p, lse, w_in, w_out, (int)stride, ws,
                                              ws_bytes, st));
        return status;
    });
}
// cache, its device, max_len, keep, first, recent, weight_in, token_in, weight_out, token_out, len_out, ws, src, stream, its device
PyObject* py_d3tom_cache_evict(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return checked(args, n, 15, [](Checked& c) {
        const d3tom_paged_cache* cache = c.host<d3tom_paged_cache>();
        Checked::need(cache != nullptr, "a cache is missing");
        c.device = c.integer();
        const int max_len = c.integer();
        const int32_t* keep = c.list<int32_t>(at::kInt, cache->B);
        const int first = c.integer(), recent = c.integer();
        int64_t stride = 0;
        const float* w_in = c.slots<float>(at::kFloat, cache->B, stride);
        const int32_t* t_in = c.slots<int32_t>(at::kInt, cache->B, stride);
        float* w_out = c.slots<float>(at::kFloat, cache->B, stride);
        int32_t* t_out = c.slots<int32_t>(at::kInt, cache->B, stride);
        int32_t* left = c.list<int32_t>(at::kInt, cache->B);
        size_t ws_bytes;
        void* ws = c.workspace(ws_bytes);
        int32_t* src = c.slots<int32_t>(at::kInt, cache->B, stride);
        void* st = c.on_stream();
        D3TOM_CALL(status, d3tom_cache_evict(cache, max_len, keep, first, recent, w_in, t_in, w_out, t_out, (int)stride, left, src, ws, ws_bytes, st));
        return status;
    });
}
#undef D3TOM_CALL

#define D3TOM_METHOD(NAME) {#NAME, (PyCFunction)(void (*)(void))py_##NAME, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    D3TOM_METHOD(d3tom_importance), D3TOM_METHOD(d3tom_importance_static), D3TOM_METHOD(d3tom_select_topk), D3TOM_METHOD(d3tom_merge),
    D3TOM_METHOD(d3tom_merge_kv), D3TOM_METHOD(d3tom_merge_layer), D3TOM_METHOD(d3tom_attend), D3TOM_METHOD(d3tom_attend_weighted),
    D3TOM_METHOD(d3tom_update_deciders), D3TOM_METHOD(d3tom_rmsnorm), D3TOM_METHOD(d3tom_rope), D3TOM_METHOD(d3tom_linear),
    D3TOM_METHOD(d3tom_linear_tile), D3TOM_METHOD(d3tom_rope_axes), D3TOM_METHOD(d3tom_cache_append), D3TOM_METHOD(d3tom_attend_cache),
    D3TOM_METHOD(d3tom_cache_evict), {nullptr, nullptr, 0, nullptr}};
#undef D3TOM_METHOD
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
