// The call from Python into the C ABI: one CPython function that turns its arguments into machine words and calls an entry
// point.  A pruning step on one image takes 9 us from Python and has 27 arguments; marshalled by ctypes they alone took 10 us
// of host time per call, so that the caller, not the GPU, set the pace.
//
//   bind(name, address) -> handle     of the entry point `name`, which the loaded library has at `address`
//   call(handle, scale, *args) -> int
//     args      the entry point's arguments in order, without its float argument if it has one, which is `scale`
//               None -> null / 0, int -> itself, bytes -> pointer to its data (parameter structs), CUDA tensor -> data pointer
//   cache_write(stream, device, K, V, cache, new_len, cache_len, seq_len, vis_start, vis_len, keep_idx, n_keep) -> int
//   cache_read(stream, device, cache, cache_len, K_out, V_out, row_begin) -> int
//   cache_attention(stream, device, q, cache, cache_len, out, workspace, scale, causal, lse) -> int
//   rotary_axes(stream, device, q, k, position, inv_freq, axis, q_out, k_out, token, seq_len, inverse) -> int
//   window_attention(stream, device, q, K, V, cache_len, out, workspace, scale, window, n_sink, query_len, lse) -> int
//   tree_attention(stream, device, q, K, V, cache_len, tree, out, workspace, scale, query_len, lse) -> int
//     check types, shapes and devices of their tensors (ValueError), take sizes and strides from them, and call the entry point of
//     that name.  (The same checks written in Python took 8 us of a decoding step's call, its kernel 5.)
// Every entry point is called through its own type (taken from the header), each word converted to the parameter's type, so
// nothing depends on a calling convention.  The interpreter lock is released during the call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>
#include <initializer_list>
#include <stdexcept>
#include <string>
#include <type_traits>
#include <utility>

#include "vitcop.h"

namespace {

constexpr int kMaxArgs = 36;

template <typename T>
T from_word(int64_t word, float scale) {
    if constexpr (std::is_floating_point_v<T>) return static_cast<T>(scale);
    else if constexpr (std::is_pointer_v<T>) return reinterpret_cast<T>(static_cast<uintptr_t>(word));
    else return static_cast<T>(word);
}

// How many of the first n parameters are integers or pointers: the word that parameter n takes.
template <typename... A>
constexpr int words_before(size_t n) {
    constexpr bool is_float[] = {std::is_floating_point_v<A>...};
    int w = 0;
    for (size_t i = 0; i < n; ++i) w += is_float[i] ? 0 : 1;
    return w;
}

template <typename... A, size_t... I>
int invoke(int (*f)(A...), const int64_t* words, float scale, std::index_sequence<I...>) {
    return f(from_word<A>(words[words_before<A...>(I) < kMaxArgs ? words_before<A...>(I) : 0], scale)...);
}

template <typename F>
struct Signature;
template <typename... A>
struct Signature<int(A...)> {
    static constexpr int kWords = words_before<A...>(sizeof...(A));
    static_assert(kWords <= kMaxArgs, "arguments of an entry point");
    static int call(uintptr_t address, const int64_t* words, float scale) {
        return invoke(reinterpret_cast<int (*)(A...)>(address), words, scale, std::index_sequence_for<A...>{});
    }
};

struct Entry {
    const char* name;
    int words;
    int (*call)(uintptr_t, const int64_t*, float);
    uintptr_t address;
};
#define ENTRY(name) {#name, Signature<decltype(name)>::kWords, Signature<decltype(name)>::call, 0}
Entry entries[] = {
    ENTRY(vitcop_knorm_score), ENTRY(vitcop_select), ENTRY(vitcop_compact_kv), ENTRY(vitcop_prune_step),
    ENTRY(vitcop_prune_step_static), ENTRY(vitcop_collaborative_step), ENTRY(vitcop_merge_clusters),
    ENTRY(vitcop_cls_saliency), ENTRY(vitcop_kproj_knorm), ENTRY(vitcop_redundancy_filter), ENTRY(vitcop_similarity_rows),
    ENTRY(vitcop_cache_write), ENTRY(vitcop_cache_read), ENTRY(vitcop_cache_attention), ENTRY(vitcop_rotary_axes),
    ENTRY(vitcop_window_attention), ENTRY(vitcop_tree_attention)};
constexpr int kEntries = sizeof(entries) / sizeof(entries[0]);

bool to_word(PyObject* o, int64_t& v) {
    if (o == Py_None) {
        v = 0;
        return true;
    }
    if (PyLong_Check(o)) {
        v = PyLong_AsLongLong(o);
        return !(v == -1 && PyErr_Occurred());
    }
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda()) {
            PyErr_SetString(PyExc_ValueError, "expected a CUDA tensor");
            return false;
        }
        if (!t.is_contiguous()) {
            PyErr_SetString(PyExc_ValueError, "expected a contiguous tensor");
            return false;
        }
        v = static_cast<int64_t>(reinterpret_cast<uintptr_t>(t.data_ptr()));
        return true;
    }
    if (PyBytes_Check(o)) {
        v = static_cast<int64_t>(reinterpret_cast<uintptr_t>(PyBytes_AS_STRING(o)));
        return true;
    }
    PyErr_Format(PyExc_TypeError, "expected a tensor, an int, bytes or None, got %.100s", Py_TYPE(o)->tp_name);
    return false;
}

PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    const char* const name = n == 2 ? PyUnicode_AsUTF8(args[0]) : nullptr;
    if (!name) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "bind(name, address)");
        return nullptr;
    }
    const unsigned long long address = PyLong_AsUnsignedLongLong(args[1]);
    if (PyErr_Occurred()) return nullptr;
    for (int e = 0; e < kEntries; ++e) {
        if (std::strcmp(entries[e].name, name) == 0) {
            entries[e].address = static_cast<uintptr_t>(address);
            return PyLong_FromLong(e);
        }
    }
    PyErr_Format(PyExc_KeyError, "no such entry point: %.100s", name);
    return nullptr;
}

PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n < 2 || n - 2 > kMaxArgs) {
        PyErr_SetString(PyExc_TypeError, "call(handle, scale, *args): wrong number of arguments");
        return nullptr;
    }
    const long handle = PyLong_AsLong(args[0]);
    if (PyErr_Occurred()) return nullptr;
    if (handle < 0 || handle >= kEntries || entries[handle].address == 0) {
        PyErr_SetString(PyExc_ValueError, "call: not a handle of bind");
        return nullptr;
    }
    const Entry& e = entries[handle];
    const double scale = PyFloat_AsDouble(args[1]);
    if (PyErr_Occurred()) return nullptr;
    int64_t a[kMaxArgs] = {};
    for (Py_ssize_t i = 2; i < n; ++i) {
        bool ok;
        try {
            ok = to_word(args[i], a[i - 2]);
        } catch (const std::exception& ex) {
            PyErr_SetString(PyExc_RuntimeError, ex.what());
            ok = false;
        }
        if (!ok) return nullptr;
    }
    if (n - 2 != e.words) {
        PyErr_Format(PyExc_TypeError, "%s takes %d arguments, got %zd", e.name, e.words, n - 2);
        return nullptr;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = e.call(e.address, a, static_cast<float>(scale));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// ---- the calls of the cache in 4 bits, of rotary positions and of the attention over bf16 rows
struct Refused : std::invalid_argument {
    using std::invalid_argument::invalid_argument;
};
[[noreturn]] void refuse(const char* what, const char* why) { throw Refused(std::string(what) + ": " + why); }

const at::Tensor* tensor_or_none(PyObject* o, const char* what) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse(what, "expected a tensor");
    return &THPVariable_Unpack(o);
}
void on_device(const at::Tensor& t, const char* what, int64_t device) {
    if (!t.is_cuda() || t.get_device() != device) refuse(what, "expected a tensor on the current CUDA device");
}
// Data of an optional dense tensor of this type and shape (-1: any extent); null for None.
template <typename T>
T* dense(PyObject* o, const char* what, int64_t device, at::ScalarType type, std::initializer_list<int64_t> shape) {
    const at::Tensor* const t = tensor_or_none(o, what);
    if (!t) return nullptr;
    on_device(*t, what, device);
    bool fits = t->scalar_type() == type && t->dim() == (int64_t)shape.size() && t->is_contiguous();
    int64_t i = 0;
    for (const int64_t n : shape) {
        if (fits && n >= 0 && t->size(i) != n) fits = false;
        ++i;
    }
    if (!fits) refuse(what, "expected another type or shape, or a contiguous tensor");
    return static_cast<T*>(t->data_ptr());
}
// bf16 rows [B, H, N, d], elements of a row side by side; a dimension of extent 1 has no stride.
struct Rows {
    void* data = nullptr;
    int64_t stride[3] = {0, 0, 0};
};
Rows rows_of(const at::Tensor* t, const char* what, int64_t device, int64_t B, int64_t H, int64_t N, int64_t d) {
    Rows r;
    if (!t) return r;
    on_device(*t, what, device);
    if (t->scalar_type() != at::kBFloat16 || t->dim() != 4 || t->size(0) != B || t->size(1) != H || t->size(2) != N || t->size(3) != d ||
        (t->numel() > 0 && t->stride(3) != 1))
        refuse(what, "expected bf16 [B, H, N, d] that fits the other tensors, elements of a row side by side");
    r.data = t->data_ptr();
    if (t->numel() > 0)
        for (int i = 0; i < 3; ++i) r.stride[i] = t->size(i) > 1 ? t->stride(i) : 0;
    return r;
}
struct Cache {
    void* data;
    int64_t B, H, Ncap, d;
};
Cache cache_of(PyObject* o, int64_t device) {
    const at::Tensor* const t = tensor_or_none(o, "cache");
    if (!t) refuse("cache", "expected a tensor");
    on_device(*t, "cache", device);
    if (t->scalar_type() != at::kByte || t->dim() != 4 || !t->is_contiguous() || t->size(3) % 40)
        refuse("cache", "expected contiguous uint8 [B, H, Ncap / 32, 40 d]");
    return {t->data_ptr(), t->size(0), t->size(1), t->size(2) * 32, t->size(3) / 40};
}
int64_t integer(PyObject* o, const char* what) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(what, "expected an int");
    }
    return v;
}
int int32_of(int64_t v, const char* what) {
    if (v < INT32_MIN || v > INT32_MAX) refuse(what, "beyond 32 bits");
    return (int)v;
}
// An int for all samples, or int32 [B].
struct PerSample {
    const int32_t* each = nullptr;
    int all = 0;
};
PerSample per_sample(PyObject* o, const char* what, int64_t device, int64_t B) {
    PerSample p;
    if (THPVariable_Check(o)) p.each = dense<int32_t>(o, what, device, at::kInt, {B});
    else p.all = int32_of(integer(o, what), what);
    return p;
}

double number(PyObject* o, const char* what) {
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        refuse(what, "expected a number");
    }
    return v;
}
bool truth(PyObject* o, const char* what) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) {
        PyErr_Clear();
        refuse(what, "expected a truth value");
    }
    return v != 0;
}

int entry(const char* name) {
    for (int e = 0; e < kEntries; ++e)
        if (std::strcmp(entries[e].name, name) == 0) return e;
    return -1;
}
template <typename F>
F* bound(int e) {
    if (entries[e].address == 0) throw std::runtime_error(std::string(entries[e].name) + " is not bound");
    return reinterpret_cast<F*>(entries[e].address);
}

// Runs `body` (which returns a status) with C++ exceptions turned into Python's.
template <typename Body>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, const char* name, Body body) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", name, want, n);
        return nullptr;
    }
    try {
        return PyLong_FromLong(body());
    } catch (const Refused& ex) {
        PyErr_SetString(PyExc_ValueError, ex.what());
    } catch (const std::exception& ex) {
        PyErr_SetString(PyExc_RuntimeError, ex.what());
    }
    return nullptr;
}
template <typename F, typename... A>
int unlocked(F* f, A... args) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(args...);
    Py_END_ALLOW_THREADS
    return rc;
}

PyObject* cache_write(PyObject*, PyObject* const* args, Py_ssize_t n) {
    static const int e = entry("vitcop_cache_write");
    return guarded(n, 12, "cache_write", [&]() -> int {
        void* const stream = reinterpret_cast<void*>(static_cast<uintptr_t>(integer(args[0], "stream")));
        const int64_t dev = integer(args[1], "device");
        const Cache c = cache_of(args[4], dev);
        const at::Tensor *const K = tensor_or_none(args[2], "K"), *const V = tensor_or_none(args[3], "V"), *const any = K ? K : V;
        if (!any || any->dim() != 4) refuse("K, V", "expected bf16 [B, H, N, d]");
        const int64_t N = any->size(2);
        const Rows k = rows_of(K, "K", dev, c.B, c.H, N, c.d), v = rows_of(V, "V", dev, c.B, c.H, N, c.d);
        int32_t* const new_len = dense<int32_t>(args[5], "new_len", dev, at::kInt, {c.B});
        const int32_t* const cache_len = dense<int32_t>(args[6], "cache_len", dev, at::kInt, {c.B});
        const int32_t* const seq_len = dense<int32_t>(args[7], "seq_len", dev, at::kInt, {c.B});
        const PerSample vis = per_sample(args[9], "vis_len", dev, c.B);
        const int32_t* const keep = dense<int32_t>(args[10], "keep_idx", dev, at::kInt, {c.B, -1});
        const int64_t keep_stride = keep ? THPVariable_Unpack(args[10]).size(1) : 0;
        const int32_t* const n_keep = dense<int32_t>(args[11], "n_keep", dev, at::kInt, {c.B});
        return unlocked(bound<decltype(vitcop_cache_write)>(e), (const void*)k.data, (const void*)v.data, int32_of(c.B, "B"), int32_of(c.H, "H"),
                        int32_of(N, "N"), int32_of(c.d, "d"), k.stride[0], k.stride[1], k.stride[2], v.stride[0], v.stride[1], v.stride[2],
                        seq_len, int32_of(integer(args[8], "vis_start"), "vis_start"), vis.each, vis.all, keep, int32_of(keep_stride, "keep_idx"),
                        n_keep, cache_len, c.data, int32_of(c.Ncap, "Ncap"), new_len, stream);
    });
}

PyObject* cache_read(PyObject*, PyObject* const* args, Py_ssize_t n) {
    static const int e = entry("vitcop_cache_read");
    return guarded(n, 7, "cache_read", [&]() -> int {
        void* const stream = reinterpret_cast<void*>(static_cast<uintptr_t>(integer(args[0], "stream")));
        const int64_t dev = integer(args[1], "device");
        const Cache c = cache_of(args[2], dev);
        const int32_t* const cache_len = dense<int32_t>(args[3], "cache_len", dev, at::kInt, {c.B});
        const at::Tensor *const K = tensor_or_none(args[4], "K_out"), *const V = tensor_or_none(args[5], "V_out"), *const any = K ? K : V;
        if (!any || any->dim() != 4) refuse("K_out, V_out", "expected bf16 [B, H, N_out, d]");
        const int64_t N = any->size(2);
        void* const k = dense<void>(args[4], "K_out", dev, at::kBFloat16, {c.B, c.H, N, c.d});
        void* const v = dense<void>(args[5], "V_out", dev, at::kBFloat16, {c.B, c.H, N, c.d});
        const PerSample begin = per_sample(args[6], "row_begin", dev, c.B);
        return unlocked(bound<decltype(vitcop_cache_read)>(e), (const void*)c.data, int32_of(c.B, "B"), int32_of(c.H, "H"), int32_of(c.Ncap, "Ncap"),
                        int32_of(c.d, "d"), cache_len, begin.each, begin.all, k, v, int32_of(N, "N_out"), stream);
    });
}

PyObject* cache_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
    static const int e = entry("vitcop_cache_attention");
    return guarded(n, 10, "cache_attention", [&]() -> int {
        void* const stream = reinterpret_cast<void*>(static_cast<uintptr_t>(integer(args[0], "stream")));
        const int64_t dev = integer(args[1], "device");
        const at::Tensor *const q = tensor_or_none(args[2], "q"), *const out = tensor_or_none(args[5], "out");
        const Cache c = cache_of(args[3], dev);
        if (!q || q->dim() != 4) refuse("q", "expected bf16 [B, Hq, Tq, d]");
        if (!out) refuse("out", "expected a tensor");
        const int64_t Hq = q->size(1), Tq = q->size(2);
        const Rows qr = rows_of(q, "q", dev, c.B, Hq, Tq, c.d), o = rows_of(out, "out", dev, c.B, Hq, Tq, c.d);
        const int32_t* const cache_len = dense<int32_t>(args[4], "cache_len", dev, at::kInt, {c.B});
        void* const workspace = dense<void>(args[6], "workspace", dev, at::kByte, {-1});
        const size_t bytes = workspace ? (size_t)THPVariable_Unpack(args[6]).numel() : 0;
        const double scale = number(args[7], "scale");
        const int causal = truth(args[8], "causal");
        float* const lse = dense<float>(args[9], "lse", dev, at::kFloat, {c.B, Hq, Tq});
        return unlocked(bound<decltype(vitcop_cache_attention)>(e), (const void*)qr.data, (const void*)c.data, int32_of(c.B, "B"), int32_of(Hq, "Hq"),
                        int32_of(c.H, "H"), int32_of(Tq, "Tq"), int32_of(c.d, "d"), int32_of(c.Ncap, "Ncap"), qr.stride[0], qr.stride[1],
                        qr.stride[2], cache_len, static_cast<float>(scale), causal, o.data, o.stride[0], o.stride[1],
                        o.stride[2], lse, workspace, bytes, stream);
    });
}

PyObject* rotary_axes(PyObject*, PyObject* const* args, Py_ssize_t n) {
    static const int e = entry("vitcop_rotary_axes");
    return guarded(n, 12, "rotary_axes", [&]() -> int {
        void* const stream = reinterpret_cast<void*>(static_cast<uintptr_t>(integer(args[0], "stream")));
        const int64_t dev = integer(args[1], "device");
        const at::Tensor *const q = tensor_or_none(args[2], "q"), *const k = tensor_or_none(args[3], "k"), *const any = q ? q : k;
        if (!any || any->dim() != 4 || (q && q->dim() != 4) || (k && k->dim() != 4)) refuse("q, k", "expected bf16 [B, H, N, d]");
        const int64_t B = any->size(0), N = any->size(2), d = any->size(3), Hq = q ? q->size(1) : 0, Hk = k ? k->size(1) : 0;
        const Rows qr = rows_of(q, "q", dev, B, Hq, N, d), kr = rows_of(k, "k", dev, B, Hk, N, d);
        const Rows qo = rows_of(tensor_or_none(args[7], "q_out"), "q_out", dev, B, Hq, N, d), ko = rows_of(tensor_or_none(args[8], "k_out"), "k_out", dev, B, Hk, N, d);
        const int32_t* const position = dense<int32_t>(args[4], "position", dev, at::kInt, {-1, B, -1});
        if (!position && args[4] == Py_None) refuse("position", "expected a tensor");
        const at::Tensor& p = THPVariable_Unpack(args[4]);
        const double* const inv_freq = dense<double>(args[5], "inv_freq", dev, at::kDouble, {-1});
        if (args[5] == Py_None) refuse("inv_freq", "expected a tensor");
        const int64_t F = THPVariable_Unpack(args[5]).size(0);
        const int32_t* const axis = dense<int32_t>(args[6], "axis", dev, at::kInt, {F});
        const int32_t* const token = dense<int32_t>(args[9], "token", dev, at::kInt, {B, N});
        const int32_t* const seq_len = dense<int32_t>(args[10], "seq_len", dev, at::kInt, {B});
        return unlocked(bound<decltype(vitcop_rotary_axes)>(e), (const void*)qr.data, (const void*)kr.data, int32_of(B, "B"), int32_of(Hq, "Hq"), int32_of(Hk, "Hk"),
                        int32_of(N, "N"), int32_of(d, "d"), qr.stride[0], qr.stride[1], qr.stride[2], kr.stride[0], kr.stride[1], kr.stride[2], position,
                        int32_of(p.size(0), "position"), int32_of(p.size(2), "position"), token, seq_len, inv_freq, axis, int32_of(F, "inv_freq"),
                        (int)truth(args[11], "inverse"), qo.data, qo.stride[0], qo.stride[1], qo.stride[2], ko.data, ko.stride[0], ko.stride[1], ko.stride[2], stream);
    });
}

// Tensors of the attention over bf16 rows, args from q on; the rest of the arguments is the callers'.
struct Attention {
    int64_t B, Hq, H, Tq, d, N;
    Rows q, K, V, out;
    const int32_t *cache_len, *query_len;
    void* workspace;
    size_t bytes;
    float* lse;
};
Attention attention_of(int64_t dev, PyObject* q_, PyObject* K_, PyObject* V_, PyObject* len, PyObject* out_, PyObject* workspace, PyObject* query_len, PyObject* lse) {
    const at::Tensor *const q = tensor_or_none(q_, "q"), *const K = tensor_or_none(K_, "K"), *const V = tensor_or_none(V_, "V"), *const out = tensor_or_none(out_, "out");
    if (!q || q->dim() != 4) refuse("q", "expected bf16 [B, Hq, Tq, d]");
    if (!K || K->dim() != 4 || !V) refuse("K, V", "expected bf16 [B, H, N, d]");
    if (!out) refuse("out", "expected a tensor");
    Attention a;
    a.B = q->size(0);
    a.Hq = q->size(1);
    a.Tq = q->size(2);
    a.d = q->size(3);
    a.H = K->size(1);
    a.N = K->size(2);
    a.q = rows_of(q, "q", dev, a.B, a.Hq, a.Tq, a.d);
    a.K = rows_of(K, "K", dev, a.B, a.H, a.N, a.d);
    a.V = rows_of(V, "V", dev, a.B, a.H, a.N, a.d);
    a.out = rows_of(out, "out", dev, a.B, a.Hq, a.Tq, a.d);
    a.cache_len = dense<int32_t>(len, "cache_len", dev, at::kInt, {a.B});
    a.query_len = dense<int32_t>(query_len, "query_len", dev, at::kInt, {a.B});
    a.workspace = dense<void>(workspace, "workspace", dev, at::kByte, {-1});
    a.bytes = a.workspace ? (size_t)THPVariable_Unpack(workspace).numel() : 0;
    a.lse = dense<float>(lse, "lse", dev, at::kFloat, {a.B, a.Hq, a.Tq});
    return a;
}

PyObject* window_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
    static const int e = entry("vitcop_window_attention");
    return guarded(n, 13, "window_attention", [&]() -> int {
        void* const stream = reinterpret_cast<void*>(static_cast<uintptr_t>(integer(args[0], "stream")));
        const Attention a = attention_of(integer(args[1], "device"), args[2], args[3], args[4], args[5], args[6], args[7], args[11], args[12]);
        const float scale = static_cast<float>(number(args[8], "scale"));
        const int window = int32_of(integer(args[9], "window"), "window"), n_sink = int32_of(integer(args[10], "n_sink"), "n_sink");
        return unlocked(bound<decltype(vitcop_window_attention)>(e), (const void*)a.q.data, (const void*)a.K.data, (const void*)a.V.data, int32_of(a.B, "B"),
                        int32_of(a.Hq, "Hq"), int32_of(a.H, "H"), int32_of(a.Tq, "Tq"), int32_of(a.d, "d"), int32_of(a.N, "N"), a.q.stride[0], a.q.stride[1],
                        a.q.stride[2], a.K.stride[0], a.K.stride[1], a.K.stride[2], a.V.stride[0], a.V.stride[1], a.V.stride[2], a.cache_len, a.query_len, window,
                        n_sink, scale, a.out.data, a.out.stride[0], a.out.stride[1], a.out.stride[2], a.lse, a.workspace, a.bytes, stream);
    });
}

PyObject* tree_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
    static const int e = entry("vitcop_tree_attention");
    return guarded(n, 12, "tree_attention", [&]() -> int {
        void* const stream = reinterpret_cast<void*>(static_cast<uintptr_t>(integer(args[0], "stream")));
        const int64_t dev = integer(args[1], "device");
        const Attention a = attention_of(dev, args[2], args[3], args[4], args[5], args[7], args[8], args[10], args[11]);
        const int64_t* const tree = dense<int64_t>(args[6], "tree", dev, at::kLong, {a.B, a.Tq});
        const float scale = static_cast<float>(number(args[9], "scale"));
        return unlocked(bound<decltype(vitcop_tree_attention)>(e), (const void*)a.q.data, (const void*)a.K.data, (const void*)a.V.data, int32_of(a.B, "B"),
                        int32_of(a.Hq, "Hq"), int32_of(a.H, "H"), int32_of(a.Tq, "Tq"), int32_of(a.d, "d"), int32_of(a.N, "N"), a.q.stride[0], a.q.stride[1],
                        a.q.stride[2], a.K.stride[0], a.K.stride[1], a.K.stride[2], a.V.stride[0], a.V.stride[1], a.V.stride[2], a.cache_len, a.query_len, tree,
                        scale, a.out.data, a.out.stride[0], a.out.stride[1], a.out.stride[2], a.lse, a.workspace, a.bytes, stream);
    });
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind)), METH_FASTCALL, "bind(name, address) -> handle"},
    {"call", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call)), METH_FASTCALL, "call(handle, scale, *args) -> int"},
    {"cache_write", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_write)), METH_FASTCALL, "vitcop_cache_write"},
    {"cache_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_read)), METH_FASTCALL, "vitcop_cache_read"},
    {"cache_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_attention)), METH_FASTCALL, "vitcop_cache_attention"},
    {"rotary_axes", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rotary_axes)), METH_FASTCALL, "vitcop_rotary_axes"},
    {"window_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(window_attention)), METH_FASTCALL, "vitcop_window_attention"},
    {"tree_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(tree_attention)), METH_FASTCALL, "vitcop_tree_attention"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", "Calls the entry points of the C ABI.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call(void) { return PyModule_Create(&module); }
