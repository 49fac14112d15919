// Marshalling of the calls of a decode step (page plan, new tokens, append, predict, decode) for torch: checks the tensors, takes their device
// pointers and the current stream, and calls the C ABI.  Nothing is computed or kept here.
//
// Through ctypes the checks and conversions of a step's 30 arguments took 20 us of Python, more than a small step takes on
// the GPU; here they take about 2.  The entry points arrive as addresses (ctypes holds the library), so this module links
// only against torch.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <initializer_list>

#include "../../include/eta.h"

namespace {

// classes of the binding: the exception, the ctypes structures
PyObject* g_error = nullptr;
PyObject *g_desc = nullptr, *g_pages = nullptr, *g_decode_params = nullptr, *g_params = nullptr, *g_kv4 = nullptr;

bool fail(const char* name, const char* what) {
    PyErr_Format(g_error, "%s must be %s", name, what);
    return false;
}

const char* dtype_name(at::ScalarType t) {
    switch (t) {
        case at::kBFloat16: return "torch.bfloat16";
        case at::kFloat: return "torch.float32";
        case at::kInt: return "torch.int32";
        case at::kByte: return "torch.uint8";
        case at::kHalf: return "torch.float16";
        case at::kLong: return "torch.int64";
        case at::kDouble: return "torch.float64";
        default: return nullptr;
    }
}

// Device pointer of a CUDA tensor of the given type; None gives a null pointer.  With `pinned`, a page-locked host tensor
// passes too (the device can address it as it is).
bool pointer(PyObject* o, at::ScalarType type, const char* name, void** out, bool pinned = false, at::ScalarType other = at::ScalarType::Undefined) {
    *out = nullptr;
    if (o == Py_None) return true;
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a torch.Tensor or None", name);
        return false;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() && !(pinned && t.is_pinned())) return fail(name, "a CUDA tensor (no CPU path exists)");
    const at::ScalarType s = t.scalar_type();
    if (s != type && (other == at::ScalarType::Undefined || s != other)) {
        const char* got = dtype_name(s);
        if (other != at::ScalarType::Undefined)
            PyErr_Format(g_error, "%s must be float16 (compact records) or uint8 (packed records), got %s", name, got ? got : "another type");
        else
            PyErr_Format(g_error, "%s must be %s, got %s", name, dtype_name(type), got ? got : "another type");
        return false;
    }
    *out = t.data_ptr();
    return true;
}
bool musig_pointer(PyObject* o, void** out) { return pointer(o, at::kHalf, "musig", out, false, at::kByte); }

// The bytes of a ctypes structure of the binding's class `cls`
template <typename T>
struct Struct {
    Py_buffer view = {};
    bool held = false;
    const T* get(PyObject* o, PyObject* cls) {
        const int is = PyObject_IsInstance(o, cls);
        if (is <= 0) {
            if (is == 0) PyErr_Format(PyExc_TypeError, "%R expected, got %s", cls, Py_TYPE(o)->tp_name);
            return nullptr;
        }
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) return nullptr;
        held = true;
        if ((size_t)view.len != sizeof(T)) {
            PyErr_SetString(PyExc_TypeError, "a structure of the wrong size");
            return nullptr;
        }
        return static_cast<const T*>(view.buf);
    }
    ~Struct() { if (held) PyBuffer_Release(&view); }
};

bool number(PyObject* o, const char* name, double* out) {
    PyObject* v = PyObject_GetAttrString(o, name);
    if (!v) return false;
    *out = PyFloat_AsDouble(v);
    Py_DECREF(v);
    return !(*out == -1.0 && PyErr_Occurred());
}
// what a ctypes integer field makes of a value: any integer (or what has __index__), modulo 2^32; floats are refused
bool integer(PyObject* o, const char* name, uint32_t* out) {
    PyObject* v = PyObject_GetAttrString(o, name);
    if (!v) return false;
    *out = (uint32_t)PyLong_AsUnsignedLongMask(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}
// A DecodeParams is read field by field, with the results its c() would have; anything else goes through its c().
bool params_of(PyObject* o, eta_params* p) {
    if ((PyObject*)Py_TYPE(o) != g_decode_params) {
        PyObject* c = PyObject_CallMethod(o, "c", nullptr);
        if (!c) return false;
        bool ok;
        {
            Struct<eta_params> ps;
            const eta_params* from = ps.get(c, g_params);
            ok = from != nullptr;
            if (ok) *p = *from;
        }
        Py_DECREF(c);
        return ok;
    }
    double z, a, beta, scale;
    uint32_t lwb, window;
    if (!number(o, "z", &z) || !number(o, "a", &a) || !number(o, "beta", &beta) || !number(o, "scale", &scale) ||
        !integer(o, "lwb", &lwb) || !integer(o, "rescue_window", &window) || !integer(o, "flags", &p->flags))
        return false;
    p->z = (float)z; p->a = (float)a; p->beta = (float)beta; p->scale = (float)scale;
    p->lwb = (int32_t)lwb; p->rescue_window = (int32_t)window;
    return true;
}

template <typename F>
bool entry(PyObject* o, F* out) {
    *out = reinterpret_cast<F>(PyLong_AsVoidPtr(o));
    return *out || !PyErr_Occurred();
}

bool count(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
    return false;
}

void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

#define PTR(o, type, name) pointer(o, type, #name, (void**)&name)

// (address, desc, [pages,] K, seq_lens, musig, mnorm, flags) -> return code
template <bool PAGED>
PyObject* append(PyObject*, PyObject* const* v, Py_ssize_t n) {
    using Plain = int (*)(const eta_cache_desc*, const void*, const int32_t*, void*, float*, uint32_t, void*);
    using Paged = int (*)(const eta_cache_desc*, const eta_page_table*, const void*, const int32_t*, void*, float*, uint32_t, void*);
    void* fn;
    Struct<eta_cache_desc> ds;
    Struct<eta_page_table> ps;
    void *K, *seq_lens, *musig, *mnorm;
    if (!count(n, PAGED ? 8 : 7) || !entry(v[0], &fn)) return nullptr;
    const eta_cache_desc* desc = ds.get(v[1], g_desc);
    if (!desc) return nullptr;
    const eta_page_table* pages = nullptr;
    if (PAGED && !(pages = ps.get(v[2], g_pages))) return nullptr;
    v += PAGED ? 3 : 2;
    if (!PTR(v[0], at::kBFloat16, K) || !PTR(v[1], at::kInt, seq_lens) || !musig_pointer(v[2], &musig) || !PTR(v[3], at::kFloat, mnorm))
        return nullptr;
    const uint32_t flags = (uint32_t)PyLong_AsUnsignedLongMask(v[4]);
    if (PyErr_Occurred()) return nullptr;
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    if (PAGED) rc = reinterpret_cast<Paged>(fn)(desc, pages, K, (const int32_t*)seq_lens, musig, (float*)mnorm, flags, s);
    else rc = reinterpret_cast<Plain>(fn)(desc, K, (const int32_t*)seq_lens, musig, (float*)mnorm, flags, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// (address, q, W, bias, tau) -> return code
PyObject* predict(PyObject*, PyObject* const* v, Py_ssize_t n) {
    using F = int (*)(int32_t, int32_t, int32_t, const void*, const float*, const float*, float*, void*);
    F fn;
    void *q, *W, *bias, *tau;
    if (!count(n, 5) || !entry(v[0], &fn)) return nullptr;
    if (!THPVariable_Check(v[1])) { PyErr_SetString(PyExc_TypeError, "q must be a torch.Tensor"); return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(v[1]);
    if (t.dim() != 3) { PyErr_SetString(PyExc_ValueError, "q must be [batch, n_q_heads, head_dim]"); return nullptr; }
    const int32_t b = (int32_t)t.size(0), h = (int32_t)t.size(1), d = (int32_t)t.size(2);
    if (!PTR(v[1], at::kBFloat16, q) || !PTR(v[2], at::kFloat, W) || !PTR(v[3], at::kFloat, bias) || !PTR(v[4], at::kFloat, tau))
        return nullptr;
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(b, h, d, q, (const float*)W, (const float*)bias, (float*)tau, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// (address, desc, [pages,] params, q, K, V, seq_lens, musig, mnorm, tau, head_const, out, sel_mask, stats, status
//  [, workspace]) -> return code
enum class Decode { PLAIN, PAGED, STATIC };
template <Decode KIND>
PyObject* decode(PyObject*, PyObject* const* v, Py_ssize_t n) {
    using Plain = int (*)(const eta_cache_desc*, const eta_params*, const void*, const void*, const void*, const int32_t*, const void*,
                          const float*, const float*, const float*, float*, uint8_t*, int32_t*, uint32_t*, void*, size_t, void*);
    using Paged = int (*)(const eta_cache_desc*, const eta_page_table*, const eta_params*, const void*, const void*, const void*,
                          const int32_t*, const void*, const float*, const float*, const float*, float*, uint8_t*, int32_t*,
                          uint32_t*, void*, size_t, void*);
    using Static = int (*)(const eta_cache_desc*, const eta_params*, const void*, const void*, const void*, const int32_t*, const void*,
                           const float*, const float*, const float*, float*, uint8_t*, int32_t*, uint32_t*, void*);
    constexpr bool PAGED = KIND == Decode::PAGED, WS = KIND != Decode::STATIC;
    void* fn;
    Struct<eta_cache_desc> ds;
    Struct<eta_page_table> ps;
    eta_params p;
    void *q, *K, *V, *seq_lens, *musig, *mnorm, *tau, *head_const, *out, *sel_mask, *stats, *status, *workspace = nullptr;
    if (!count(n, 15 + PAGED + WS) || !entry(v[0], &fn)) return nullptr;
    const eta_cache_desc* desc = ds.get(v[1], g_desc);
    if (!desc) return nullptr;
    const eta_page_table* pages = nullptr;
    if (PAGED && !(pages = ps.get(v[2], g_pages))) return nullptr;
    v += PAGED ? 3 : 2;
    if (!params_of(v[0], &p)) return nullptr;
    if (!PTR(v[1], at::kBFloat16, q) || !PTR(v[2], at::kBFloat16, K) || !PTR(v[3], at::kBFloat16, V) || !PTR(v[4], at::kInt, seq_lens) ||
        !musig_pointer(v[5], &musig) || !PTR(v[6], at::kFloat, mnorm) || !PTR(v[7], at::kFloat, tau) ||
        !PTR(v[8], at::kFloat, head_const) || !pointer(v[9], at::kFloat, "out", &out, true) || !PTR(v[10], at::kByte, sel_mask) ||
        !PTR(v[11], at::kInt, stats) || !PTR(v[12], at::kInt, status) || (WS && !PTR(v[13], at::kByte, workspace)))
        return nullptr;
    const size_t bytes = workspace ? (size_t)THPVariable_Unpack(v[13]).numel() : 0;
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    if (KIND == Decode::PAGED)
        rc = reinterpret_cast<Paged>(fn)(desc, pages, &p, q, K, V, (const int32_t*)seq_lens, musig, (const float*)mnorm, (const float*)tau,
                                         (const float*)head_const, (float*)out, (uint8_t*)sel_mask, (int32_t*)stats,
                                         (uint32_t*)status, workspace, bytes, s);
    else if (KIND == Decode::PLAIN)
        rc = reinterpret_cast<Plain>(fn)(desc, &p, q, K, V, (const int32_t*)seq_lens, musig, (const float*)mnorm, (const float*)tau,
                                         (const float*)head_const, (float*)out, (uint8_t*)sel_mask, (int32_t*)stats,
                                         (uint32_t*)status, workspace, bytes, s);
    else
        rc = reinterpret_cast<Static>(fn)(desc, &p, q, K, V, (const int32_t*)seq_lens, musig, (const float*)mnorm, (const float*)tau,
                                          (const float*)head_const, (float*)out, (uint8_t*)sel_mask, (int32_t*)stats,
                                          (uint32_t*)status, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// A contiguous CUDA tensor of the given type on the current device, of n elements (n < 0: any number); None where `optional`.
bool vector(PyObject* o, at::ScalarType type, const char* name, int64_t n, void** out, bool optional = false) {
    if (o == Py_None && !optional) return fail(name, "a tensor, not None");
    if (!pointer(o, type, name, out)) return false;
    if (o == Py_None) return true;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.device().index() != c10::cuda::current_device()) return fail(name, "on the current CUDA device");
    if (!t.is_contiguous()) return fail(name, "contiguous");
    if (n >= 0 && t.numel() != n) {
        PyErr_Format(g_error, "%s must have %lld elements, got %lld", name, (long long)n, (long long)t.numel());
        return false;
    }
    return true;
}
#define VEC(o, type, name, n) vector(o, type, #name, n, (void**)&name)
#define OPT(o, type, name, n) vector(o, type, #name, n, (void**)&name, true)

bool int32_of(PyObject* o, int32_t* out) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) return false;
    if (v < INT32_MIN || v > INT32_MAX) {
        PyErr_SetString(PyExc_OverflowError, "an argument does not fit 32 bits");
        return false;
    }
    *out = (int32_t)v;
    return true;
}

// (address, block_size, t_cap, new_lens, release, seq_lens, seq_lens_out, block_table, free_pages, n_free, n_free_out, slot_map,
//  positions, row_start, granted, status) -> return code
PyObject* plan(PyObject*, PyObject* const* v, Py_ssize_t n) {
    using F = int (*)(int32_t, int32_t, int32_t, const int32_t*, const int32_t*, const int32_t*, int32_t*, int32_t*, int32_t, int32_t*,
                      const int32_t*, int32_t*, int32_t, int32_t, int64_t*, int32_t*, int32_t*, int32_t*, uint32_t*, void*);
    F fn;
    int32_t block_size, t_cap, *new_lens, *release, *seq_lens, *seq_lens_out, *block_table, *free_pages, *n_free, *n_free_out, *positions,
        *row_start, *granted;
    int64_t* slot_map;
    uint32_t* status;
    if (!count(n, 16) || !entry(v[0], &fn) || !int32_of(v[1], &block_size) || !int32_of(v[2], &t_cap)) return nullptr;
    if (!VEC(v[3], at::kInt, new_lens, -1)) return nullptr;
    const int64_t batch = THPVariable_Unpack(v[3]).numel();
    if (!OPT(v[4], at::kInt, release, batch) || !VEC(v[5], at::kInt, seq_lens, batch) || !VEC(v[6], at::kInt, seq_lens_out, batch) ||
        !VEC(v[8], at::kInt, free_pages, -1) || !VEC(v[9], at::kInt, n_free, 1) || !VEC(v[10], at::kInt, n_free_out, 1) ||
        !OPT(v[11], at::kLong, slot_map, -1))
        return nullptr;
    const int64_t rows = v[11] == Py_None ? 0 : THPVariable_Unpack(v[11]).numel(), pages = THPVariable_Unpack(v[8]).numel();
    if (!(v[11] == Py_None ? OPT(v[12], at::kInt, positions, -1) : VEC(v[12], at::kInt, positions, rows)) ||
        !VEC(v[13], at::kInt, row_start, batch + 1) || !VEC(v[14], at::kInt, granted, batch) || !OPT(v[15], at::kInt, status, 1))
        return nullptr;
    if (!PTR(v[7], at::kInt, block_table)) return nullptr;
    if (!block_table && v[7] == Py_None) return fail("block_table", "a tensor, not None"), nullptr;
    const at::Tensor& table = THPVariable_Unpack(v[7]);
    if (table.device().index() != c10::cuda::current_device()) return fail("block_table", "on the current CUDA device"), nullptr;
    if (table.dim() != 2 || table.size(0) != batch || table.stride(1) != 1 || (batch > 1 && table.stride(0) < table.size(1)))
        return fail("block_table", "[batch, pages of a sequence] with unit stride along its second axis"), nullptr;
    // the row's stride where there is a next row, its length where not
    const int64_t stride = batch > 1 ? table.stride(0) : table.size(1);
    if (table.size(1) * (int64_t)block_size < t_cap) return fail("block_table", "wide enough for t_cap tokens"), nullptr;
    if (batch > INT32_MAX || rows > INT32_MAX || pages > INT32_MAX || stride > INT32_MAX) return fail("sizes", "below 2^31"), nullptr;
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn((int32_t)batch, block_size, t_cap, new_lens, release, seq_lens, seq_lens_out, block_table, (int32_t)stride, free_pages, n_free,
            n_free_out, (int32_t)pages, (int32_t)rows, slot_map, positions, row_start, granted, status, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// A CUDA tensor on the current device with unit stride along its last axis and the given sizes (-1: any).
bool shaped(PyObject* o, at::ScalarType type, const char* name, std::initializer_list<int64_t> sizes, void** out) {
    if (o == Py_None) return fail(name, "a tensor, not None");
    if (!pointer(o, type, name, out)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.device().index() != c10::cuda::current_device()) return fail(name, "on the current CUDA device");
    bool ok = t.dim() == (int64_t)sizes.size() && t.stride(-1) == 1;
    int64_t k = 0;
    for (int64_t n : sizes) {
        ok = ok && (n < 0 || t.size(k) == n);
        ++k;
    }
    return ok || fail(name, "of the shape that the call's descriptors say, with unit stride along its last axis");
}
// the stride of an axis, 0 where it has one element and torch may say anything
int64_t stride_of(const at::Tensor& t, int64_t axis) { return t.size(axis) > 1 ? t.stride(axis) : 0; }

// K or V as the descriptor has it: contiguous [batch, n_kv_heads, t_cap, head_dim], paged [n_pages, n_kv_heads, block_size, head_dim]
bool cache_tensor(PyObject* o, const char* name, const eta_cache_desc* d, bool paged, void** out) {
    return shaped(o, at::kBFloat16, name, {paged ? -1 : d->batch, d->n_kv_heads, paged ? d->block_size : d->t_cap, d->head_dim}, out);
}
bool same_strides(PyObject* o, const char* name, std::initializer_list<int64_t> strides) {
    const at::Tensor& t = THPVariable_Unpack(o);
    int64_t k = 0;
    for (int64_t s : strides) {
        if (t.size(k) > 1 && t.stride(k) != s) return fail(name, "the tensor that its descriptor was made for (other strides)");
        ++k;
    }
    return true;
}
// the pool of a 4-bit cache: [n_pages, n_kv_heads, bytes] (paged) or [batch, n_kv_heads, blocks, bytes]; *n_pages: 0 where not paged
bool pool_tensor(PyObject* o, const eta_cache_desc* d, const eta_kv4_desc* q4, void** out, int32_t* n_pages) {
    if (!pointer(o, at::kByte, "pool", out)) return false;
    if (o == Py_None) return fail("pool", "a tensor, not None");
    const at::Tensor& t = THPVariable_Unpack(o);
    const int64_t bytes = 2 * (int64_t)d->block_size * (d->head_dim / 2 + d->head_dim / 16);
    const bool paged = t.dim() == 3;
    *n_pages = 0;
    if (paged) {
        if (!shaped(o, at::kByte, "pool", {-1, d->n_kv_heads, bytes}, out) || !same_strides(o, "pool", {q4->stride_b, q4->stride_h})) return false;
        if (t.size(0) > INT32_MAX || t.size(0) < 1) return fail("pool", "of 1 to 2^31 - 1 pages");
        *n_pages = (int32_t)t.size(0);
        return true;
    }
    if (!shaped(o, at::kByte, "pool", {d->batch, d->n_kv_heads, -1, bytes}, out) ||
        !same_strides(o, "pool", {q4->stride_b, q4->stride_h, q4->stride_j}))
        return false;
    return t.size(2) * (int64_t)d->block_size >= d->t_cap || fail("pool", "large enough for t_cap tokens");
}

// (address, desc, kv4 or None, q, k, v, q_weight, k_weight, inv_freq, positions, slot_map, paged, q_out, K or pool, V or None, status, eps,
//  flags) -> return code
PyObject* tokens(PyObject*, PyObject* const* v, Py_ssize_t n) {
    using Plain = int (*)(const eta_cache_desc*, const eta_tokens_desc*, const void*, const void*, const void*, const float*, const float*,
                          const double*, const int32_t*, const int64_t*, int32_t, void*, void*, void*, uint32_t*, void*);
    using Kv4 = int (*)(const eta_cache_desc*, const eta_kv4_desc*, const eta_tokens_desc*, const void*, const void*, const void*, const float*,
                        const float*, const double*, const int32_t*, const int64_t*, int32_t, void*, void*, uint32_t*, void*);
    void *fn, *q, *k, *x, *q_out, *K, *V = nullptr;
    Struct<eta_cache_desc> ds;
    Struct<eta_kv4_desc> qs;
    if (!count(n, 18) || !entry(v[0], &fn)) return nullptr;
    const eta_cache_desc* desc = ds.get(v[1], g_desc);
    if (!desc) return nullptr;
    const eta_kv4_desc* q4 = nullptr;
    if (v[2] != Py_None && !(q4 = qs.get(v[2], g_kv4))) return nullptr;
    if (!THPVariable_Check(v[3])) { PyErr_SetString(PyExc_TypeError, "q must be a torch.Tensor"); return nullptr; }
    const at::ScalarType type = THPVariable_Unpack(v[3]).scalar_type();
    if (type != at::kBFloat16 && type != at::kHalf && type != at::kFloat) return fail("q", "bfloat16, float16 or float32"), nullptr;
    if (!shaped(v[3], type, "q", {-1, desc->n_q_heads, desc->head_dim}, &q)) return nullptr;
    const at::Tensor& tq = THPVariable_Unpack(v[3]);
    const int64_t rows = tq.size(0);
    if (rows > INT32_MAX) return fail("q", "of fewer than 2^31 rows"), nullptr;
    if (!shaped(v[4], type, "k", {rows, desc->n_kv_heads, desc->head_dim}, &k) || !shaped(v[5], type, "v", {rows, desc->n_kv_heads, desc->head_dim}, &x))
        return nullptr;
    const at::Tensor &tk = THPVariable_Unpack(v[4]), &tv = THPVariable_Unpack(v[5]);
    float *q_weight, *k_weight;
    double* inv_freq;
    int32_t *positions, n_pages = 0;
    int64_t* slot_map;
    uint32_t* status;
    if (!OPT(v[6], at::kFloat, q_weight, desc->head_dim) || !OPT(v[7], at::kFloat, k_weight, desc->head_dim) || !OPT(v[8], at::kDouble, inv_freq, -1) ||
        !OPT(v[9], at::kInt, positions, rows) || !VEC(v[10], at::kLong, slot_map, rows) ||
        !VEC(v[12], at::kBFloat16, q_out, rows * desc->n_q_heads * desc->head_dim) || !OPT(v[15], at::kInt, status, 1))
        return nullptr;
    if (q4) {
        if (!pool_tensor(v[13], desc, q4, &K, &n_pages)) return nullptr;
    } else {
        const int paged = PyObject_IsTrue(v[11]);
        if (paged < 0) return nullptr;
        if (!cache_tensor(v[13], "K", desc, paged != 0, &K) || !same_strides(v[13], "K", {desc->k_stride_b, desc->k_stride_h, desc->k_stride_t}) ||
            !cache_tensor(v[14], "V", desc, paged != 0, &V) || !same_strides(v[14], "V", {desc->v_stride_b, desc->v_stride_h, desc->v_stride_t}))
            return nullptr;
        if (paged) {
            const int64_t pk = THPVariable_Unpack(v[13]).size(0);
            if (pk != THPVariable_Unpack(v[14]).size(0) || pk < 1 || pk > INT32_MAX) return fail("K and V", "pools of the same number of pages"), nullptr;
            n_pages = (int32_t)pk;
        }
    }
    eta_tokens_desc t;
    t.n_rows = (int32_t)rows;
    t.type = type == at::kBFloat16 ? ETA_TYPE_BF16 : (type == at::kHalf ? ETA_TYPE_FP16 : ETA_TYPE_FP32);
    const int64_t half = v[8] == Py_None ? 0 : THPVariable_Unpack(v[8]).numel();
    if (2 * half > desc->head_dim) return fail("inv_freq", "of at most head_dim / 2 elements"), nullptr;
    t.rotary_dim = (int32_t)(2 * half);
    t.q_stride_r = stride_of(tq, 0); t.q_stride_h = stride_of(tq, 1);
    t.k_stride_r = stride_of(tk, 0); t.k_stride_h = stride_of(tk, 1);
    t.v_stride_r = stride_of(tv, 0); t.v_stride_h = stride_of(tv, 1);
    t.eps = (float)PyFloat_AsDouble(v[16]);
    t.flags = (uint32_t)PyLong_AsUnsignedLongMask(v[17]);
    if (PyErr_Occurred()) return nullptr;
    if (rows == 0) return PyLong_FromLong(ETA_OK);           // empty tensors have no address
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    if (q4)
        rc = reinterpret_cast<Kv4>(fn)(desc, q4, &t, q, k, x, q_weight, k_weight, inv_freq, positions, slot_map, n_pages, q_out, K, status, s);
    else
        rc = reinterpret_cast<Plain>(fn)(desc, &t, q, k, x, q_weight, k_weight, inv_freq, positions, slot_map, n_pages, q_out, K, V, status, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// (address, desc, kv4, pool, K, V) -> return code; K and V of any strides
PyObject* unpack(PyObject*, PyObject* const* v, Py_ssize_t n) {
    using F = int (*)(const eta_cache_desc*, const eta_kv4_desc*, const void*, int32_t, void*, void*, void*);
    F fn;
    void *pool, *K, *V;
    int32_t n_pages;
    Struct<eta_cache_desc> ds;
    Struct<eta_kv4_desc> qs;
    if (!count(n, 6) || !entry(v[0], &fn)) return nullptr;
    const eta_cache_desc* from = ds.get(v[1], g_desc);
    if (!from) return nullptr;
    const eta_kv4_desc* q4 = qs.get(v[2], g_kv4);
    if (!q4 || !pool_tensor(v[3], from, q4, &pool, &n_pages)) return nullptr;
    if (!cache_tensor(v[4], "K", from, n_pages > 0, &K) || !cache_tensor(v[5], "V", from, n_pages > 0, &V)) return nullptr;
    const at::Tensor &k = THPVariable_Unpack(v[4]), &x = THPVariable_Unpack(v[5]);
    if (n_pages && (k.size(0) != n_pages || x.size(0) != n_pages)) return fail("K and V", "of as many pages as the pool"), nullptr;
    eta_cache_desc d = *from;
    d.k_stride_b = stride_of(k, 0); d.k_stride_h = stride_of(k, 1); d.k_stride_t = k.size(2) > 1 ? k.stride(2) : d.head_dim;
    d.v_stride_b = stride_of(x, 0); d.v_stride_h = stride_of(x, 1); d.v_stride_t = x.size(2) > 1 ? x.stride(2) : d.head_dim;
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(&d, q4, pool, n_pages, K, V, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// the page table of a 4-bit cache's call, or none: what the pool says
bool pages_of(PyObject* o, Struct<eta_page_table>& ps, int32_t n_pages, const eta_page_table** out) {
    *out = nullptr;
    if (o != Py_None && !(*out = ps.get(o, g_pages))) return false;
    if ((n_pages > 0) != (*out != nullptr)) return fail("pages", n_pages ? "the page table of the paged pool" : "None: the pool is contiguous");
    return !*out || (*out)->n_pages <= n_pages || fail("pages", "of a pool with no more pages than this one");
}

// (address, desc, kv4, pages or None, pool, seq_lens, musig, mnorm, flags) -> return code; the build and the append
PyObject* index_kv4(PyObject*, PyObject* const* v, Py_ssize_t n) {
    using F = int (*)(const eta_cache_desc*, const eta_kv4_desc*, const eta_page_table*, const void*, const int32_t*, void*, float*, uint32_t,
                      void*);
    F fn;
    Struct<eta_cache_desc> ds;
    Struct<eta_kv4_desc> qs;
    Struct<eta_page_table> ps;
    void *pool, *musig;
    int32_t n_pages, *seq_lens;
    float* mnorm;
    const eta_page_table* pages;
    if (!count(n, 9) || !entry(v[0], &fn)) return nullptr;
    const eta_cache_desc* desc = ds.get(v[1], g_desc);
    if (!desc) return nullptr;
    const eta_kv4_desc* q4 = qs.get(v[2], g_kv4);
    if (!q4 || !pool_tensor(v[4], desc, q4, &pool, &n_pages) || !pages_of(v[3], ps, n_pages, &pages)) return nullptr;
    const uint32_t flags = (uint32_t)PyLong_AsUnsignedLongMask(v[8]);
    if (PyErr_Occurred()) return nullptr;
    const int64_t blocks = (int64_t)desc->batch * desc->n_kv_heads * desc->nb_cap;
    const bool packed = (flags & ETA_BUILD_PACKED_SIGMA) != 0;
    if (!VEC(v[5], at::kInt, seq_lens, desc->batch) ||
        !vector(v[6], packed ? at::kByte : at::kHalf, "musig", blocks * desc->head_dim * (packed ? 3 : 2), &musig) || !VEC(v[7], at::kFloat, mnorm, blocks))
        return nullptr;
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(desc, q4, pages, pool, seq_lens, musig, mnorm, flags, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// (address, desc, kv4, pages or None, params, q, pool, seq_lens, musig, mnorm, tau, head_const, out, sel_mask, stats, status, workspace)
// -> return code
PyObject* decode_kv4(PyObject*, PyObject* const* v, Py_ssize_t n) {
    using F = int (*)(const eta_cache_desc*, const eta_kv4_desc*, const eta_page_table*, const eta_params*, const void*, const void*,
                      const int32_t*, const void*, const float*, const float*, const float*, float*, uint8_t*, int32_t*, uint32_t*, void*, size_t,
                      void*);
    F fn;
    Struct<eta_cache_desc> ds;
    Struct<eta_kv4_desc> qs;
    Struct<eta_page_table> ps;
    eta_params p;
    void *q, *pool, *musig, *workspace, *out;
    int32_t n_pages, *seq_lens, *stats;
    float *mnorm, *tau, *head_const;
    uint8_t* sel_mask;
    uint32_t* status;
    const eta_page_table* pages;
    if (!count(n, 17) || !entry(v[0], &fn)) return nullptr;
    const eta_cache_desc* d = ds.get(v[1], g_desc);
    if (!d) return nullptr;
    const eta_kv4_desc* q4 = qs.get(v[2], g_kv4);
    if (!q4 || !params_of(v[4], &p) || !pool_tensor(v[6], d, q4, &pool, &n_pages) || !pages_of(v[3], ps, n_pages, &pages)) return nullptr;
    const int64_t rows = (int64_t)d->batch * d->n_kv_heads, heads = (int64_t)d->batch * d->n_q_heads, blocks = rows * d->nb_cap;
    const bool packed = (p.flags & ETA_FLAG_PACKED_SIGMA) != 0, index = (p.flags & ETA_FLAG_DENSE) == 0;
    if (!VEC(v[5], at::kBFloat16, q, heads * d->head_dim) || !VEC(v[7], at::kInt, seq_lens, d->batch) ||
        !vector(v[8], packed ? at::kByte : at::kHalf, "musig", blocks * d->head_dim * (packed ? 3 : 2), &musig, !index) ||
        !vector(v[9], at::kFloat, "mnorm", blocks, (void**)&mnorm, !index) || !OPT(v[10], at::kFloat, tau, heads) ||
        !OPT(v[11], at::kFloat, head_const, d->n_q_heads) || !VEC(v[13], at::kByte, sel_mask, blocks) || !OPT(v[14], at::kInt, stats, rows) ||
        !OPT(v[15], at::kInt, status, 1) || !VEC(v[16], at::kByte, workspace, -1))
        return nullptr;
    // the output may be page-locked host memory
    if (!pointer(v[12], at::kFloat, "out", &out, true)) return nullptr;
    if (v[12] == Py_None) return fail("out", "a tensor, not None"), nullptr;
    const at::Tensor& o = THPVariable_Unpack(v[12]);
    if (!o.is_contiguous() || o.numel() != heads * d->head_dim || (o.is_cuda() && o.device().index() != c10::cuda::current_device()))
        return fail("out", "contiguous [batch, n_q_heads, head_dim] on the current CUDA device or in page-locked memory"), nullptr;
    const size_t bytes = (size_t)THPVariable_Unpack(v[16]).numel();
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(d, q4, pages, &p, q, pool, seq_lens, musig, mnorm, tau, head_const, (float*)out, sel_mask, stats, status, workspace, bytes, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// the eta_params a call would get, as bytes (for the tests)
PyObject* params(PyObject*, PyObject* const* v, Py_ssize_t n) {
    eta_params p;
    if (!count(n, 1) || !params_of(v[0], &p)) return nullptr;
    return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&p), sizeof p);
}

// (EtaError, CacheDesc, PageTable, DecodeParams, Params, Kv4Desc)
PyObject* set_classes(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (!count(n, 6)) return nullptr;
    PyObject** const to[6] = {&g_error, &g_desc, &g_pages, &g_decode_params, &g_params, &g_kv4};
    for (int k = 0; k < 6; ++k) {
        Py_INCREF(v[k]);
        Py_XSETREF(*to[k], v[k]);
    }
    Py_RETURN_NONE;
}

// no C++ exception (torch reports its errors with them) crosses into the interpreter
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* v, Py_ssize_t n) {
    try {
        return F(self, v, n);
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyMethodDef methods[] = {
    {"append", (PyCFunction)(void (*)(void))guarded<append<false>>, METH_FASTCALL, nullptr},
    {"append_paged", (PyCFunction)(void (*)(void))guarded<append<true>>, METH_FASTCALL, nullptr},
    {"predict", (PyCFunction)(void (*)(void))guarded<predict>, METH_FASTCALL, nullptr},
    {"decode", (PyCFunction)(void (*)(void))guarded<decode<Decode::PLAIN>>, METH_FASTCALL, nullptr},
    {"decode_paged", (PyCFunction)(void (*)(void))guarded<decode<Decode::PAGED>>, METH_FASTCALL, nullptr},
    {"decode_static", (PyCFunction)(void (*)(void))guarded<decode<Decode::STATIC>>, METH_FASTCALL, nullptr},
    {"tokens", (PyCFunction)(void (*)(void))guarded<tokens>, METH_FASTCALL, nullptr},
    {"index_kv4", (PyCFunction)(void (*)(void))guarded<index_kv4>, METH_FASTCALL, nullptr},
    {"decode_kv4", (PyCFunction)(void (*)(void))guarded<decode_kv4>, METH_FASTCALL, nullptr},
    {"unpack", (PyCFunction)(void (*)(void))guarded<unpack>, METH_FASTCALL, nullptr},
    {"plan", (PyCFunction)(void (*)(void))guarded<plan>, METH_FASTCALL, nullptr},
    {"params", (PyCFunction)(void (*)(void))guarded<params>, METH_FASTCALL, nullptr},
    {"set_classes", (PyCFunction)(void (*)(void))set_classes, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_eta_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__eta_torch(void) { return PyModule_Create(&module); }
