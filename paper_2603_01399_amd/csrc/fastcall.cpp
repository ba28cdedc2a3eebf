// The argument marshalling of the linears, the fused linears and the paged cache in native code: what binding.py does for an ordinary call - plain CUDA tensors, of a
// linear with an output given - without its Python and ctypes steps.  Scratch that a call uses comes from torch's allocator, on the stream of the call.
//
// Every function returns the status of the C entry point it calls, or -1 for "not an ordinary call": binding.py then goes its
// own way, which raises what is to be raised.  Nothing is kept from one call for the next.
//
// What it measured, one 1024 x 1024 linear of 8 tokens through the binding, us of host time: 6.1 -> 4.0, of which the launch
// itself takes 2.9 (the kernel 3.4 on the GPU); a decoder block whose six calls are host-bound 40.9 -> 33.8.  A call with scratch and two
// launches (1024 x 8256 with a residual, 9 tokens; 7.3 in a graph): 13.0 through Python, 7.9 so.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/core/Allocator.h>
#include <c10/util/Exception.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <new>
#include <type_traits>

#include "../../include/quasar.h"
#include "unlocked.hpp"

namespace {

using quasar::call;
using quasar::status_of;

// entry points of the library that binding.py has loaded, and torch's own two functions for the current stream
decltype(&quasar_w8_linear) p_w8_linear;
decltype(&quasar_bf16_linear) p_bf16_linear;
decltype(&quasar_w8a8_linear_split) p_w8a8_linear;
decltype(&quasar_w4_linear_split) p_w4_linear;
decltype(&quasar_w4_packed_bytes) p_w4_packed_bytes;
decltype(&quasar_w8a8_workspace_bytes) p_w8a8_workspace_bytes;
decltype(&quasar_w4_workspace_bytes) p_w4_workspace_bytes;
decltype(&quasar_w8_linear_fused_split) p_w8_linear_fused;
decltype(&quasar_w8_gateup_swiglu_split) p_w8_gateup_swiglu;
decltype(&quasar_w8_fused_workspace_bytes) p_w8_fused_workspace_bytes;
decltype(&quasar_w8_gateup_workspace_bytes) p_w8_gateup_workspace_bytes;
decltype(&quasar_paged_prepare) p_paged_prepare;
decltype(&quasar_paged_attention) p_paged_attention;
decltype(&quasar_paged_attention_workspace_bytes) p_paged_attention_workspace_bytes;
decltype(&quasar_prompt_attention) p_prompt_attention;
decltype(&quasar_prompt_attention_workspace_bytes) p_prompt_attention_workspace_bytes;
decltype(&quasar_pages_reserve) p_pages_reserve;
decltype(&quasar_pages_fork) p_pages_fork;
decltype(&quasar_pages_compact) p_pages_compact;
decltype(&quasar_paged_prepare_rope) p_paged_prepare_rope;
decltype(&quasar_paged_attention_window) p_paged_attention_window;
decltype(&quasar_prompt_attention_window) p_prompt_attention_window;
decltype(&quasar_pages_trim) p_pages_trim;
decltype(&quasar_sample_tokens) p_sample_tokens;
decltype(&quasar_sample_tokens_workspace_bytes) p_sample_tokens_workspace_bytes;
decltype(&quasar_verify_tokens) p_verify_tokens;
decltype(&quasar_verify_tokens_workspace_bytes) p_verify_tokens_workspace_bytes;
PyObject *g_device, *g_stream;

struct NotOrdinary {};

// a tensor of exactly torch's class (or a parameter) on the GPU; a subclass may stand for something else
const at::Tensor &cuda_tensor(PyObject *o, at::ScalarType type) {
    if (!THPVariable_CheckExact(o)) throw NotOrdinary{};
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type) throw NotOrdinary{};
    return t;
}
const at::Tensor &any_tensor(PyObject *o) {
    if (!THPVariable_CheckExact(o)) throw NotOrdinary{};
    return THPVariable_Unpack(o);
}
int64_t integer(PyObject *o) {
    if (!PyLong_CheckExact(o)) throw NotOrdinary{};
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow) throw NotOrdinary{};
    return v;
}

struct Activations {
    const uint16_t *x;
    int64_t M, K, ldx;
    explicit Activations(PyObject *o) {
        const at::Tensor &t = cuda_tensor(o, at::kBFloat16);
        if (t.dim() != 2) throw NotOrdinary{};
        x = static_cast<const uint16_t *>(t.data_ptr());
        M = t.size(0);
        K = t.size(1);
        ldx = t.stride(0);
    }
};
struct Output {
    uint16_t *y;
    int64_t ldy;
    explicit Output(PyObject *o) {
        const at::Tensor &t = any_tensor(o);
        if (t.dim() < 1) throw NotOrdinary{};
        y = static_cast<uint16_t *>(t.data_ptr());
        ldy = t.stride(0);
    }
};
struct Workspace {
    void *p = nullptr;
    size_t bytes = 0;
    explicit Workspace(PyObject *o) {
        if (o == Py_None) return;
        const at::Tensor &t = any_tensor(o);
        p = t.data_ptr();
        bytes = t.nbytes();
    }
};

void *current_stream() {
    PyObject *dev = PyObject_CallNoArgs(g_device);
    PyObject *raw = dev ? PyObject_CallOneArg(g_stream, dev) : nullptr;
    Py_XDECREF(dev);
    if (!raw) throw NotOrdinary{};
    void *s = PyLong_AsVoidPtr(raw);
    Py_DECREF(raw);
    if (PyErr_Occurred()) throw NotOrdinary{};
    return s;
}

// A call with `need` bytes of scratch: entry(.., scratch, bytes, stream).  The scratch is given back behind the launch, for work that
// follows on the same stream.  Scratch makes a call faster and no call needs it: where memory is short it runs without.
template <typename Entry, typename... Args>
int call_with_scratch(Entry entry, size_t need, void *stream, Args... args) {
    quasar::Unlocked unlocked;
    c10::DataPtr scratch;
    if (need) {
        try {
            scratch = c10::GetAllocator(c10::DeviceType::CUDA)->allocate(need);
        } catch (const c10::OutOfMemoryError &) {
        }
    }
    return entry(args..., scratch.get(), scratch ? need : 0, stream);
}

// (x, wq_packed, scales, N, y, workspace)
PyObject *w8_linear(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return status_of(n, 6, [&] {
        const Activations x(a[0]);
        const void *w = cuda_tensor(a[1], at::kChar).data_ptr(), *sc = cuda_tensor(a[2], at::kBFloat16).data_ptr();
        const Output y(a[4]);
        const Workspace ws(a[5]);
        return call(p_w8_linear, x.x, x.M, x.K, x.ldx, static_cast<const int8_t *>(w), static_cast<const uint16_t *>(sc), integer(a[3]), y.y,
                           y.ldy, ws.p, ws.bytes, current_stream());
    });
}

// (x, w_packed, N, y, workspace)
PyObject *bf16_linear(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return status_of(n, 5, [&] {
        const Activations x(a[0]);
        const void *w = cuda_tensor(a[1], at::kBFloat16).data_ptr();
        const Output y(a[3]);
        const Workspace ws(a[4]);
        return call(p_bf16_linear, x.x, x.M, x.K, x.ldx, static_cast<const uint16_t *>(w), integer(a[2]), y.y, y.ldy, ws.p, ws.bytes,
                             current_stream());
    });
}

// (x, wq_packed, scales, N, smooth, y)
PyObject *w8a8_linear(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return status_of(n, 6, [&] {
        const Activations x(a[0]);
        const int64_t N = integer(a[3]);
        const void *w = cuda_tensor(a[1], at::kChar).data_ptr(), *sc = cuda_tensor(a[2], at::kBFloat16).data_ptr();
        const float *smooth = nullptr;
        if (a[4] != Py_None) {
            const at::Tensor &s = cuda_tensor(a[4], at::kFloat);
            if (s.numel() != x.K || !s.is_contiguous()) throw NotOrdinary{};
            smooth = static_cast<const float *>(s.data_ptr());
        }
        const Output y(a[5]);
        return call_with_scratch(p_w8a8_linear, p_w8a8_workspace_bytes(x.M, N, x.K), current_stream(), x.x, x.M, x.K, x.ldx, smooth,
                                 static_cast<const int8_t *>(w), static_cast<const uint16_t *>(sc), N, y.y, y.ldy);
    });
}

// (x, w4_packed, N, y)
PyObject *w4_linear(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return status_of(n, 4, [&] {
        const Activations x(a[0]);
        const at::Tensor &w = cuda_tensor(a[1], at::kByte);
        const int64_t N = integer(a[2]);
        if (w.numel() < (int64_t)p_w4_packed_bytes(N, x.K)) throw NotOrdinary{};
        const Output y(a[3]);
        return call_with_scratch(p_w4_linear, p_w4_workspace_bytes(x.M, N, x.K), current_stream(), x.x, x.M, x.K, x.ldx,
                                 static_cast<const void *>(w.data_ptr()), N, y.y, y.ldy);
    });
}

struct Gamma {
    const uint16_t *p = nullptr;
    Gamma(PyObject *o, int64_t K) {
        if (o == Py_None) return;
        const at::Tensor &t = cuda_tensor(o, at::kBFloat16);
        if (t.numel() != K || !t.is_contiguous()) throw NotOrdinary{};
        p = static_cast<const uint16_t *>(t.data_ptr());
    }
};
float real(PyObject *o) {
    if (!PyFloat_CheckExact(o)) throw NotOrdinary{};
    return static_cast<float>(PyFloat_AS_DOUBLE(o));
}

// (x, wq_packed, scales, N, gamma, eps, residual, y)
PyObject *w8_linear_fused(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return status_of(n, 8, [&] {
        const Activations x(a[0]);
        const void *w = cuda_tensor(a[1], at::kChar).data_ptr(), *sc = cuda_tensor(a[2], at::kBFloat16).data_ptr();
        const int64_t N = integer(a[3]);
        const Gamma gamma(a[4], x.K);
        const uint16_t *residual = nullptr;
        int64_t ldr = 0;
        if (a[6] != Py_None) {
            const at::Tensor &r = cuda_tensor(a[6], at::kBFloat16);
            if (r.dim() != 2 || r.size(0) != x.M || r.size(1) != N || r.stride(1) != 1) throw NotOrdinary{};
            residual = static_cast<const uint16_t *>(r.data_ptr());
            ldr = r.stride(0);
        }
        const float eps = real(a[5]);
        const Output y(a[7]);
        return call_with_scratch(p_w8_linear_fused, p_w8_fused_workspace_bytes(x.M, N, x.K, gamma.p != nullptr, residual != nullptr),
                                 current_stream(), x.x, x.M, x.K, x.ldx, gamma.p, eps, static_cast<const int8_t *>(w),
                                 static_cast<const uint16_t *>(sc), N, residual, ldr, y.y, y.ldy);
    });
}

// (x, wq_packed, scales, I, gamma, eps, y)
PyObject *w8_gateup_swiglu(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return status_of(n, 7, [&] {
        const Activations x(a[0]);
        const void *w = cuda_tensor(a[1], at::kChar).data_ptr(), *sc = cuda_tensor(a[2], at::kBFloat16).data_ptr();
        const int64_t I = integer(a[3]);
        const Gamma gamma(a[4], x.K);
        const float eps = real(a[5]);
        const Output y(a[6]);
        return call_with_scratch(p_w8_gateup_swiglu, p_w8_gateup_workspace_bytes(x.M, I, x.K, gamma.p != nullptr), current_stream(),
                                 x.x, x.M, x.K, x.ldx, gamma.p, eps, static_cast<const int8_t *>(w), static_cast<const uint16_t *>(sc), I,
                                 y.y, y.ldy);
    });
}

// ---- the paged cache: calls on a handle, which answer with the tensor that they return in Python, else with the status or -1

// One of a cache's buffers, held, and where it lay when the cache was made: `tensor.data = ...` or a resize gives the same tensor other memory.
struct Buffer {
    at::Tensor t;
    void *at = nullptr;
    size_t bytes = 0;
    explicit Buffer(PyObject *o) {
        if (o == Py_None) return;
        if (!THPVariable_Check(o)) throw NotOrdinary{};
        t = THPVariable_Unpack(o);
        at = t.data_ptr();
        bytes = t.nbytes();
    }
    bool as_made() const { return !t.defined() || (t.is_contiguous() && t.nbytes() == bytes && t.data_ptr() == at); }
};
// What PagedKvCache is made of.
struct PagedCache {
    long long n_layers, n_kv_heads, n_pages, page_len, max_seqs, max_pages, code, layer_bytes, workspace_bytes;
    Buffer pool, books, refs, lengths, table, k_scale, v_scale;
    int device;
    bool as_made() const {
        for (const Buffer *b : {&pool, &books, &refs, &lengths, &table, &k_scale, &v_scale})
            if (!b->as_made()) return false;
        return true;
    }
};
constexpr const char *kCacheName = "quasar.PagedCache";

// (the sizes in order; pool, books, refs, lengths, table, k_scale or None, v_scale or None)
PyObject *paged_cache(PyObject *, PyObject *args) {
    long long n[9];
    PyObject *b[7];
    if (!PyArg_ParseTuple(args, "LLLLLLLLLOOOOOOO", &n[0], &n[1], &n[2], &n[3], &n[4], &n[5], &n[6], &n[7], &n[8], &b[0], &b[1], &b[2], &b[3], &b[4], &b[5], &b[6]))
        return nullptr;
    PagedCache *held = nullptr;
    try {
        const Buffer pool(b[0]);
        const int device = pool.t.defined() ? pool.t.device().index() : -1;
        held = new (std::nothrow) PagedCache{n[0], n[1], n[2], n[3], n[4], n[5], n[6], n[7], n[8], pool, Buffer(b[1]), Buffer(b[2]), Buffer(b[3]), Buffer(b[4]),
                                             Buffer(b[5]), Buffer(b[6]), device};
    } catch (...) {
        PyErr_SetString(PyExc_TypeError, "a cache's buffers are tensors");
        return nullptr;
    }
    if (!held) return PyErr_NoMemory();
    PyObject *o = PyCapsule_New(held, kCacheName, [](PyObject *o) { delete static_cast<PagedCache *>(PyCapsule_GetPointer(o, kCacheName)); });
    if (!o) delete held;
    return o;
}
// (handle) -> whether the cache's buffers lie where they lay when it was made
PyObject *paged_cache_as_made(PyObject *, PyObject *o) {
    const auto *c = static_cast<const PagedCache *>(PyCapsule_GetPointer(o, kCacheName));
    if (!c) return nullptr;
    try {
        return PyBool_FromLong(c->as_made());
    } catch (...) {                                              // (a storage without memory)
        Py_RETURN_FALSE;
    }
}
template <class T> T *address(const Buffer &b, long long bytes = 0) { return reinterpret_cast<T *>(static_cast<unsigned char *>(b.at) + bytes); }

// A handle and, on its device, which is the current one, what a call is given.
struct PagedCall {
    const PagedCache *c;
    explicit PagedCall(PyObject *o) {
        if (!PyCapsule_IsValid(o, kCacheName)) throw NotOrdinary{};
        c = static_cast<const PagedCache *>(PyCapsule_GetPointer(o, kCacheName));
        PyObject *dev = PyObject_CallNoArgs(g_device);
        const long now = dev ? PyLong_AsLong(dev) : -1;
        Py_XDECREF(dev);
        if (now != c->device || !c->as_made()) throw NotOrdinary{};
    }
    const at::Tensor &tensor(PyObject *o, at::ScalarType type) const {
        const at::Tensor &t = cuda_tensor(o, type);
        if (t.device().index() != c->device) throw NotOrdinary{};
        return t;
    }
    const at::Tensor &rows(PyObject *o, int64_t width) const {
        const at::Tensor &t = tensor(o, at::kBFloat16);
        if (t.dim() != 2 || t.size(0) < 1 || t.size(1) != width || t.stride(1) != 1) throw NotOrdinary{};
        return t;
    }
    const int32_t *per_sequence(PyObject *o) const {
        const at::Tensor &t = tensor(o, at::kInt);
        if (t.dim() != 1 || t.size(0) != c->max_seqs || !t.is_contiguous()) throw NotOrdinary{};
        return static_cast<const int32_t *>(t.data_ptr());
    }
    int64_t layer(PyObject *o) const {
        const int64_t v = integer(o);
        if (v < 0 || v >= c->n_layers) throw NotOrdinary{};
        return v;
    }
    const float *scale(const Buffer &b, int64_t layer) const { return b.at ? address<const float>(b) + layer * c->n_kv_heads : nullptr; }
    at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type) const {
        return at::empty(shape, at::TensorOptions().dtype(type).device(at::kCUDA, static_cast<c10::DeviceIndex>(c->device)));
    }
};
int64_t ld_of(const at::Tensor &t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }   // (torch gives a tensor of one row any stride)
uint16_t *bits(const at::Tensor &t) { return static_cast<uint16_t *>(t.data_ptr()); }
struct RowStart {
    const int32_t *p;
    int64_t n_seqs;
    RowStart(const PagedCall &call, PyObject *o) {
        const at::Tensor &t = call.tensor(o, at::kInt);
        if (t.dim() != 1 || t.size(0) < 2 || t.size(0) > call.c->max_seqs + 1 || !t.is_contiguous()) throw NotOrdinary{};
        p = static_cast<const int32_t *>(t.data_ptr());
        n_seqs = t.size(0) - 1;
    }
};
// the tensor that a call writes, new where none is given
at::Tensor output(const PagedCall &call, PyObject *o, int64_t rows, int64_t width) {
    if (o == Py_None) return call.fresh({rows, width}, at::kBFloat16);
    const at::Tensor &t = call.rows(o, width);
    if (t.size(0) != rows) throw NotOrdinary{};
    return t;
}
// body(out) -> status; the answer is out where that is 0
template <typename Body>
PyObject *tensor_of(Py_ssize_t got, Py_ssize_t want, Body body) {
    at::Tensor out;
    long status = -1;
    try {
        if (got == want) status = body(out);
        if (status == 0) {
            PyObject *o = THPVariable_Wrap(std::move(out));
            if (o) return o;
            status = -1;
        }
    } catch (...) {
        status = -1;
    }
    if (PyErr_Occurred()) PyErr_Clear();
    return PyLong_FromLong(status);
}
c10::DataPtr scratch_of(size_t bytes) { return c10::GetAllocator(c10::DeviceType::CUDA)->allocate(bytes); }
int64_t heads_of(PyObject *o) {
    const int64_t n = integer(o);
    if (n < 1 || n > 1 << 20) throw NotOrdinary{};
    return n;
}

int64_t window_of(PyObject *o, int64_t least) {
    const int64_t n = integer(o);
    if (n < least) throw NotOrdinary{};
    return n;
}

// qkv, n_q_heads, layer, row_start, q_gamma, k_gamma (None where they may be): entry(.., gammas, rope.., q_out, ..)
template <typename Entry, typename... Rope>
int prepare_on(Entry entry, const PagedCall &p, PyObject *const *a, bool normed, PyObject *given, at::Tensor &out, float eps, Rope... rope) {
    const PagedCache &c = *p.c;
    const int64_t hq = heads_of(a[1]), layer = p.layer(a[2]);
    const at::Tensor &x = p.rows(a[0], (hq + 2 * c.n_kv_heads) * 128);
    const RowStart starts(p, a[3]);
    const uint16_t *gamma[2] = {nullptr, nullptr};
    for (int i = 0; normed && i < 2; ++i) {
        const at::Tensor &g = p.tensor(a[4 + i], at::kBFloat16);
        if (g.numel() != 128 || !g.is_contiguous()) throw NotOrdinary{};
        gamma[i] = bits(g);
    }
    out = output(p, given, x.size(0), hq * 128);
    return call(entry, bits(x), x.size(0), ld_of(x), hq, c.n_kv_heads, starts.p, starts.n_seqs, gamma[0], gamma[1], eps, rope..., bits(out), ld_of(out),
                address<void>(c.pool, layer * c.layer_bytes), c.n_pages, c.page_len, (int)c.code, p.scale(c.k_scale, layer), p.scale(c.v_scale, layer),
                address<const int32_t>(c.table), c.max_pages, c.max_pages, address<const int32_t>(c.lengths), current_stream());
}
// (handle, qkv, n_q_heads, layer, row_start, q_gamma, k_gamma, eps, rope_theta, q_out)
PyObject *paged_prepare(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return tensor_of(n, 10, [&](at::Tensor &out) {
        return prepare_on(p_paged_prepare, PagedCall(a[0]), a + 1, true, a[9], out, real(a[7]), real(a[8]));
    });
}
// (handle, qkv, n_q_heads, layer, row_start, q_gamma, k_gamma, eps, layout, dims, inv_freq, magnitude, q_out)
PyObject *paged_prepare_rope(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return tensor_of(n, 13, [&](at::Tensor &out) {
        const PagedCall p(a[0]);
        const int64_t dims = integer(a[9]);
        const at::Tensor &f = p.tensor(a[10], at::kDouble);
        if (f.dim() != 1 || 2 * f.numel() != dims || !f.is_contiguous()) throw NotOrdinary{};
        return prepare_on(p_paged_prepare_rope, p, a + 1, a[5] != Py_None || a[6] != Py_None, a[12], out, real(a[7]), (int)integer(a[8]), dims,
                          static_cast<const double *>(f.data_ptr()), real(a[11]));
    });
}

// q, n_q_heads, layer, row_start, max_new: entry(.., window.., out, ..)
template <typename Entry, typename... Window>
int step_on(Entry entry, const PagedCall &p, PyObject *const *a, PyObject *workspace, PyObject *given, at::Tensor &out, Window... window) {
    const PagedCache &c = *p.c;
    const int64_t hq = heads_of(a[1]), layer = p.layer(a[2]), max_new = integer(a[4]);
    const at::Tensor &q = p.rows(a[0], hq * 128);
    const RowStart starts(p, a[3]);
    out = output(p, given, q.size(0), hq * 128);
    void *ws, *stream = current_stream();
    size_t bytes;
    c10::DataPtr scratch;
    if (workspace == Py_None) {
        bytes = p_paged_attention_workspace_bytes(max_new, hq, c.n_kv_heads);
        if (!bytes) throw NotOrdinary{};
        scratch = scratch_of(bytes);
        ws = scratch.get();
    } else {
        const at::Tensor &t = any_tensor(workspace);
        if (!t.is_cuda() || t.device().index() != c.device || !t.is_contiguous()) throw NotOrdinary{};   // (an expanded one holds less than nbytes)
        ws = t.data_ptr();
        bytes = t.nbytes();
    }
    return call(entry, bits(q), q.size(0), ld_of(q), hq, c.n_kv_heads, starts.p, starts.n_seqs, max_new, address<const void>(c.pool, layer * c.layer_bytes),
                c.n_pages, c.page_len, (int)c.code, p.scale(c.k_scale, layer), p.scale(c.v_scale, layer), address<const int32_t>(c.table), c.max_pages, c.max_pages,
                address<const int32_t>(c.lengths), window..., bits(out), ld_of(out), ws, bytes, stream);
}
// (handle, q, n_q_heads, layer, row_start, max_new, workspace, out)
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return tensor_of(n, 8, [&](at::Tensor &out) { return step_on(p_paged_attention, PagedCall(a[0]), a + 1, a[6], a[7], out); });
}
// (handle, q, n_q_heads, layer, row_start, max_new, window, sinks, workspace, out)
PyObject *paged_attention_window(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return tensor_of(n, 10, [&](at::Tensor &out) {
        return step_on(p_paged_attention_window, PagedCall(a[0]), a + 1, a[8], a[9], out, window_of(a[6], 1), window_of(a[7], 0));
    });
}

// q, n_q_heads, layer, row_start: entry(.., window.., out, ..)
template <typename Entry, typename... Window>
int prompt_on(Entry entry, const PagedCall &p, PyObject *const *a, PyObject *given, at::Tensor &out, Window... window) {
    const PagedCache &c = *p.c;
    const int64_t hq = heads_of(a[1]), layer = p.layer(a[2]);
    const at::Tensor &q = p.rows(a[0], hq * 128);
    const RowStart starts(p, a[3]);
    out = output(p, given, q.size(0), hq * 128);
    return call_with_scratch(entry, p_prompt_attention_workspace_bytes(q.size(0), hq, c.n_kv_heads, starts.n_seqs), current_stream(), bits(q), q.size(0),
                             ld_of(q), hq, c.n_kv_heads, starts.p, starts.n_seqs, address<const void>(c.pool, layer * c.layer_bytes), c.n_pages, c.page_len, (int)c.code,
                             p.scale(c.k_scale, layer), p.scale(c.v_scale, layer), address<const int32_t>(c.table), c.max_pages, c.max_pages,
                             address<const int32_t>(c.lengths), window..., bits(out), ld_of(out));
}
// (handle, q, n_q_heads, layer, row_start, out)
PyObject *prompt_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return tensor_of(n, 6, [&](at::Tensor &out) { return prompt_on(p_prompt_attention, PagedCall(a[0]), a + 1, a[5], out); });
}
// (handle, q, n_q_heads, layer, row_start, window, sinks, out)
PyObject *prompt_attention_window(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return tensor_of(n, 8, [&](at::Tensor &out) {
        return prompt_on(p_prompt_attention_window, PagedCall(a[0]), a + 1, a[7], out, window_of(a[5], 1), window_of(a[6], 0));
    });
}

// (handle, n_new)
PyObject *pages_reserve(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return tensor_of(n, 2, [&](at::Tensor &out) {
        const PagedCall p(a[0]);
        const PagedCache &c = *p.c;
        const int32_t *n_new = p.per_sequence(a[1]);
        out = p.fresh({c.max_seqs}, at::kInt);
        const c10::DataPtr scratch = scratch_of(c.workspace_bytes);
        return call(p_pages_reserve, address<int32_t>(c.table), c.max_pages, c.max_seqs, c.max_pages, address<const int32_t>(c.lengths), n_new, address<int32_t>(c.refs),
                    c.n_pages, c.page_len, static_cast<int32_t *>(out.data_ptr()), address<void>(c.pool), c.n_layers, c.n_kv_heads, (int)c.code, scratch.get(),
                    (size_t)c.workspace_bytes, current_stream());
    });
}

// (handle, parent, keep)
PyObject *pages_fork(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return status_of(n, 3, [&] {
        const PagedCall p(a[0]);
        const PagedCache &c = *p.c;
        return call(p_pages_fork, address<int32_t>(c.table), c.max_pages, c.max_seqs, c.max_pages, address<int32_t>(c.lengths), p.per_sequence(a[1]),
                    a[2] == Py_None ? nullptr : p.per_sequence(a[2]), address<int32_t>(c.refs), c.n_pages, c.page_len, current_stream());
    });
}

// (handle, window, sinks)
PyObject *pages_trim(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return status_of(n, 3, [&] {
        const PagedCall p(a[0]);
        const PagedCache &c = *p.c;
        return call(p_pages_trim, address<int32_t>(c.table), c.max_pages, c.max_seqs, c.max_pages, address<const int32_t>(c.lengths), window_of(a[1], 1), window_of(a[2], 0),
                    address<int32_t>(c.refs), c.n_pages, c.page_len, current_stream());
    });
}

// (handle)
PyObject *pages_compact(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return tensor_of(n, 1, [&](at::Tensor &out) {
        const PagedCall p(a[0]);
        const PagedCache &c = *p.c;
        out = p.fresh({c.n_pages}, at::kInt);
        const c10::DataPtr scratch = scratch_of(c.workspace_bytes);
        return call(p_pages_compact, address<int32_t>(c.table), c.max_pages, c.max_seqs, c.max_pages, address<int32_t>(c.refs), c.n_pages, c.page_len,
                    static_cast<int32_t *>(out.data_ptr()), address<void>(c.pool), c.n_layers, c.n_kv_heads, (int)c.code, scratch.get(), (size_t)c.workspace_bytes,
                    current_stream());
    });
}

// ---- tokens: calls that answer with a tuple of tensors, else with the status or -1

template <size_t N, typename Body>
PyObject *tensors_of(Py_ssize_t got, Py_ssize_t want, Body body) {
    at::Tensor out[N];
    long status = -1;
    try {
        if (got == want) status = body(out);
        if (status == 0) {
            PyObject *t = PyTuple_New(N);
            for (size_t i = 0; t && i < N; ++i) {
                PyObject *o = THPVariable_Wrap(std::move(out[i]));
                if (!o) Py_CLEAR(t);
                else PyTuple_SET_ITEM(t, i, o);
            }
            if (t) return t;
            status = -1;
        }
    } catch (...) {
        status = -1;
    }
    if (PyErr_Occurred()) PyErr_Clear();
    return PyLong_FromLong(status);
}
// Logits of one row or more on the current device, and vectors beside them.
struct Logits {
    const at::Tensor &t;
    int dtype, device;
    explicit Logits(PyObject *o) : t(any_tensor(o)) {
        if (!t.is_cuda() || t.dim() != 2 || t.size(0) < 1 || t.size(1) < 1 || t.stride(1) != 1) throw NotOrdinary{};
        if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) throw NotOrdinary{};
        dtype = t.scalar_type() == at::kFloat ? QUASAR_F32 : QUASAR_BF16;
        PyObject *dev = PyObject_CallNoArgs(g_device);
        const long now = dev ? PyLong_AsLong(dev) : -1;
        Py_XDECREF(dev);
        device = t.device().index();
        if (now != device) throw NotOrdinary{};
    }
    int64_t rows() const { return t.size(0); }
    template <class T> const T *vector(PyObject *o, at::ScalarType type, int64_t n) const {
        const at::Tensor &v = cuda_tensor(o, type);
        if (v.device().index() != device || v.dim() != 1 || v.size(0) != n || !v.is_contiguous()) throw NotOrdinary{};
        return static_cast<const T *>(v.data_ptr());
    }
    template <class T> const T *vector_or_none(PyObject *o, at::ScalarType type, int64_t n) const { return o == Py_None ? nullptr : vector<T>(o, type, n); }
    at::Tensor fresh(int64_t n, at::ScalarType type) const {
        return at::empty({n}, at::TensorOptions().dtype(type).device(at::kCUDA, static_cast<c10::DeviceIndex>(device)));
    }
};
struct TokenFilters {
    const float *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p;
    TokenFilters(const Logits &z, PyObject *const *a, int64_t n)
        : temperature(z.vector_or_none<float>(a[0], at::kFloat, n)), top_k(z.vector_or_none<int32_t>(a[1], at::kInt, n)),
          top_p(z.vector_or_none<float>(a[2], at::kFloat, n)), min_p(z.vector_or_none<float>(a[3], at::kFloat, n)) {}
};

// (logits, u, temperature, top_k, top_p, min_p) -> (token, p)
PyObject *sample_tokens(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return tensors_of<2>(n, 6, [&](at::Tensor *out) {
        const Logits z(a[0]);
        const int64_t T = z.rows(), V = z.t.size(1);
        const TokenFilters f(z, a + 2, T);
        const float *u = z.vector<float>(a[1], at::kFloat, T);
        const size_t bytes = p_sample_tokens_workspace_bytes(T, V);
        if (!bytes) throw NotOrdinary{};
        out[0] = z.fresh(T, at::kInt);
        out[1] = z.fresh(T, at::kFloat);
        const c10::DataPtr scratch = scratch_of(bytes);
        return call(p_sample_tokens, static_cast<const void *>(z.t.data_ptr()), z.dtype, T, V, ld_of(z.t), f.temperature, f.top_k, f.top_p, f.min_p, u,
                    static_cast<int32_t *>(out[0].data_ptr()), static_cast<float *>(out[1].data_ptr()), scratch.get(), bytes, current_stream());
    });
}

// (logits, row_start, draft_ids, u_accept, u_sample, temperature, top_k, top_p, min_p) -> (accepted, token, p)
PyObject *verify_tokens(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return tensors_of<3>(n, 9, [&](at::Tensor *out) {
        const Logits z(a[0]);
        const int64_t T = z.rows(), V = z.t.size(1), seqs = any_tensor(a[1]).numel() - 1;
        if (seqs < 1 || seqs > 1024) throw NotOrdinary{};
        const int32_t *starts = z.vector<int32_t>(a[1], at::kInt, seqs + 1), *draft = z.vector<int32_t>(a[2], at::kInt, T);
        const float *ua = z.vector<float>(a[3], at::kFloat, T), *us = z.vector<float>(a[4], at::kFloat, T);
        const TokenFilters f(z, a + 5, seqs);
        const size_t bytes = p_verify_tokens_workspace_bytes(T, V);
        if (!bytes) throw NotOrdinary{};
        out[0] = z.fresh(seqs, at::kInt);
        out[1] = z.fresh(seqs, at::kInt);
        out[2] = z.fresh(T, at::kFloat);
        const c10::DataPtr scratch = scratch_of(bytes);
        return call(p_verify_tokens, static_cast<const void *>(z.t.data_ptr()), z.dtype, T, V, ld_of(z.t), starts, seqs, draft, f.temperature, f.top_k, f.top_p, f.min_p,
                    ua, us, static_cast<int32_t *>(out[0].data_ptr()), static_cast<int32_t *>(out[1].data_ptr()), static_cast<float *>(out[2].data_ptr()),
                    scratch.get(), bytes, current_stream());
    });
}

// every entry point, in the order of binding.py's _NATIVE_ENTRIES
template <typename Each> void each_entry(Each each) {
    each(p_w8_linear); each(p_bf16_linear); each(p_w8a8_linear); each(p_w4_linear); each(p_w4_packed_bytes); each(p_w8a8_workspace_bytes);
    each(p_w4_workspace_bytes); each(p_w8_linear_fused); each(p_w8_gateup_swiglu); each(p_w8_fused_workspace_bytes); each(p_w8_gateup_workspace_bytes);
    each(p_paged_prepare); each(p_paged_attention); each(p_paged_attention_workspace_bytes); each(p_prompt_attention); each(p_prompt_attention_workspace_bytes);
    each(p_pages_reserve); each(p_pages_fork); each(p_pages_compact);
    each(p_paged_prepare_rope); each(p_paged_attention_window); each(p_prompt_attention_window); each(p_pages_trim);
    each(p_sample_tokens); each(p_sample_tokens_workspace_bytes); each(p_verify_tokens); each(p_verify_tokens_workspace_bytes);
}
Py_ssize_t entries() {
    Py_ssize_t n = 0;
    each_entry([&](auto &) { ++n; });
    return n;
}

// (addresses of the entry points, current device, current raw stream)
PyObject *bind(PyObject *, PyObject *args) {
    PyObject *addresses, *device, *stream;
    if (!PyArg_ParseTuple(args, "O!OO", &PyTuple_Type, &addresses, &device, &stream)) return nullptr;
    if (PyTuple_GET_SIZE(addresses) != entries()) {
        PyErr_SetString(PyExc_TypeError, "as many addresses as entry points");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < entries(); ++i)
        if (!PyLong_Check(PyTuple_GET_ITEM(addresses, i)) || (PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(addresses, i)), PyErr_Occurred())) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "addresses are integers");
            return nullptr;
        }
    Py_ssize_t i = 0;
    each_entry([&](auto &entry) {
        entry = reinterpret_cast<std::decay_t<decltype(entry)>>(static_cast<uintptr_t>(PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(addresses, i++))));
    });
    Py_INCREF(device);
    Py_INCREF(stream);
    Py_XSETREF(g_device, device);
    Py_XSETREF(g_stream, stream);
    Py_RETURN_NONE;
}

// the addresses that bind() was given
PyObject *bound(PyObject *, PyObject *) {
    PyObject *t = PyTuple_New(entries());
    if (!t) return nullptr;
    Py_ssize_t i = 0;
    each_entry([&](auto &entry) { PyTuple_SET_ITEM(t, i++, PyLong_FromUnsignedLongLong(static_cast<unsigned long long>(reinterpret_cast<uintptr_t>(entry)))); });
    return t;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(w8_linear), FAST(bf16_linear), FAST(w8a8_linear), FAST(w4_linear),
                         FAST(w8_linear_fused), FAST(w8_gateup_swiglu),
                         FAST(paged_prepare), FAST(paged_attention), FAST(prompt_attention), FAST(pages_reserve), FAST(pages_fork), FAST(pages_compact),
                         FAST(paged_prepare_rope), FAST(paged_attention_window), FAST(prompt_attention_window), FAST(pages_trim), FAST(sample_tokens), FAST(verify_tokens),
                         {"paged_cache", paged_cache, METH_VARARGS, nullptr}, {"paged_cache_as_made", paged_cache_as_made, METH_O, nullptr},
                         {"bind", bind, METH_VARARGS, nullptr}, {"bound", bound, METH_NOARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) { return PyModule_Create(&module); }
