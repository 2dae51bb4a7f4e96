// The way from Python into the draft step, for plain calls: argument checks and marshalling of binding.py's hottest functions in
// native code.  A step of a small head is over on the GPU sooner than Python has described it: d = 256, k = 1024 takes the GPU 8.0 us,
// and took the host 9.9, of which the two launches are 5 (through here 6.1; the step 9.6 -> 8.2 us, a draft round of three levels
// on a head of 5000 rows 57.4 -> 53.2).
//
// Every function here returns the status of the library's call, or -1 for a call that is not plain -- a tensor subclass or a
// wrapped tensor (vmap, functionalisation, lazy negation), a host tensor, a stride, a type or a shape that does not fit, an argument
// that is no tensor: binding.py then goes its own way, which has the checks and the messages.  Nothing is kept between calls but
// the addresses of the library's functions.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <c10/core/DispatchKeySet.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <limits>

#include "vocabtrim.h"
#include "vocabtrim_attention.h"

namespace {

decltype(&vt_draft_head_step) g_step = nullptr;
decltype(&vt_draft_head_step_static) g_step_static = nullptr;
decltype(&vt_draft_tree_level) g_level = nullptr;
decltype(&vt_tree_rerank) g_rerank = nullptr;
decltype(&vt_count_tokens) g_count = nullptr;
PyObject *g_raw_stream = nullptr;      // torch's: device index -> handle of its current stream

struct NotPlain {};

// What makes a tensor more than its memory: the pointer of such a one is not what Python would be given.
bool wrapped(const at::Tensor &t) {
    constexpr c10::DispatchKeySet special({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched,
                                           c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize,
                                           c10::DispatchKey::Conjugate, c10::DispatchKey::Negative, c10::DispatchKey::ZeroTensor});
    return t.unsafeGetTensorImpl()->key_set().has_any(special);
}
const at::Tensor &tensor(PyObject *o) {
    if (!THPVariable_CheckExact(o)) throw NotPlain();
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != c10::kStrided || !t.has_storage() || wrapped(t)) throw NotPlain();
    return t;
}
// a tensor of the device, contiguous
const at::Tensor &operand(PyObject *o) {
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda() || !t.is_contiguous()) throw NotPlain();
    return t;
}
int32_t int32(int64_t v) {
    if (v < 0 || v > std::numeric_limits<int32_t>::max()) throw NotPlain();
    return (int32_t)v;
}
int32_t int32(PyObject *o) {
    if (!PyLong_CheckExact(o)) throw NotPlain();
    int overflow = 0;
    const long v = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow != 0) throw NotPlain();
    return int32((int64_t)v);
}
int element(const at::Tensor &t) {
    if (t.scalar_type() == at::kBFloat16) return VT_BF16;
    if (t.scalar_type() == at::kFloat) return VT_F32;
    throw NotPlain();
}
void *stream_of(const at::Tensor &t) {
    const auto index = t.device().index();
    if (index < 0 || g_raw_stream == nullptr) throw NotPlain();
    PyObject *i = PyLong_FromLong(index);
    if (i == nullptr) throw NotPlain();
    PyObject *r = PyObject_CallOneArg(g_raw_stream, i);
    Py_DECREF(i);
    if (r == nullptr) throw NotPlain();
    void *p = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    if (PyErr_Occurred()) throw NotPlain();
    return p;
}

// h, W_trim, map of a step, checked against one another
struct Head {
    const void *h, *W;
    const int32_t *map;
    int h_type, w_type;
    int32_t n, k, d, m;
    void *stream;
    Head(PyObject *h_, PyObject *W_, PyObject *map_, PyObject *m_) {
        if (at::impl::torch_function_mode_enabled()) throw NotPlain();
        const at::Tensor &th = operand(h_), &tW = operand(W_), &tmap = operand(map_);
        if (th.dim() != 2 || tW.dim() != 2) throw NotPlain();
        n = int32(th.size(0));
        d = int32(th.size(1));
        k = int32(tW.size(0));
        m = int32(m_);
        if (tW.size(1) != d || tmap.numel() != k || tmap.scalar_type() != at::kInt) throw NotPlain();
        h_type = element(th);
        w_type = element(tW);
        stream = stream_of(th);
        h = th.data_ptr();
        W = tW.data_ptr();
        map = static_cast<const int32_t *>(tmap.data_ptr());
    }
};

template <typename T>
T *pointer(PyObject *o) {
    return static_cast<T *>(tensor(o).data_ptr());
}

// Runs call() without the interpreter's lock; -1 where the arguments were not plain.
template <typename F>
PyObject *status_of(F &&prepare) {
    int status = -1;
    try {
        auto call = prepare();
        Py_BEGIN_ALLOW_THREADS status = call();
        Py_END_ALLOW_THREADS
    } catch (const NotPlain &) {
        PyErr_Clear();
    } catch (const std::exception &) {
        PyErr_Clear();      // (what torch refuses here it refuses there, with its own message)
    }
    return PyLong_FromLong(status);
}

// step(h, W_trim, map, m, workspace, out_ids, out_logp)
PyObject *step(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return status_of([&] {
        if (n_args != 7 || g_step == nullptr) throw NotPlain();
        const Head x(a[0], a[1], a[2], a[3]);
        const at::Tensor &ws = tensor(a[4]);
        void *const wsp = ws.data_ptr();
        const size_t ws_bytes = (size_t)ws.numel();
        int32_t *const ids = pointer<int32_t>(a[5]);
        float *const logp = pointer<float>(a[6]);
        return [=] {
            return g_step(x.h, x.h_type, x.n, x.W, x.w_type, x.k, x.d, x.map, x.m, ids, logp, nullptr, nullptr, wsp, ws_bytes, x.stream);
        };
    });
}

// step_static(h, W_trim, map, m, out_ids, out_logp)
PyObject *step_static(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return status_of([&] {
        if (n_args != 6 || g_step_static == nullptr) throw NotPlain();
        const Head x(a[0], a[1], a[2], a[3]);
        const at::Tensor &ids = operand(a[4]), &logp = operand(a[5]);
        const int64_t items = (int64_t)x.n * x.m;
        if (ids.scalar_type() != at::kInt || logp.scalar_type() != at::kFloat || ids.numel() != items || logp.numel() != items) throw NotPlain();
        int32_t *const pi = static_cast<int32_t *>(ids.data_ptr());
        float *const pl = static_cast<float *>(logp.data_ptr());
        return [=] { return g_step_static(x.h, x.h_type, x.n, x.W, x.w_type, x.k, x.d, x.map, x.m, pi, pl, nullptr, nullptr, x.stream); };
    });
}

// level(h, W_trim, map, m, parent_cum, K, workspace, parent, token, cum, out_ids, out_logp)
PyObject *level(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return status_of([&] {
        if (n_args != 12 || g_level == nullptr) throw NotPlain();
        const Head x(a[0], a[1], a[2], a[3]);
        const at::Tensor &from = operand(a[4]);
        if (from.scalar_type() != at::kFloat || from.numel() != x.n) throw NotPlain();
        const float *const cum = static_cast<const float *>(from.data_ptr());
        const int32_t K = int32(a[5]);
        const at::Tensor &ws = tensor(a[6]);
        void *const wsp = ws.data_ptr();
        const size_t ws_bytes = (size_t)ws.numel();
        int32_t *const parent = pointer<int32_t>(a[7]), *const token = pointer<int32_t>(a[8]), *const ids = pointer<int32_t>(a[10]);
        float *const score = pointer<float>(a[9]), *const logp = pointer<float>(a[11]);
        return [=] {
            return g_level(x.h, x.h_type, x.n, x.W, x.w_type, x.k, x.d, x.map, x.m, cum, K, parent, token, score, ids, logp, wsp, ws_bytes,
                           x.stream);
        };
    });
}

// rerank(cum, T, out)
PyObject *rerank(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return status_of([&] {
        if (n_args != 3 || g_rerank == nullptr || at::impl::torch_function_mode_enabled()) throw NotPlain();
        const at::Tensor &cum = operand(a[0]), &out = tensor(a[2]);
        const int32_t T = int32(a[1]), N = int32(cum.numel());
        if (cum.scalar_type() != at::kFloat || cum.dim() != 1 || !out.is_cuda() || out.scalar_type() != at::kInt || out.numel() < T) throw NotPlain();
        const float *const pc = static_cast<const float *>(cum.data_ptr());
        int32_t *const po = static_cast<int32_t *>(out.data_ptr());
        void *const stream = stream_of(cum);
        return [=] { return g_rerank(pc, N, T, po, stream); };
    });
}

// count(ids, V, counts, workspace)
PyObject *count(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return status_of([&] {
        if (n_args != 4 || g_count == nullptr || at::impl::torch_function_mode_enabled()) throw NotPlain();
        const at::Tensor &ids = operand(a[0]), &counts = operand(a[2]), &ws = operand(a[3]);
        const int type = ids.scalar_type() == at::kInt ? VT_I32 : ids.scalar_type() == at::kLong ? VT_I64 : -1;
        if (type < 0) throw NotPlain();
        const int32_t V = int32(a[1]);
        const int64_t n = ids.numel();
        const void *const p = n != 0 ? ids.data_ptr() : nullptr;
        int64_t *const pc = static_cast<int64_t *>(counts.data_ptr());
        void *const wsp = ws.data_ptr(), *const stream = stream_of(ids);
        const size_t ws_bytes = (size_t)ws.numel();
        return [=] { return g_count(p, type, n, V, pc, nullptr, wsp, ws_bytes, stream); };
    });
}

// ------------------------------------------------------------------ the attention's calls (attention.py)
// These make their results, too, and return them; None for a call that is not plain, a number for a status that is not VT_OK.
decltype(&vt_qk_norm_rope) g_norm = nullptr;
decltype(&vt_qk_norm_rope_backward) g_norm_backward = nullptr;
decltype(&vt_qk_norm_rope_backward_ws_bytes) g_norm_backward_ws = nullptr;
decltype(&vt_qkv_to_cache) g_to_cache = nullptr;
decltype(&vt_kv_cache_read) g_read = nullptr;
decltype(&vt_paged_attention) g_attend = nullptr;
decltype(&vt_paged_attention_window) g_attend_window = nullptr;

bool given(PyObject *o) { return o != Py_None; }
// A gradient is asked for of the tensor, or it has a tangent: autograd's business, or a refusal
const at::Tensor &plain(const at::Tensor &t) {
    if ((c10::GradMode::is_enabled() && t.requires_grad()) || t._fw_grad(0).defined()) throw NotPlain();
    return t;
}

// A tensor of heads [n, heads, head_dim], its rows apart
struct Heads {
    at::Tensor t;
    void *p = nullptr;
    int64_t n = 0, stride = 0;
    int32_t heads = 0, D = 0;
    Heads() = default;
    explicit Heads(const at::Tensor &x) : t(x) {
        plain(t);
        if (!t.is_cuda() || t.dim() != 3) throw NotPlain();
        n = t.size(0);
        heads = int32(t.size(1));
        D = int32(t.size(2));
        if (n == 0 || heads == 0 || D < 2 || t.stride(2) != 1 || (heads > 1 && t.stride(1) != D)) throw NotPlain();
        stride = n > 1 ? t.stride(0) : (int64_t)heads * D;
        p = t.data_ptr();
    }
    void like(const Heads &x) const {
        if (n != x.n || heads != x.heads || D != x.D || t.scalar_type() != x.t.scalar_type()) throw NotPlain();
    }
};
Heads heads_of(PyObject *o) { return Heads(tensor(o)); }
// ... of a result, made where none is given
Heads result(PyObject *o, const Heads &like) {
    Heads r(given(o) ? tensor(o) : at::empty({like.n, like.heads, like.D}, like.t.options()));
    r.like(like);
    return r;
}
struct Index {
    const void *p = nullptr;
    int type = VT_I32;
    int64_t n = 0;
    Index() = default;
    explicit Index(PyObject *o) {
        const at::Tensor &t = operand(o);
        if (t.scalar_type() != at::kInt && t.scalar_type() != at::kLong) throw NotPlain();
        type = t.scalar_type() == at::kInt ? VT_I32 : VT_I64;
        n = t.numel();
        p = t.data_ptr();
    }
};
double number(PyObject *o) {
    if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
    if (!PyLong_CheckExact(o)) throw NotPlain();
    return (double)int32(o);
}
bool truth(PyObject *o) {
    if (o != Py_True && o != Py_False) throw NotPlain();
    return o == Py_True;
}
// Weights, table and positions of a call on n rows of heads of size D: positions, table, q_weight, k_weight, eps, interleaved
struct Norm {
    const void *wq = nullptr, *wk = nullptr;
    const float *table = nullptr;
    int64_t rows = 0;
    int32_t rot = 0;
    Index positions;
    float eps;
    int style;
    Norm(PyObject *const *a, const Heads &x) {
        if (given(a[0]) != given(a[1]) || given(a[2]) != given(a[3])) throw NotPlain();
        if (given(a[1])) {
            const at::Tensor &t = plain(operand(a[1]));
            if (t.scalar_type() != at::kFloat || t.dim() != 2) throw NotPlain();
            table = static_cast<const float *>(t.data_ptr());
            rows = t.size(0);
            rot = int32(t.size(1));
            positions = Index(a[0]);
            if (positions.n != x.n) throw NotPlain();
        }
        if (given(a[2])) {
            wq = weight(a[2], x);
            wk = weight(a[3], x);
        }
        eps = (float)number(a[4]);
        style = truth(a[5]) ? VT_ROPE_NEIGHBOURS : VT_ROPE_HALVES;
    }
    static const void *weight(PyObject *o, const Heads &x) {
        const at::Tensor &t = plain(operand(o));
        if (t.scalar_type() != x.t.scalar_type() || t.numel() != x.D) throw NotPlain();
        return t.data_ptr();
    }
};

PyObject *wrap(const at::Tensor &t) { return THPVariable_Wrap(t); }
template <typename... T>
PyObject *tuple_of(const T &...t) {
    PyObject *items[] = {t...};
    constexpr Py_ssize_t count = sizeof...(t);
    PyObject *r = PyTuple_New(count);
    for (Py_ssize_t i = 0; i < count; ++i) {
        if (r != nullptr && items[i] != nullptr) PyTuple_SET_ITEM(r, i, items[i]);
        else Py_XDECREF(items[i]);
    }
    return r;
}
template <typename F>
PyObject *result_of(F &&call) {
    try {
        if (at::impl::torch_function_mode_enabled()) throw NotPlain();
        return call();
    } catch (const NotPlain &) {
        PyErr_Clear();
    } catch (const std::exception &) {
        PyErr_Clear();
    }
    Py_RETURN_NONE;
}
template <typename F>
int unlocked(F &&call) {
    int status;
    Py_BEGIN_ALLOW_THREADS status = call();
    Py_END_ALLOW_THREADS
    return status;
}

// norm(q, k, positions, table, q_weight, k_weight, eps, interleaved, q_out, k_out)
PyObject *norm(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return result_of([&]() -> PyObject * {
        if (n_args != 10 || g_norm == nullptr) throw NotPlain();
        const Heads q = heads_of(a[0]), k = heads_of(a[1]);
        if (k.n != q.n || k.D != q.D || k.t.scalar_type() != q.t.scalar_type()) throw NotPlain();
        const Norm x(a + 2, q);
        const Heads qo = result(a[8], q), ko = result(a[9], k);
        const int type = element(q.t);
        void *const stream = stream_of(q.t);
        const int status = unlocked([&] {
            return g_norm(q.p, q.stride, k.p, k.stride, type, q.n, q.heads, k.heads, q.D, x.wq, x.wk, x.eps, x.table, x.rows, x.rot, x.style,
                          x.positions.p, x.positions.type, qo.p, qo.stride, ko.p, ko.stride, stream);
        });
        return status != VT_OK ? PyLong_FromLong(status) : tuple_of(wrap(qo.t), wrap(ko.t));
    });
}

// norm_backward(gq, gk, q, k, positions, table, q_weight, k_weight, eps, interleaved): with weights, results and workspace made here
PyObject *norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return result_of([&]() -> PyObject * {
        if (n_args != 10 || g_norm_backward == nullptr || !given(a[6])) throw NotPlain();
        const Heads gq = heads_of(a[0]), gk = heads_of(a[1]), q = heads_of(a[2]), k = heads_of(a[3]);
        gq.like(q);
        gk.like(k);
        if (k.n != q.n || k.D != q.D || k.t.scalar_type() != q.t.scalar_type()) throw NotPlain();
        const Norm x(a + 4, q);
        const Heads dq = result(Py_None, q), dk = result(Py_None, k);
        const int type = element(q.t);
        const at::Tensor dw = at::empty({2, q.D}, q.t.options().dtype(at::kFloat));
        float *const pw = dw.data_ptr<float>();
        const size_t ws_bytes = g_norm_backward_ws(q.n, q.D);
        const at::Tensor ws = at::empty({(int64_t)ws_bytes}, q.t.options().dtype(at::kByte));
        void *const wsp = ws.data_ptr(), *const stream = stream_of(q.t);
        const int status = unlocked([&] {
            return g_norm_backward(gq.p, gq.stride, gk.p, gk.stride, q.p, q.stride, k.p, k.stride, type, q.n, q.heads, k.heads, q.D, x.wq, x.wk,
                                   x.eps, x.table, x.rows, x.rot, x.style, x.positions.p, x.positions.type, dq.p, dq.stride, dk.p, dk.stride, pw,
                                   pw + q.D, wsp, ws_bytes, stream);
        });
        return status != VT_OK ? PyLong_FromLong(status) : tuple_of(wrap(dq.t), wrap(dk.t), wrap(dw.select(0, 0)), wrap(dw.select(0, 1)));
    });
}

const vt_kv_cache *cache_of(PyObject *address) {
    const auto *c = static_cast<const vt_kv_cache *>(PyLong_AsVoidPtr(address));
    if (c == nullptr || PyErr_Occurred()) throw NotPlain();
    return c;
}

// to_cache(q, k, v, cache address, slots, positions, table, q_weight, k_weight, eps, interleaved, q_out)
PyObject *to_cache(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return result_of([&]() -> PyObject * {
        if (n_args != 12 || g_to_cache == nullptr) throw NotPlain();
        const Heads q = heads_of(a[0]), k = heads_of(a[1]), v = heads_of(a[2]);
        v.like(k);
        const vt_kv_cache *const cache = cache_of(a[3]);
        if (k.n != q.n || k.D != q.D || k.t.scalar_type() != q.t.scalar_type() || k.heads != cache->heads || k.D != cache->head_dim) throw NotPlain();
        const Index slots(a[4]);
        if (slots.n != k.n) throw NotPlain();
        const Norm x(a + 5, k);
        const Heads qo = result(a[11], q);
        const int type = element(q.t);
        void *const stream = stream_of(q.t);
        const int status = unlocked([&] {
            return g_to_cache(q.p, q.stride, k.p, k.stride, v.p, v.stride, type, k.n, q.heads, x.wq, x.wk, x.eps, x.table, x.rows, x.rot, x.style,
                              x.positions.p, x.positions.type, qo.p, qo.stride, cache, slots.p, slots.type, stream);
        });
        return status != VT_OK ? PyLong_FromLong(status) : wrap(qo.t);
    });
}

// cache_read(cache address, slots, f32)
PyObject *cache_read(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return result_of([&]() -> PyObject * {
        if (n_args != 3 || g_read == nullptr) throw NotPlain();
        const vt_kv_cache *const cache = cache_of(a[0]);
        const Index slots(a[1]);
        if (slots.n == 0) throw NotPlain();
        const bool f32 = truth(a[2]);
        const at::Tensor &s = THPVariable_Unpack(a[1]);
        const auto options = s.options().dtype(f32 ? at::kFloat : at::kBFloat16);
        const at::Tensor k = at::empty({slots.n, cache->heads, cache->head_dim}, options), v = at::empty({slots.n, cache->heads, cache->head_dim}, options);
        void *const kp = k.data_ptr(), *const vp = v.data_ptr(), *const stream = stream_of(s);
        const int status = unlocked([&] { return g_read(cache, slots.p, slots.type, slots.n, kp, vp, f32 ? VT_F32 : VT_BF16, stream); });
        return status != VT_OK ? PyLong_FromLong(status) : tuple_of(wrap(k), wrap(v));
    });
}

// attend(q, cache address, page_table, lengths, row_start, max_rows, tail_mask, max_length, scale, workspace, out, return_lse, out_lse, window, sinks,
// positions)
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return result_of([&]() -> PyObject * {
        if (n_args != 16 || g_attend == nullptr || g_attend_window == nullptr) throw NotPlain();
        const Heads q = heads_of(a[0]);
        const vt_kv_cache *const cache = cache_of(a[1]);
        const at::Tensor &table = operand(a[2]), &lengths = operand(a[3]), &ws = operand(a[9]);
        if (table.scalar_type() != at::kInt || table.dim() != 2 || lengths.scalar_type() != at::kInt || q.D != cache->head_dim) throw NotPlain();
        const int32_t requests = int32(table.size(0)), pages = int32(table.size(1));
        if (lengths.numel() != requests || ws.scalar_type() != at::kByte) throw NotPlain();
        const int32_t *start = nullptr;
        int32_t max_rows = 1;
        if (given(a[4])) {
            const at::Tensor &t = operand(a[4]);
            if (t.scalar_type() != at::kInt || t.numel() != (int64_t)requests + 1) throw NotPlain();
            start = static_cast<const int32_t *>(t.data_ptr());
            max_rows = int32(a[5]);
        } else if (given(a[5])) {
            max_rows = int32(a[5]);
        }
        const uint64_t *mask = nullptr;
        if (given(a[6])) {
            const at::Tensor &t = operand(a[6]);
            if (t.scalar_type() != at::kLong || t.numel() != q.n) throw NotPlain();
            mask = static_cast<const uint64_t *>(t.data_ptr());
        }
        const int64_t most = given(a[7]) ? int32(a[7]) : (int64_t)pages * cache->page_size;
        const float scale = given(a[8]) ? (float)number(a[8]) : (float)std::pow((double)q.D, -0.5);
        const bool windowed = given(a[13]);
        const int64_t window = windowed ? int32(a[13]) : 0, sinks = int32(a[14]);
        Index positions;
        if (given(a[15])) {
            if (mask == nullptr) throw NotPlain();
            positions = Index(a[15]);
            if (positions.n != q.n) throw NotPlain();
        }
        if (!windowed && (sinks != 0 || positions.p != nullptr)) throw NotPlain();
        const Heads out = result(a[10], q);
        const bool with_lse = truth(a[11]);
        at::Tensor lse;
        if (given(a[12])) {
            lse = plain(operand(a[12]));
            if (lse.scalar_type() != at::kFloat || lse.numel() != q.n * q.heads) throw NotPlain();
        } else if (with_lse) {
            lse = at::empty({q.n, q.heads}, q.t.options().dtype(at::kFloat));
        }
        float *const pl = lse.defined() ? lse.data_ptr<float>() : nullptr;
        const int type = element(q.t);
        const int32_t *const pt = static_cast<const int32_t *>(table.data_ptr()), *const len = static_cast<const int32_t *>(lengths.data_ptr());
        void *const wsp = ws.data_ptr(), *const stream = stream_of(q.t);
        const size_t ws_bytes = (size_t)ws.numel();
        const int status = unlocked([&] {
            if (!windowed)
                return g_attend(q.p, q.stride, type, q.n, q.heads, cache, pt, pages, len, requests, start, max_rows, mask, most, scale, out.p, out.stride,
                                pl, wsp, ws_bytes, stream);
            return g_attend_window(q.p, q.stride, type, q.n, q.heads, cache, pt, pages, len, requests, start, max_rows, mask, positions.p,
                                   positions.type, window, sinks, most, scale, out.p, out.stride, pl, wsp, ws_bytes, stream);
        });
        if (status != VT_OK) return PyLong_FromLong(status);
        return with_lse ? tuple_of(wrap(out.t), wrap(lse)) : wrap(out.t);
    });
}

// connect(raw_stream, step, step_static, level, rerank, count, norm, norm_backward, its workspace's size, to_cache, cache_read, attend,
// attend_window):
// torch's stream query and the addresses of the library's functions
PyObject *connect(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    constexpr int kFunctions = 12;
    if (n_args != 1 + kFunctions) {
        PyErr_SetString(PyExc_TypeError, "connect takes torch's stream query and twelve addresses");
        return nullptr;
    }
    void *p[kFunctions];
    for (int i = 0; i < kFunctions; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i + 1]);
        if (PyErr_Occurred()) return nullptr;
    }
    Py_INCREF(a[0]);
    Py_XDECREF(g_raw_stream);
    g_raw_stream = a[0];
    g_step = reinterpret_cast<decltype(g_step)>(p[0]);
    g_step_static = reinterpret_cast<decltype(g_step_static)>(p[1]);
    g_level = reinterpret_cast<decltype(g_level)>(p[2]);
    g_rerank = reinterpret_cast<decltype(g_rerank)>(p[3]);
    g_count = reinterpret_cast<decltype(g_count)>(p[4]);
    g_norm = reinterpret_cast<decltype(g_norm)>(p[5]);
    g_norm_backward = reinterpret_cast<decltype(g_norm_backward)>(p[6]);
    g_norm_backward_ws = reinterpret_cast<decltype(g_norm_backward_ws)>(p[7]);
    g_to_cache = reinterpret_cast<decltype(g_to_cache)>(p[8]);
    g_read = reinterpret_cast<decltype(g_read)>(p[9]);
    g_attend = reinterpret_cast<decltype(g_attend)>(p[10]);
    g_attend_window = reinterpret_cast<decltype(g_attend_window)>(p[11]);
    Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyCFunction fast() {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F));
}
PyMethodDef methods[] = {{"connect", fast<connect>(), METH_FASTCALL, nullptr},
                         {"step", fast<step>(), METH_FASTCALL, nullptr},
                         {"step_static", fast<step_static>(), METH_FASTCALL, nullptr},
                         {"level", fast<level>(), METH_FASTCALL, nullptr},
                         {"rerank", fast<rerank>(), METH_FASTCALL, nullptr},
                         {"count", fast<count>(), METH_FASTCALL, nullptr},
                         {"norm", fast<norm>(), METH_FASTCALL, nullptr},
                         {"norm_backward", fast<norm_backward>(), METH_FASTCALL, nullptr},
                         {"to_cache", fast<to_cache>(), METH_FASTCALL, nullptr},
                         {"cache_read", fast<cache_read>(), METH_FASTCALL, nullptr},
                         {"attend", fast<attend>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_vt_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch and the interpreter whose headers this was compiled with (binding.py compares them with its own)
PyMODINIT_FUNC PyInit__vt_bind(void) {
    PyObject *m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "built_for", VT_BUILT_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
