// _marshal: what the binding's Python does for a call of the usual form (device tensors of the right types on the current device,
// outputs left to the binding), in native code.  Every function takes the binding's arguments with the current device and its stream
// behind them and returns what the entry point returns, the library's code if that is not 0, or None for a call of any other form,
// which the Python then takes, checks and answers or refuses.  Results are the same either way.
//
// A call on a small corpus is bound by the host: Python checks, two allocations and the conversions of a dozen arguments took 5.4 us of
// the 8.3 of a call of one launch (11.2 of two); here they take 1.9.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "../../include/ann.h"

namespace {

// the entry points of the library that the binding has loaded
decltype(&ann_flat_search_typed) flat_search;
decltype(&ann_flat_search_after_typed) flat_search_after;
decltype(&ann_graph_search_typed) graph_search;
decltype(&ann_graph_search_entries_typed) graph_search_entries;
decltype(&ann_graph_search_nonstall_typed) graph_search_nonstall;
decltype(&ann_gather_ids) gather_ids;
decltype(&ann_priority_order) priority_order;
decltype(&ann_qk_norm_rotate) qk_norm_rotate;
decltype(&ann_paged_attention) paged_attention;
decltype(&ann_cache_evict) cache_evict;
decltype(&ann_logit_rules) logit_rules;
decltype(&ann_rotate_append) rotate_append;
decltype(&ann_chunk_attention) chunk_attention;
decltype(&ann_shared_attention) shared_attention;

struct OtherForm {};                                      // the call is not of the usual form

const at::Tensor &tensor(PyObject *o) {
    if (!THPVariable_CheckExact(o)) throw OtherForm();
    return THPVariable_Unpack(o);
}
// a contiguous device tensor with memory of its own
const at::Tensor &on_device(PyObject *o, int64_t device, at::ScalarType type) {
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || !t.has_storage() ||
        t.unsafeGetTensorImpl()->is_python_dispatch() || !t.is_contiguous())
        throw OtherForm();
    return t;
}
int64_t integer(PyObject *o, int64_t least, int64_t most) {
    if (!PyLong_CheckExact(o)) throw OtherForm();
    int overflow = 0;
    const int64_t v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow != 0 || v < least || v > most) throw OtherForm();
    return v;
}
int32_t int32(PyObject *o) { return (int32_t)integer(o, INT32_MIN, INT32_MAX); }
int32_t count(int64_t n) {
    if (n > INT32_MAX) throw OtherForm();
    return (int32_t)n;
}
void *stream_of(PyObject *o) {
    void *p = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        throw OtherForm();
    }
    return p;
}

struct Call {                                             // corpus, queries and what they say
    int64_t device, N;
    int32_t d, dtype, B;
    const at::Tensor *x, *q;
    Call(PyObject *corpus, PyObject *queries, int64_t device_) : device(device_) {
        const at::ScalarType type = tensor(corpus).scalar_type();
        dtype = type == at::kHalf ? ANN_F16 : type == at::kBFloat16 ? ANN_BF16 : type == at::kFloat ? ANN_F32 : -1;
        if (dtype < 0) throw OtherForm();
        x = &on_device(corpus, device, type);
        q = &on_device(queries, device, type);
        if (x->dim() != 2 || q->dim() != 2 || x->size(1) != q->size(1)) throw OtherForm();
        N = x->size(0);
        d = count(x->size(1));
        B = count(q->size(0));
    }
};
at::Tensor empty(at::IntArrayRef size, at::ScalarType type, const at::Tensor &like) {
    return at::empty(size, at::TensorOptions().dtype(type).device(like.device()));
}
const int32_t *graph_of(PyObject *o, const Call &c, int32_t *R) {
    const at::Tensor &g = on_device(o, c.device, at::kInt);
    if (g.dim() != 2 || g.size(0) != c.N) throw OtherForm();
    *R = count(g.size(1));
    return static_cast<const int32_t *>(g.data_ptr());
}
const int32_t *entries_of(PyObject *o, const Call &c, int32_t *E) {
    const at::Tensor &e = on_device(o, c.device, at::kInt);
    if (!((e.dim() == 1 || (e.dim() == 2 && e.size(1) >= 1)) && e.size(0) == c.B)) throw OtherForm();
    *E = e.dim() == 1 ? 1 : count(e.size(1));
    return static_cast<const int32_t *>(e.data_ptr());
}
int32_t *ints(const at::Tensor &t) { return static_cast<int32_t *>(t.data_ptr()); }
float *floats(const at::Tensor &t) { return static_cast<float *>(t.data_ptr()); }

PyObject *answer(int code, std::initializer_list<const at::Tensor *> out) {
    if (code != ANN_OK) return PyLong_FromLong(code);
    PyObject *tuple = PyTuple_New((Py_ssize_t)out.size());
    if (!tuple) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor *t : out) {
        PyObject *o = THPVariable_Wrap(*t);
        if (!o) {
            Py_DECREF(tuple);
            return nullptr;
        }
        PyTuple_SET_ITEM(tuple, i++, o);
    }
    return tuple;
}

// body(args), and None where that says so, or meets an error: the Python gives it its name.
template <int N, class Body>
PyObject *usual(PyObject *const *args, Py_ssize_t n, Body &&body) {
    if (n != N || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) Py_RETURN_NONE;
    try {
        return body(args);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}
template <class F, class... A>
int without_gil(F *f, A... a) {
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = f(a...);
    Py_END_ALLOW_THREADS
    return code;
}

// corpus, queries, k, after scores, after ids (None, None: no boundary), device, stream
PyObject *flat(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<7>(args, n, [](PyObject *const *a) {
        const Call c(a[0], a[1], integer(a[5], 0, INT32_MAX));
        const int32_t k = int32(a[2]);
        const at::Tensor *s = nullptr, *i = nullptr;
        if (a[3] != Py_None || a[4] != Py_None) {
            s = &on_device(a[3], c.device, at::kFloat);
            i = &on_device(a[4], c.device, at::kInt);
            if (s->dim() != 1 || i->dim() != 1 || s->size(0) != c.B || i->size(0) != c.B) throw OtherForm();
        }
        void *stream = stream_of(a[6]);
        const at::Tensor ids = empty({c.B, k}, at::kInt, *c.x), scores = empty({c.B, k}, at::kFloat, *c.x);
        const int code = s ? without_gil(flat_search_after, c.x->data_ptr(), c.N, c.d, c.dtype, c.q->data_ptr(), c.B, k, floats(*s),
                                         ints(*i), ints(ids), floats(scores), stream)
                           : without_gil(flat_search, c.x->data_ptr(), c.N, c.d, c.dtype, c.q->data_ptr(), c.B, k, ints(ids),
                                         floats(scores), stream);
        return answer(code, {&ids, &scores});
    });
}

// corpus, graph, entry (ENTRIES: the tensor of one entry per query, else a number), queries, k, ef, device, stream
template <bool ENTRIES>
PyObject *graph_of_either(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<8>(args, n, [](PyObject *const *a) {
        const Call c(a[0], a[3], integer(a[6], 0, INT32_MAX));
        const int32_t k = int32(a[4]), ef = int32(a[5]);
        int32_t R, E = 0;
        const int32_t *g = graph_of(a[1], c, &R), *entries = nullptr;
        int32_t entry = 0;
        if (ENTRIES) {
            entries = entries_of(a[2], c, &E);
            if (tensor(a[2]).dim() != 1) throw OtherForm();
        } else {
            entry = int32(a[2]);
        }
        void *stream = stream_of(a[7]);
        const at::Tensor ids = empty({c.B, k}, at::kInt, *c.x), scores = empty({c.B, k}, at::kFloat, *c.x);
        const int code = ENTRIES ? without_gil(graph_search_entries, c.x->data_ptr(), c.N, c.d, c.dtype, g, R, entries, c.q->data_ptr(), c.B, k,
                                         ef, ints(ids), floats(scores), stream)
                                 : without_gil(graph_search, c.x->data_ptr(), c.N, c.d, c.dtype, g, R, entry, c.q->data_ptr(), c.B, k, ef,
                                         ints(ids), floats(scores), stream);
        return answer(code, {&ids, &scores});
    });
}

PyObject *graph(PyObject *self, PyObject *const *args, Py_ssize_t n) { return graph_of_either<false>(self, args, n); }
PyObject *graph_entries(PyObject *self, PyObject *const *args, Py_ssize_t n) { return graph_of_either<true>(self, args, n); }

// corpus, graph, entry, queries, k, ef, entries or None, tau, window, device, stream
PyObject *nonstall(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<11>(args, n, [](PyObject *const *a) {
        const Call c(a[0], a[3], integer(a[9], 0, INT32_MAX));
        const int32_t entry = int32(a[2]), k = int32(a[4]), ef = int32(a[5]), window = int32(a[8]);
        int32_t R, E = 0;
        const int32_t *g = graph_of(a[1], c, &R), *entries = a[6] != Py_None ? entries_of(a[6], c, &E) : nullptr;
        if (!PyFloat_CheckExact(a[7])) throw OtherForm();
        const float tau = (float)PyFloat_AS_DOUBLE(a[7]);
        void *stream = stream_of(a[10]);
        const at::Tensor ids = empty({c.B, k}, at::kInt, *c.x), scores = empty({c.B, k}, at::kFloat, *c.x),
                         stats = empty({c.B, 3}, at::kInt, *c.x), ema = empty({c.B}, at::kFloat, *c.x);
        const int code = without_gil(graph_search_nonstall, c.x->data_ptr(), c.N, c.d, c.dtype, g, R, entry, c.q->data_ptr(), c.B, k, ef,
                                     entries, E, tau, window, nullptr, ints(ids), floats(scores), ints(stats), floats(ema), stream);
        return answer(code, {&ids, &scores, &stats, &ema});
    });
}

// table, idx, device, stream
PyObject *gather(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<4>(args, n, [](PyObject *const *a) {
        const int64_t device = integer(a[2], 0, INT32_MAX);
        const at::Tensor &table = on_device(a[0], device, at::kInt), &idx = on_device(a[1], device, at::kInt);
        if (idx.dim() != 1) throw OtherForm();
        void *stream = stream_of(a[3]);
        const at::Tensor out = empty({idx.size(0)}, at::kInt, idx);
        return answer(without_gil(gather_ids, ints(table), table.numel(), ints(idx), idx.numel(), ints(out), stream), {&out});
    });
}

// R, W, C, Wcur, G, device, stream
PyObject *order(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<7>(args, n, [](PyObject *const *a) {
        const int64_t device = integer(a[5], 0, INT32_MAX);
        const at::Tensor &R = on_device(a[0], device, at::kInt), &W = on_device(a[1], device, at::kDouble),
                         &C = on_device(a[2], device, at::kInt), &Wcur = on_device(a[3], device, at::kDouble);
        const int32_t m = count(R.numel()), G = int32(a[4]);
        if (W.numel() != m || C.numel() != m || Wcur.numel() != m) throw OtherForm();
        void *stream = stream_of(a[6]);
        const at::Tensor level = empty({m}, at::kInt, R), rank = empty({m}, at::kInt, R);
        const int code = without_gil(priority_order, ints(R), static_cast<const double *>(W.data_ptr()), ints(C),
                                     static_cast<const double *>(Wcur.data_ptr()), m, G, ints(level), ints(rank), stream);
        return answer(code, {&level, &rank});
    });
}

// ---- the step between two retrievals

int32_t type_code(const at::Tensor &t) {
    const at::ScalarType type = t.scalar_type();
    if (type == at::kHalf) return ANN_F16;
    if (type == at::kBFloat16) return ANN_BF16;
    if (type == at::kFloat) return ANN_F32;
    throw OtherForm();
}
// a device tensor of `dim` dimensions with memory of its own whose rows are contiguous
const at::Tensor &rows_on_device(PyObject *o, int64_t device, at::ScalarType type, int64_t dim) {
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || !t.has_storage() ||
        t.unsafeGetTensorImpl()->is_python_dispatch() || t.dim() != dim || (t.size(dim - 1) > 1 && t.stride(dim - 1) != 1))
        throw OtherForm();
    return t;
}
const at::Tensor &array_on_device(PyObject *o, int64_t device, at::ScalarType type, std::initializer_list<int64_t> size) {
    const at::Tensor &t = on_device(o, device, type);
    if (t.dim() != (int64_t)size.size()) throw OtherForm();
    int64_t i = 0;
    for (int64_t n : size) {
        if (n >= 0 && t.size(i) != n) throw OtherForm();
        ++i;
    }
    return t;
}
int64_t step_of(const at::Tensor &t, int64_t i) { return t.size(i) > 1 ? t.stride(i) : 0; }
double number(PyObject *o) {
    if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
    return (double)integer(o, -(1ll << 53), 1ll << 53);
}
ann_paged_cache cache_of(PyObject *keys, PyObject *values, int64_t device) {
    const at::ScalarType type = tensor(keys).scalar_type();
    const at::Tensor &k = rows_on_device(keys, device, type, 4), &v = rows_on_device(values, device, type, 4);
    if (k.sizes() != v.sizes()) throw OtherForm();
    ann_paged_cache c;
    c.k = k.data_ptr();
    c.v = v.data_ptr();
    c.k_page = step_of(k, 0); c.k_head = step_of(k, 1); c.k_slot = step_of(k, 2);
    c.v_page = step_of(v, 0); c.v_head = step_of(v, 1); c.v_slot = step_of(v, 2);
    c.pages = count(k.size(0)); c.heads = count(k.size(1)); c.slots = count(k.size(2)); c.d = count(k.size(3));
    c.dtype = type_code(k);
    return c;
}

// qkv, q_weight, k_weight, positions, cos_sin, slots, k_cache, v_cache, eps, interleaved, device, stream
PyObject *rotate(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<12>(args, n, [](PyObject *const *a) {
        const int64_t device = integer(a[10], 0, INT32_MAX);
        const ann_paged_cache c = cache_of(a[6], a[7], device);
        const at::ScalarType type = tensor(a[6]).scalar_type();
        const at::Tensor &qkv = rows_on_device(a[0], device, type, 3);
        const int32_t T = count(qkv.size(0)), q_heads = count(qkv.size(1)) - 2 * c.heads;
        if (qkv.size(2) != c.d || c.heads > 65536 || q_heads < 1) throw OtherForm();
        const at::Tensor &qw = array_on_device(a[1], device, type, {c.d}), &kw = array_on_device(a[2], device, type, {c.d});
        const at::Tensor &positions = array_on_device(a[3], device, at::kInt, {T}), &turn = array_on_device(a[4], device, at::kFloat, {-1, -1}),
                         &slots = array_on_device(a[5], device, at::kInt, {T});
        const double eps = number(a[8]);
        if (!PyBool_Check(a[9])) throw OtherForm();
        void *stream = stream_of(a[11]);
        const at::Tensor q = empty({T, q_heads, c.d}, type, qkv);
        return answer(without_gil(qk_norm_rotate, (const void *)qkv.data_ptr(), step_of(qkv, 0), step_of(qkv, 1), T, q_heads, (const void *)qw.data_ptr(),
                                  (const void *)kw.data_ptr(), (float)eps, (const int32_t *)ints(positions), (const float *)floats(turn),
                                  count(turn.size(0)), count(turn.size(1)), (int32_t)(a[9] == Py_True), (const int32_t *)ints(slots), &c,
                                  q.data_ptr(), stream), {&q});
    });
}

// q, k_cache, v_cache, page_table, lengths, scale or None, window, max_length or None, mass or None, device, stream
PyObject *attend(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<11>(args, n, [](PyObject *const *a) {
        const int64_t device = integer(a[9], 0, INT32_MAX);
        const ann_paged_cache c = cache_of(a[1], a[2], device);
        const at::ScalarType type = tensor(a[1]).scalar_type();
        const at::Tensor &q = rows_on_device(a[0], device, type, 3);
        const int32_t B = count(q.size(0)), q_heads = count(q.size(1));
        if (q.size(2) != c.d) throw OtherForm();
        const at::Tensor &table = array_on_device(a[3], device, at::kInt, {B, -1}), &lengths = array_on_device(a[4], device, at::kInt, {B});
        const double scale = a[5] == Py_None ? 1.0 / std::sqrt((double)c.d) : number(a[5]);
        const int32_t window = int32(a[6]), width = count(table.size(1)),
                      most = a[7] == Py_None ? (int32_t)std::min<int64_t>(INT32_MAX, (int64_t)width * c.slots) : int32(a[7]);
        const at::Tensor *mass = a[8] == Py_None ? nullptr : &array_on_device(a[8], device, at::kFloat, {B, c.heads, -1});
        void *stream = stream_of(a[10]);
        const at::Tensor out = empty({B, q_heads, c.d}, type, q), lse = empty({B, q_heads}, at::kFloat, q);
        return answer(without_gil(paged_attention, (const void *)q.data_ptr(), step_of(q, 0), step_of(q, 1), B, q_heads, &c, (const int32_t *)ints(table), width,
                                  (const int32_t *)ints(lengths), most, (float)scale, window, out.data_ptr(), floats(lse),
                                  mass ? floats(*mass) : nullptr, mass ? mass->size(2) : (int64_t)0, stream), {&out, &lse});
    });
}

// k_cache, v_cache, page_table, lengths, mass, new_page_table, budget, first, recent, device, stream
PyObject *evict(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<11>(args, n, [](PyObject *const *a) {
        const int64_t device = integer(a[9], 0, INT32_MAX);
        const ann_paged_cache c = cache_of(a[0], a[1], device);
        const at::Tensor &table = array_on_device(a[2], device, at::kInt, {-1, -1});
        const int32_t B = count(table.size(0)), budget = (int32_t)integer(a[6], 0, INT32_MAX), first = int32(a[7]), recent = int32(a[8]);
        const at::Tensor &lengths = array_on_device(a[3], device, at::kInt, {B}), &mass = array_on_device(a[4], device, at::kFloat, {B, c.heads, -1}),
                         &next = array_on_device(a[5], device, at::kInt, {B, -1});
        const int64_t slots = next.size(1) * c.slots;
        void *stream = stream_of(a[10]);
        const at::Tensor kept = empty({B, c.heads, budget}, at::kInt, mass), left = empty({B}, at::kInt, mass),
                         new_mass = empty({B, c.heads, slots}, at::kFloat, mass);
        return answer(without_gil(cache_evict, &c, (const int32_t *)ints(table), count(table.size(1)), (const int32_t *)ints(lengths), B,
                                  (const float *)floats(mass), mass.size(2), (const int32_t *)ints(next), count(next.size(1)), budget, first, recent,
                                  ints(kept), ints(left), floats(new_mass), slots, stream), {&kept, &left, &new_mass});
    });
}

// logits, tokens, lengths, prompt_lengths, repetition, presence, frequency, bias_tokens, bias_values, masks, mask_rows (or None), device, stream
PyObject *rules(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<13>(args, n, [](PyObject *const *a) {
        const int64_t device = integer(a[11], 0, INT32_MAX);
        const at::ScalarType type = tensor(a[0]).scalar_type();
        const int32_t code = type_code(tensor(a[0]));
        const at::Tensor &x = rows_on_device(a[0], device, type, 2);
        const int32_t B = count(x.size(0)), V = count(x.size(1));
        const at::Tensor &tokens = array_on_device(a[1], device, at::kInt, {B, -1}), &lengths = array_on_device(a[2], device, at::kInt, {B}),
                         &prompts = array_on_device(a[3], device, at::kInt, {B}), &r = array_on_device(a[4], device, at::kFloat, {B}),
                         &p = array_on_device(a[5], device, at::kFloat, {B}), &f = array_on_device(a[6], device, at::kFloat, {B});
        int32_t K = 0, M = 0;
        const int32_t *bias_tokens = nullptr, *mask_rows = nullptr;
        const float *bias_values = nullptr;
        const uint32_t *masks = nullptr;
        if (a[7] != Py_None || a[8] != Py_None) {
            const at::Tensor &t = array_on_device(a[7], device, at::kInt, {B, -1}), &v = array_on_device(a[8], device, at::kFloat, {B, t.size(1)});
            K = count(t.size(1));
            if (K) { bias_tokens = ints(t); bias_values = floats(v); }
        }
        if (a[9] != Py_None || a[10] != Py_None) {
            const at::Tensor &m = array_on_device(a[9], device, at::kInt, {-1, ((int64_t)V + 31) / 32}), &w = array_on_device(a[10], device, at::kInt, {B});
            M = count(m.size(0));
            if (M) { masks = reinterpret_cast<const uint32_t *>(ints(m)); mask_rows = ints(w); }
        }
        void *stream = stream_of(a[12]);
        const at::Tensor out = empty({B, V}, type, x);
        return answer(without_gil(logit_rules, (const void *)x.data_ptr(), B > 1 ? x.stride(0) : (int64_t)V, B, V, code, (const int32_t *)ints(tokens),
                                  count(tokens.size(1)), (const int32_t *)ints(lengths), (const int32_t *)ints(prompts), (const float *)floats(r),
                                  (const float *)floats(p), (const float *)floats(f), bias_tokens, bias_values, K, masks, M, mask_rows, out.data_ptr(),
                                  (int64_t)V, stream), {&out});
    });
}

// ---- many tokens at once

// qkv, starts, lengths, page_table, frequencies or None, k_cache, v_cache, positions or None, amplitude, interleaved, device, stream
PyObject *append(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<12>(args, n, [](PyObject *const *a) {
        const int64_t device = integer(a[10], 0, INT32_MAX);
        const ann_paged_cache c = cache_of(a[5], a[6], device);
        const at::ScalarType type = tensor(a[5]).scalar_type();
        const at::Tensor &qkv = rows_on_device(a[0], device, type, 3);
        const int32_t T = count(qkv.size(0)), q_heads = count(qkv.size(1)) - 2 * c.heads;
        if (qkv.size(2) != c.d || c.heads > 65536 || q_heads < 1) throw OtherForm();
        const at::Tensor &lengths = array_on_device(a[2], device, at::kInt, {-1});
        const int32_t B = count(lengths.size(0));
        const at::Tensor &starts = array_on_device(a[1], device, at::kInt, {(int64_t)B + 1}), &table = array_on_device(a[3], device, at::kInt, {B, -1});
        const at::Tensor *turns = a[4] == Py_None ? nullptr : &array_on_device(a[4], device, at::kDouble, {-1}),
                         *positions = a[7] == Py_None ? nullptr : &array_on_device(a[7], device, at::kInt, {T});
        if (turns && turns->size(0) > 65536) throw OtherForm();
        const double amplitude = number(a[8]);
        if (!PyBool_Check(a[9])) throw OtherForm();
        void *stream = stream_of(a[11]);
        const at::Tensor q = empty({T, q_heads, c.d}, type, qkv);
        return answer(without_gil(rotate_append, (const void *)qkv.data_ptr(), step_of(qkv, 0), step_of(qkv, 1), T, q_heads, (const int32_t *)ints(starts), B,
                                  (const int32_t *)ints(lengths), (const int32_t *)ints(table), count(table.size(1)),
                                  positions ? (const int32_t *)ints(*positions) : nullptr, turns ? static_cast<const double *>(turns->data_ptr()) : nullptr,
                                  turns ? (int32_t)(2 * turns->size(0)) : 0, (float)amplitude, (int32_t)(a[9] == Py_True), &c, q.data_ptr(), stream), {&q});
    });
}

// q, k_cache, v_cache, page_table, lengths, starts, scale or None, window, max_length or None, device, stream
PyObject *chunk(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<11>(args, n, [](PyObject *const *a) {
        const int64_t device = integer(a[9], 0, INT32_MAX);
        const ann_paged_cache c = cache_of(a[1], a[2], device);
        const at::ScalarType type = tensor(a[1]).scalar_type();
        const at::Tensor &q = rows_on_device(a[0], device, type, 3);
        const int32_t T = count(q.size(0)), q_heads = count(q.size(1));
        if (q.size(2) != c.d) throw OtherForm();
        const at::Tensor &lengths = array_on_device(a[4], device, at::kInt, {-1});
        const int32_t B = count(lengths.size(0));
        const at::Tensor &table = array_on_device(a[3], device, at::kInt, {B, -1}), &starts = array_on_device(a[5], device, at::kInt, {(int64_t)B + 1});
        const double scale = a[6] == Py_None ? 1.0 / std::sqrt((double)c.d) : number(a[6]);
        const int32_t window = int32(a[7]), width = count(table.size(1)),
                      most = a[8] == Py_None ? (int32_t)std::min<int64_t>(INT32_MAX, (int64_t)width * c.slots) : int32(a[8]);
        void *stream = stream_of(a[10]);
        const at::Tensor out = empty({T, q_heads, c.d}, type, q), lse = empty({T, q_heads}, at::kFloat, q);
        return answer(without_gil(chunk_attention, (const void *)q.data_ptr(), step_of(q, 0), step_of(q, 1), T, q_heads, (const int32_t *)ints(starts), B, &c,
                                  (const int32_t *)ints(table), width, (const int32_t *)ints(lengths), most, (float)scale, window, out.data_ptr(), floats(lse),
                                  stream), {&out, &lse});
    });
}

// q, k_cache, v_cache, page_table, lengths, group_starts, shared, max_shared or None, max_own or None, scale or None, device, stream
PyObject *shared(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return usual<12>(args, n, [](PyObject *const *a) {
        const int64_t device = integer(a[10], 0, INT32_MAX);
        const ann_paged_cache c = cache_of(a[1], a[2], device);
        const at::ScalarType type = tensor(a[1]).scalar_type();
        const at::Tensor &q = rows_on_device(a[0], device, type, 3);
        const int32_t B = count(q.size(0)), q_heads = count(q.size(1));
        if (q.size(2) != c.d) throw OtherForm();
        const at::Tensor &table = array_on_device(a[3], device, at::kInt, {B, -1}), &lengths = array_on_device(a[4], device, at::kInt, {B}),
                         &common = array_on_device(a[6], device, at::kInt, {-1});
        const int32_t groups = count(common.size(0)), width = count(table.size(1)), all = (int32_t)std::min<int64_t>(INT32_MAX, (int64_t)width * c.slots);
        const at::Tensor &starts = array_on_device(a[5], device, at::kInt, {(int64_t)groups + 1});
        const int32_t most_shared = a[7] == Py_None ? all : int32(a[7]), most_own = a[8] == Py_None ? all : int32(a[8]);
        const double scale = a[9] == Py_None ? 1.0 / std::sqrt((double)c.d) : number(a[9]);
        void *stream = stream_of(a[11]);
        const at::Tensor out = empty({B, q_heads, c.d}, type, q), lse = empty({B, q_heads}, at::kFloat, q);
        return answer(without_gil(shared_attention, (const void *)q.data_ptr(), step_of(q, 0), step_of(q, 1), B, q_heads, &c, (const int32_t *)ints(table), width,
                                  (const int32_t *)ints(lengths), (const int32_t *)ints(starts), (const int32_t *)ints(common), groups, most_shared, most_own,
                                  (float)scale, out.data_ptr(), floats(lse), stream), {&out, &lse});
    });
}

// addresses of the three, in the order of their declarations above
PyObject *bind_many(PyObject *, PyObject *const *args, Py_ssize_t n) {
    void *p[3];
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "bind_many takes 3 addresses");
        return nullptr;
    }
    for (int i = 0; i < 3; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    rotate_append = reinterpret_cast<decltype(rotate_append)>(p[0]);
    chunk_attention = reinterpret_cast<decltype(chunk_attention)>(p[1]);
    shared_attention = reinterpret_cast<decltype(shared_attention)>(p[2]);
    Py_RETURN_NONE;
}

// addresses of the four, in the order of their declarations above
PyObject *bind_decode(PyObject *, PyObject *const *args, Py_ssize_t n) {
    void *p[4];
    if (n != 4) {
        PyErr_SetString(PyExc_TypeError, "bind_decode takes 4 addresses");
        return nullptr;
    }
    for (int i = 0; i < 4; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    qk_norm_rotate = reinterpret_cast<decltype(qk_norm_rotate)>(p[0]);
    paged_attention = reinterpret_cast<decltype(paged_attention)>(p[1]);
    cache_evict = reinterpret_cast<decltype(cache_evict)>(p[2]);
    logit_rules = reinterpret_cast<decltype(logit_rules)>(p[3]);
    Py_RETURN_NONE;
}

// addresses of the entry points, in the order of their declarations above
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n) {
    void *p[7];
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "bind takes 7 addresses");
        return nullptr;
    }
    for (int i = 0; i < 7; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    flat_search = reinterpret_cast<decltype(flat_search)>(p[0]);
    flat_search_after = reinterpret_cast<decltype(flat_search_after)>(p[1]);
    graph_search = reinterpret_cast<decltype(graph_search)>(p[2]);
    graph_search_entries = reinterpret_cast<decltype(graph_search_entries)>(p[3]);
    graph_search_nonstall = reinterpret_cast<decltype(graph_search_nonstall)>(p[4]);
    gather_ids = reinterpret_cast<decltype(gather_ids)>(p[5]);
    priority_order = reinterpret_cast<decltype(priority_order)>(p[6]);
    Py_RETURN_NONE;
}

#define ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(bind), ENTRY(flat), ENTRY(graph), ENTRY(graph_entries), ENTRY(nonstall), ENTRY(gather), ENTRY(order),
                         ENTRY(bind_decode), ENTRY(rotate), ENTRY(attend), ENTRY(evict), ENTRY(rules),
                         ENTRY(bind_many), ENTRY(append), ENTRY(chunk), ENTRY(shared), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// (asks nothing of torch's objects: the binding looks at built_for before it binds)
PyMODINIT_FUNC PyInit__marshal() {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", ANN_BUILT_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
