// Argument marshalling of the hot calls, from torch tensors to libssd's C entry points.
//
// A decoding step is five calls of a few microseconds of GPU work each; marshalled in Python
// through ctypes they took 52 us of host time, more than the GPU needs for a small batch.  Each
// function here takes what the binding function of the same name takes, with the result buffers
// given and no launch options, and answers the C call's status -- or None, having done nothing,
// for anything that is not plainly fine (another type, a host tensor, a missing buffer, a shape
// the binding refuses): the binding then goes its general way and raises what it always raised.
#include <torch/csrc/autograd/python_variable.h>
#include <c10/cuda/CUDAStream.h>

#include <climits>

#include "../../include/ssd.h"

namespace {

struct Unhandled {};

const at::Tensor &tensor(PyObject *o) {
    if (!o || !THPVariable_Check(o)) throw Unhandled{};
    return THPVariable_Unpack(o);
}
void *address(const at::Tensor &t) {
    if (!t.is_cuda()) throw Unhandled{};
    return t.data_ptr();
}
void *address(PyObject *o) { return address(tensor(o)); }
void *address_or_null(PyObject *o) { return !o || o == Py_None ? nullptr : address(o); }

// the buffer `key` of the dict of results; absent or None where the call allows it
PyObject *entry(PyObject *out, PyObject *key) {
    PyObject *v = PyDict_GetItemWithError(out, key);
    if (!v && PyErr_Occurred()) { PyErr_Clear(); throw Unhandled{}; }
    return v;
}

struct Rows {
    void *p;
    int64_t n, ld, V;
    ssd_dtype dtype;
};
Rows rows(PyObject *o, PyObject *V) {
    const at::Tensor &t = tensor(o);
    if (t.dim() != 2 || t.stride(1) != 1) throw Unhandled{};
    Rows r;
    r.n = t.size(0);
    r.ld = r.n > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1));
    if (t.scalar_type() == at::kFloat) r.dtype = SSD_F32;
    else if (t.scalar_type() == at::kBFloat16) r.dtype = SSD_BF16;
    else throw Unhandled{};
    r.V = t.size(1);
    if (V != Py_None) {
        if (!PyLong_Check(V)) throw Unhandled{};
        int over = 0;
        r.V = PyLong_AsLongLongAndOverflow(V, &over);
        if (over) throw Unhandled{};
    }
    if (r.V < INT_MIN || r.V > INT_MAX) throw Unhandled{};
    r.p = address(t);
    return r;
}
const at::Tensor &typed(PyObject *o, at::ScalarType type) {
    const at::Tensor &t = tensor(o);
    if (t.scalar_type() != type || t.dim() < 1) throw Unhandled{};
    return t;
}
int32_t utterances(const at::Tensor &off) {
    const int64_t B = off.size(0) - 1;
    if (B < 0 || B > INT_MAX) throw Unhandled{};
    return (int32_t)B;
}
int32_t int32(PyObject *o) {
    if (!PyLong_Check(o)) throw Unhandled{};
    int over = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &over);
    if (over || v < INT_MIN || v > INT_MAX) throw Unhandled{};
    return (int32_t)v;
}
float number(PyObject *o) {
    if (PyFloat_Check(o)) return (float)PyFloat_AS_DOUBLE(o);
    if (!PyLong_Check(o)) throw Unhandled{};
    const double v = PyLong_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); throw Unhandled{}; }
    return (float)v;
}
void *stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

PyObject *K_workspace, *K_frame_entropy, *K_frame_argmax, *K_frame_lse, *K_frame_logprob,
    *K_draft_tokens, *K_draft_frames, *K_draft_len, *K_draft_full_len, *K_utt_max_entropy,
    *K_utt_status, *K_gate_accept, *K_max_entropy, *K_token_logp, *K_row_lse, *K_accepted_len,
    *K_all_accepted, *K_rows_read, *K_final_tokens, *K_final_len, *K_is_final, *K_ar_count, *K_ar_utt,
    *K_ar_resume, *K_next_token, *K_next_logp, *K_row_status, *K_out, *K_lse, *K_path, *K_path_len,
    *K_on_path, *K_new_len, *K_kept, *K_weight;

struct Scratch {
    void *p;
    size_t bytes;
};
Scratch scratch(PyObject *o, bool needed) {
    if (!o || o == Py_None) {
        if (needed) throw Unhandled{};
        return {nullptr, 0};
    }
    const at::Tensor &t = tensor(o);
    return {address(t), (size_t)t.numel()};
}

// Runs `body`, which marshals under the interpreter lock and returns what to call without it.
template <typename Body> PyObject *guarded(Py_ssize_t have, Py_ssize_t want, Body body) {
    try {
        if (have != want) throw Unhandled{};
        auto call = body();
        int32_t rc;
        Py_BEGIN_ALLOW_THREADS
        rc = call();
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (...) {
        // only marshalling throws (the entry points are C): nothing has been enqueued
        Py_RETURN_NONE;
    }
}

// a subclass may answer for its items itself
void need_dict(PyObject *o) { if (!PyDict_CheckExact(o)) throw Unhandled{}; }

// ctc_draft(logits, frame_off, blank_id, max_draft_len, V, out)
PyObject *ctc_draft(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 6, [&] {
        const Rows x = rows(a[0], a[4]);
        const at::Tensor &off = typed(a[1], at::kLong);
        const int32_t B = utterances(off), blank = int32(a[2]), cap = int32(a[3]);
        PyObject *o = a[5];
        need_dict(o);
        const Scratch ws = scratch(entry(o, K_workspace), false);
        auto *fo = (const int64_t *)address(off);
        auto *fe = (float *)address(entry(o, K_frame_entropy));
        auto *fa = (int32_t *)address(entry(o, K_frame_argmax));
        auto *fl = (float *)address_or_null(entry(o, K_frame_lse));
        auto *lp = (float *)address_or_null(entry(o, K_frame_logprob));
        auto *dt = (int32_t *)address(entry(o, K_draft_tokens));
        auto *df = (int32_t *)address_or_null(entry(o, K_draft_frames));
        auto *dl = (int32_t *)address(entry(o, K_draft_len));
        auto *du = (int32_t *)address(entry(o, K_draft_full_len));
        auto *um = (float *)address(entry(o, K_utt_max_entropy));
        auto *us = (uint32_t *)address(entry(o, K_utt_status));
        void *st = stream();
        return [=] {
            return ssd_ctc_draft(x.p, x.dtype, (int32_t)x.V, x.ld, fo, B, x.n, blank, cap, fe, fa, fl,
                                 lp, dt, df, dl, du, um, us, ws.p, ws.bytes, st, nullptr);
        };
    });
}

// gate_from_maxima(utt_max_entropy, utt_status, tau_ctc, out)
PyObject *gate_from_maxima(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 4, [&] {
        const at::Tensor &um = typed(a[0], at::kFloat), &us = typed(a[1], at::kInt);
        const int64_t B64 = um.size(0);
        if (B64 > INT_MAX) throw Unhandled{};
        const int32_t B = (int32_t)B64;
        const float tau = number(a[2]);
        need_dict(a[3]);
        auto *ga = (uint8_t *)address(entry(a[3], K_gate_accept));
        auto *me = (float *)address(entry(a[3], K_max_entropy));
        auto *ump = (const float *)address(um);
        auto *usp = (const uint32_t *)address(us);
        void *st = stream();
        return [=] {
            return ssd_entropy_gate(nullptr, nullptr, B, 0, tau, ga, me, nullptr, ump, usp, st);
        };
    });
}

// what ssd_verify and ssd_verify_early_exit have in common
struct Verify {
    Rows x;
    const int64_t *off;
    const int32_t *ids;
    int32_t B;
    float tau;
    const uint8_t *skip;
    float *logp, *lse;
    int32_t *len;
    uint8_t *all;
    uint32_t *status;
    Scratch ws;
    void *st;
};
// (logits, tok_off, draft_ids, tau_slm, skip, V, out)
Verify verify_args(PyObject *const *a) {
    Verify v;
    v.x = rows(a[0], a[5]);
    const at::Tensor &off = typed(a[1], at::kLong), &ids = typed(a[2], at::kInt);
    v.B = utterances(off);
    v.tau = number(a[3]);
    v.skip = a[4] == Py_None ? nullptr : (const uint8_t *)address(typed(a[4], at::kByte));
    PyObject *o = a[6];
    need_dict(o);
    v.off = (const int64_t *)address(off);
    v.ids = (const int32_t *)address(ids);
    v.logp = (float *)address(entry(o, K_token_logp));
    v.lse = (float *)address_or_null(entry(o, K_row_lse));
    v.len = (int32_t *)address(entry(o, K_accepted_len));
    v.all = (uint8_t *)address(entry(o, K_all_accepted));
    v.status = (uint32_t *)address(entry(o, K_utt_status));
    v.ws = scratch(entry(o, K_workspace), true);
    v.st = stream();
    return v;
}
PyObject *verify(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 7, [&] {
        const Verify v = verify_args(a);
        return [=] {
            return ssd_verify(v.x.p, v.x.dtype, (int32_t)v.x.V, v.x.ld, v.off, v.ids, v.B, v.x.n, v.tau,
                              v.skip, v.logp, v.lse, v.len, v.all, v.status, v.ws.p, v.ws.bytes, v.st,
                              nullptr);
        };
    });
}
PyObject *verify_early_exit(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 7, [&] {
        const Verify v = verify_args(a);
        auto *rr = (int32_t *)address_or_null(entry(a[6], K_rows_read));
        return [=] {
            return ssd_verify_early_exit(v.x.p, v.x.dtype, (int32_t)v.x.V, v.x.ld, v.off, v.ids, v.B,
                                         v.x.n, v.tau, v.skip, v.logp, v.lse, v.len, v.all, v.status,
                                         rr, v.ws.p, v.ws.bytes, v.st, nullptr);
        };
    });
}

// verify_shard(logits, col0, tok_off, draft_ids, skip, V_local, stats, workspace)
PyObject *verify_shard(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        const Rows x = rows(a[0], a[5]);
        if (!PyLong_Check(a[1])) throw Unhandled{};
        int over = 0;
        const int64_t col0 = PyLong_AsLongLongAndOverflow(a[1], &over);
        if (over) throw Unhandled{};
        const at::Tensor &off = typed(a[2], at::kLong), &ids = typed(a[3], at::kInt);
        const int32_t B = utterances(off);
        auto *skip = a[4] == Py_None ? nullptr : (const uint8_t *)address(typed(a[4], at::kByte));
        auto *offp = (const int64_t *)address(off);
        auto *idsp = (const int32_t *)address(ids);
        auto *stats = (float *)address(a[6]);
        const Scratch ws = scratch(a[7], true);
        void *st = stream();
        return [=] {
            return ssd_verify_shard(x.p, x.dtype, (int32_t)x.V, x.ld, col0, offp, idsp, B, x.n, skip,
                                    stats, ws.p, ws.bytes, st, nullptr);
        };
    });
}

// verify_combine(stats_all, V_total, tok_off, draft_ids, tau_slm, skip, out)
PyObject *verify_combine(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 7, [&] {
        const at::Tensor &s = typed(a[0], at::kFloat);
        if (s.dim() != 3 || s.size(2) != 3 || !s.is_contiguous() || s.size(0) > INT_MAX) throw Unhandled{};
        const int32_t R = (int32_t)s.size(0);
        const int64_t M = s.size(1);
        if (!PyLong_Check(a[1])) throw Unhandled{};
        int over = 0;
        const int64_t V = PyLong_AsLongLongAndOverflow(a[1], &over);
        if (over) throw Unhandled{};
        const at::Tensor &off = typed(a[2], at::kLong), &ids = typed(a[3], at::kInt);
        const int32_t B = utterances(off);
        const float tau = number(a[4]);
        auto *skip = (const uint8_t *)address_or_null(a[5]);
        PyObject *o = a[6];
        need_dict(o);
        auto *sp = (const float *)address(s);
        auto *offp = (const int64_t *)address(off);
        auto *idsp = (const int32_t *)address(ids);
        auto *logp = (float *)address(entry(o, K_token_logp));
        auto *lse = (float *)address_or_null(entry(o, K_row_lse));
        auto *len = (int32_t *)address(entry(o, K_accepted_len));
        auto *all = (uint8_t *)address(entry(o, K_all_accepted));
        auto *status = (uint32_t *)address(entry(o, K_utt_status));
        void *st = stream();
        return [=] {
            return ssd_verify_combine(sp, R, V, offp, idsp, B, M, tau, skip, logp, lse, len, all, status, st);
        };
    });
}

// assemble(tokens, tok_off, gate_accept, accepted_len, all_accepted, out)
PyObject *assemble(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 6, [&] {
        const at::Tensor &tok = typed(a[0], at::kInt), &off = typed(a[1], at::kLong);
        const at::Tensor &ga = typed(a[2], at::kByte), &len = typed(a[3], at::kInt),
                         &all = typed(a[4], at::kByte);
        const int32_t B = utterances(off);
        const int64_t M = tok.size(0);
        PyObject *o = a[5];
        need_dict(o);
        auto *tokp = (const int32_t *)address(tok);
        auto *offp = (const int64_t *)address(off);
        auto *gap = (const uint8_t *)address(ga);
        auto *lenp = (const int32_t *)address(len);
        auto *allp = (const uint8_t *)address(all);
        auto *ft = (int32_t *)address(entry(o, K_final_tokens));
        auto *fl = (int32_t *)address(entry(o, K_final_len));
        auto *fin = (uint8_t *)address(entry(o, K_is_final));
        auto *ac = (int32_t *)address(entry(o, K_ar_count));
        auto *au = (int32_t *)address(entry(o, K_ar_utt));
        auto *ar = (int32_t *)address(entry(o, K_ar_resume));
        void *st = stream();
        return [=] {
            return ssd_assemble(tokp, offp, B, M, gap, lenp, allp, ft, fl, fin, ac, au, ar, st);
        };
    });
}

// greedy_step(logits, V, out)
PyObject *greedy_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 3, [&] {
        const Rows x = rows(a[0], a[1]);
        PyObject *o = a[2];
        need_dict(o);
        auto *nt = (int32_t *)address(entry(o, K_next_token));
        auto *lp = (float *)address_or_null(entry(o, K_next_logp));
        auto *lse = (float *)address_or_null(entry(o, K_row_lse));
        auto *rs = (uint32_t *)address_or_null(entry(o, K_row_status));
        const Scratch ws = scratch(entry(o, K_workspace), true);
        void *st = stream();
        return [=] {
            return ssd_greedy_step(x.p, x.dtype, (int32_t)x.V, x.ld, x.n, nt, lp, lse, rs, ws.p, ws.bytes,
                                   st, nullptr);
        };
    });
}

// ---- draft trees and their cache ----------------------------------------------------------------
// the library launches on the current device
void *here(const at::Tensor &t) {
    void *p = address(t);
    if (t.get_device() != c10::cuda::current_device()) throw Unhandled{};
    return p;
}
Scratch scratch_here(PyObject *o) {
    const Scratch ws = scratch(o, true);
    here(tensor(o));
    return ws;
}
ssd_dtype kv_type(const at::Tensor &t) {
    if (t.scalar_type() == at::kBFloat16) return SSD_BF16;
    if (t.scalar_type() == at::kHalf) return SSD_F16;
    throw Unhandled{};
}
// [rows, heads, head_dim] with contiguous heads
struct HeadsArg {
    ssd_heads h;
    int64_t rows, D;
    ssd_dtype dtype;
};
HeadsArg heads(PyObject *o) {
    const at::Tensor &t = tensor(o);
    if (t.dim() != 3 || (t.size(2) > 1 && t.stride(2) != 1) || t.size(1) > INT_MAX) throw Unhandled{};
    HeadsArg a;
    a.dtype = kv_type(t);
    a.h.data = here(t);
    a.h.row_stride = t.stride(0);
    a.h.head_stride = t.stride(1);
    a.h.heads = (int32_t)t.size(1);
    a.rows = t.size(0);
    a.D = t.size(2);
    return a;
}
// k_cache, v_cache (or null), page_table, cache_len of B utterances
ssd_kv_cache kv_cache(PyObject *ko, PyObject *vo, PyObject *table_o, PyObject *len_o, int32_t B) {
    const at::Tensor &k = tensor(ko), &table = typed(table_o, at::kInt), &len = typed(len_o, at::kInt);
    if (k.dim() != 4 || (k.size(3) > 1 && k.stride(3) != 1)) throw Unhandled{};
    ssd_kv_cache c;
    c.dtype = kv_type(k);
    c.k = here(k);
    c.v = nullptr;
    if (vo) {
        const at::Tensor &v = tensor(vo);
        if (v.scalar_type() != k.scalar_type() || v.dim() != 4) throw Unhandled{};
        for (int i = 0; i < 4; ++i)
            if (v.size(i) != k.size(i) || (k.size(i) > 1 && v.stride(i) != k.stride(i))) throw Unhandled{};
        c.v = here(v);
    }
    for (int i = 0; i < 4; ++i)
        if (k.size(i) > INT_MAX) throw Unhandled{};
    c.page_stride = k.stride(0); c.slot_stride = k.stride(1); c.head_stride = k.stride(2);
    c.pages = (int32_t)k.size(0); c.page_size = (int32_t)k.size(1); c.heads = (int32_t)k.size(2); c.head_dim = (int32_t)k.size(3);
    if (table.dim() != 2 || table.size(0) != B || (table.size(1) > 1 && table.stride(1) != 1) || table.size(1) > INT_MAX) throw Unhandled{};
    if (len.dim() != 1 || len.size(0) != B || (B > 1 && len.stride(0) != 1)) throw Unhandled{};
    c.max_pages = (int32_t)table.size(1);
    c.page_table = (const int32_t *)here(table);
    c.table_stride = B > 1 ? table.stride(0) : std::max(table.stride(0), table.size(1));
    c.len = (const int32_t *)here(len);
    return c;
}
// a contiguous array of n values of a type, or null for None
template <typename T> T *flat(PyObject *o, at::ScalarType type, int64_t n, bool nullable) {
    if (nullable && (!o || o == Py_None)) return nullptr;
    const at::Tensor &t = typed(o, type);
    if (t.dim() != 1 || t.size(0) != n || !t.is_contiguous()) throw Unhandled{};
    return (T *)here(t);
}
const int64_t *offsets(PyObject *o, int32_t &B) {
    const at::Tensor &t = typed(o, at::kLong);
    if (t.dim() != 1 || !t.is_contiguous()) throw Unhandled{};
    B = utterances(t);
    return (const int64_t *)here(t);
}
// [B, slots] of weights
struct WeightArg {
    float *p;
    int64_t stride;
    int32_t cols;
};
WeightArg weights(PyObject *o, int32_t B, bool nullable) {
    if (nullable && (!o || o == Py_None)) return {nullptr, 0, 0};
    const at::Tensor &t = typed(o, at::kFloat);
    if (t.dim() != 2 || t.size(0) != B || (t.size(1) > 1 && t.stride(1) != 1) || t.size(1) > INT_MAX) throw Unhandled{};
    return {(float *)here(t), B > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1)), (int32_t)t.size(1)};
}
// a contiguous float32 [rows, heads], or null
float *per_head(PyObject *o, int64_t rows, int64_t n, bool nullable) {
    if (nullable && (!o || o == Py_None)) return nullptr;
    const at::Tensor &t = typed(o, at::kFloat);
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != n || !t.is_contiguous()) throw Unhandled{};
    return (float *)here(t);
}

// tree_attention(q, tree_k, tree_v, k_cache, v_cache, page_table, cache_len, tok_off, max_nodes, parent, scale, cap, out)
PyObject *tree_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 13, [&] {
        int32_t B;
        const int64_t *off = offsets(a[7], B);
        const HeadsArg q = heads(a[0]), tk = heads(a[1]), tv = heads(a[2]);
        const ssd_kv_cache c = kv_cache(a[3], a[4], a[5], a[6], B);
        const int32_t max_nodes = int32(a[8]);
        auto *parent = flat<const int32_t>(a[9], at::kInt, q.rows, true);
        const float scale = number(a[10]), cap = number(a[11]);
        need_dict(a[12]);
        const HeadsArg o = heads(entry(a[12], K_out));
        for (const HeadsArg *x : {&tk, &tv, &o})
            if (x->dtype != q.dtype || x->rows != q.rows || x->D != q.D) throw Unhandled{};
        if (c.dtype != q.dtype || c.head_dim != q.D || o.h.heads != q.h.heads) throw Unhandled{};
        float *lse = per_head(entry(a[12], K_lse), q.rows, q.h.heads, true);
        const Scratch ws = scratch_here(entry(a[12], K_workspace));
        auto *us = flat<uint32_t>(entry(a[12], K_utt_status), at::kInt, B, false);
        void *st = stream();
        return [=] {
            return ssd_tree_attention(&q.h, &tk.h, &tv.h, &c, off, parent, B, q.rows, max_nodes, scale, cap, &o.h, lse, us,
                                      ws.p, ws.bytes, st);
        };
    });
}

// verify_tree(logits, tok_off, draft_ids, parent, tau_slm, skip, V, out)
PyObject *verify_tree(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        const Rows x = rows(a[0], a[6]);
        here(tensor(a[0]));
        int32_t B;
        const int64_t *off = offsets(a[1], B);
        auto *ids = flat<const int32_t>(a[2], at::kInt, x.n, false);
        auto *parent = flat<const int32_t>(a[3], at::kInt, x.n, true);
        const float tau = number(a[4]);
        auto *skip = flat<const uint8_t>(a[5], at::kByte, B, true);
        PyObject *o = a[7];
        need_dict(o);
        auto *logp = flat<float>(entry(o, K_token_logp), at::kFloat, x.n, false);
        auto *lse = flat<float>(entry(o, K_row_lse), at::kFloat, x.n, true);
        auto *path = flat<int32_t>(entry(o, K_path), at::kInt, x.n, false);
        auto *len = flat<int32_t>(entry(o, K_path_len), at::kInt, B, false);
        auto *on = flat<uint8_t>(entry(o, K_on_path), at::kByte, x.n, false);
        auto *us = flat<uint32_t>(entry(o, K_utt_status), at::kInt, B, false);
        const Scratch ws = scratch_here(entry(o, K_workspace));
        void *st = stream();
        return [=] {
            return ssd_verify_tree(x.p, x.dtype, (int32_t)x.V, x.ld, off, ids, parent, B, x.n, tau, skip, logp, lse, path, len, on, us,
                                   ws.p, ws.bytes, st, nullptr);
        };
    });
}

// cache_append(tree_k, tree_v, tok_off, path, path_len, k_cache, v_cache, page_table, cache_len, weight, out)
PyObject *cache_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 11, [&] {
        int32_t B;
        const int64_t *off = offsets(a[2], B);
        const HeadsArg tk = heads(a[0]), tv = heads(a[1]);
        auto *path = flat<const int32_t>(a[3], at::kInt, tk.rows, true);
        auto *len = flat<const int32_t>(a[4], at::kInt, B, false);
        const ssd_kv_cache c = kv_cache(a[5], a[6], a[7], a[8], B);
        if (tv.rows != tk.rows || tk.D != c.head_dim || tv.D != c.head_dim || tk.dtype != c.dtype || tv.dtype != c.dtype) throw Unhandled{};
        const WeightArg w = weights(a[9], B, true);
        need_dict(a[10]);
        auto *nl = flat<int32_t>(entry(a[10], K_new_len), at::kInt, B, false);
        auto *us = flat<uint32_t>(entry(a[10], K_utt_status), at::kInt, B, false);
        void *st = stream();
        return [=] {
            return ssd_cache_append(&tk.h, &tv.h, &c, off, path, len, B, tk.rows, w.p, w.stride, w.cols, nl, us, st);
        };
    });
}

// cache_weights(q, lse, k_cache, page_table, cache_len, tok_off, max_nodes, weight, use, scale, cap, out)
PyObject *cache_weights(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 12, [&] {
        int32_t B;
        const int64_t *off = offsets(a[5], B);
        const HeadsArg q = heads(a[0]);
        const float *lse = per_head(a[1], q.rows, q.h.heads, false);
        const ssd_kv_cache c = kv_cache(a[2], nullptr, a[3], a[4], B);
        if (c.dtype != q.dtype || c.head_dim != q.D) throw Unhandled{};
        const int32_t max_nodes = int32(a[6]);
        const WeightArg w = weights(a[7], B, false);
        auto *use = flat<const uint8_t>(a[8], at::kByte, q.rows, true);
        const float scale = number(a[9]), cap = number(a[10]);
        need_dict(a[11]);
        auto *us = flat<uint32_t>(entry(a[11], K_utt_status), at::kInt, B, false);
        void *st = stream();
        return [=] {
            return ssd_cache_weights(&q.h, lse, &c, off, B, q.rows, max_nodes, scale, cap, use, w.p, w.stride, w.cols, us, st);
        };
    });
}

// cache_evict(k_cache, v_cache, page_table, cache_len, weight, budget, sink, recent, out)
PyObject *cache_evict(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&] {
        const at::Tensor &len = typed(a[3], at::kInt);
        if (len.dim() != 1 || len.size(0) > INT_MAX) throw Unhandled{};
        const int32_t B = (int32_t)len.size(0);
        const ssd_kv_cache c = kv_cache(a[0], a[1], a[2], a[3], B);
        const WeightArg w = weights(a[4], B, false);
        const int32_t budget = int32(a[5]), sink = int32(a[6]), recent = int32(a[7]);
        need_dict(a[8]);
        const at::Tensor &kept = typed(entry(a[8], K_kept), at::kInt);
        if (kept.dim() != 2 || kept.size(0) != B || kept.size(1) != budget || !kept.is_contiguous()) throw Unhandled{};
        auto *kp = (int32_t *)here(kept);
        const WeightArg wo = weights(entry(a[8], K_weight), B, true);
        if (wo.p && wo.cols < budget) throw Unhandled{};
        auto *nl = flat<int32_t>(entry(a[8], K_new_len), at::kInt, B, false);
        auto *us = flat<uint32_t>(entry(a[8], K_utt_status), at::kInt, B, false);
        void *st = stream();
        return [=] {
            return ssd_cache_evict(&c, w.p, w.stride, w.cols, B, budget, sink, recent, kp, wo.p, wo.stride, nl, us, st);
        };
    });
}

#define SSD_METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SSD_METHOD(ctc_draft), SSD_METHOD(gate_from_maxima), SSD_METHOD(verify),
                         SSD_METHOD(verify_early_exit), SSD_METHOD(verify_shard),
                         SSD_METHOD(verify_combine), SSD_METHOD(assemble), SSD_METHOD(greedy_step),
                         SSD_METHOD(tree_attention), SSD_METHOD(verify_tree), SSD_METHOD(cache_append),
                         SSD_METHOD(cache_weights), SSD_METHOD(cache_evict),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ssd_call", nullptr, -1, methods};
// torch's C++ types change from release to release: the binding compares before the first call
const char kBuiltFor[] = "_ssd_call for " SSD_BUILT_FOR;

}  // namespace

PyMODINIT_FUNC PyInit__ssd_call() {
#define SSD_KEY(k) if (!(K_##k = PyUnicode_InternFromString(#k))) return nullptr;
    SSD_KEY(workspace) SSD_KEY(frame_entropy) SSD_KEY(frame_argmax) SSD_KEY(frame_lse)
    SSD_KEY(frame_logprob) SSD_KEY(draft_tokens) SSD_KEY(draft_frames) SSD_KEY(draft_len)
    SSD_KEY(draft_full_len) SSD_KEY(utt_max_entropy) SSD_KEY(utt_status) SSD_KEY(gate_accept)
    SSD_KEY(max_entropy) SSD_KEY(token_logp) SSD_KEY(row_lse) SSD_KEY(accepted_len)
    SSD_KEY(all_accepted) SSD_KEY(rows_read) SSD_KEY(final_tokens) SSD_KEY(final_len)
    SSD_KEY(is_final) SSD_KEY(ar_count) SSD_KEY(ar_utt) SSD_KEY(ar_resume) SSD_KEY(next_token)
    SSD_KEY(next_logp) SSD_KEY(row_status) SSD_KEY(out) SSD_KEY(lse) SSD_KEY(path)
    SSD_KEY(path_len) SSD_KEY(on_path) SSD_KEY(new_len) SSD_KEY(kept) SSD_KEY(weight)
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", kBuiltFor) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
