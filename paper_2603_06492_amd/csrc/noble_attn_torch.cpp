// The attention side's calls on torch tensors, in native code: argument checks, buffers and the library call of the
// functions of attention.py.  As in noble_torch.cpp, each serves the well-formed call on ordinary tensors and returns
// None for every other one, which the Python code then checks and runs; a status other than NOBLE_OK comes back as an
// int.  The library's entry points come in as addresses (init).
#include "noble_torch_call.hpp"

namespace {

decltype(&noble_qk_rope_fwd) p_rope_fwd;
decltype(&noble_qk_rope_bwd) p_rope_bwd;
decltype(&noble_qk_rope_scratch_size) p_rope_size;
decltype(&noble_kv_append) p_append;
decltype(&noble_attn_fwd) p_attn_fwd;
decltype(&noble_attn_bwd) p_attn_bwd;
decltype(&noble_attn_bwd_scratch_size) p_bwd_size;
decltype(&noble_attn_paged) p_paged;
decltype(&noble_attn_paged_scratch_size) p_paged_size;

// (qkv, q_weight, k_weight, cos, sin, positions, heads, kv_heads, eps, interleaved) of the calls over Q/K/V rows.
struct RopeIn {
    noble_rope_desc d{};
    const void* x = nullptr;
    float *wq = nullptr, *wk = nullptr, *cos = nullptr, *sin = nullptr;
    int32_t* positions = nullptr;
    RopeIn(Call& c, PyObject* const* a) {
        const at::Tensor* t = c.first(a[0]);
        d.heads = (int32_t)c.integer(a[6], 0, 4096);
        d.kv_heads = (int32_t)c.integer(a[7], 0, 4096);
        const int64_t n = d.heads + 2 * (int64_t)d.kv_heads;
        if (!c.ok || t->dim() != 2 || n < 1 || t->size(1) % n || (t->size(1) > 1 && t->stride(1) != 1)) {
            c.ok = false;
            return;
        }
        const int64_t D = t->size(1) / n;
        x = t->data_ptr();
        d.T = t->size(0);
        d.x_row = d.T > 1 ? t->stride(0) : t->size(1);
        d.head_dim = (int32_t)std::min<int64_t>(D, INT32_MAX);
        d.dtype = c.dtype;
        d.eps = c.number(a[8]);
        d.interleaved = c.truth(a[9]);
        if ((a[1] == Py_None) != (a[2] == Py_None) || (a[3] == Py_None) != (a[4] == Py_None)) c.ok = false;
        wq = c.floats(a[1], {D});
        wk = c.floats(a[2], {D});
        if (a[3] != Py_None) {
            const at::Tensor* tc = c.tensor(a[3]);
            if (!c.ok || tc->dim() != 2 || tc->size(1) > 4096) {
                c.ok = false;
                return;
            }
            d.table_rows = tc->size(0);
            d.rot = (int32_t)(2 * tc->size(1));
            cos = c.floats(a[3], {tc->size(0), tc->size(1)});
            sin = c.floats(a[4], {tc->size(0), tc->size(1)});
        }
        positions = c.ints(a[5], {d.T});
    }
};

// rope_fwd(10 of RopeIn, q, k) -> (q, k).
PyObject* rope_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    Call c;
    const RopeIn in(c, a);
    if (!c.ok) Py_RETURN_NONE;
    const Output q(c, a[10], {in.d.T, in.d.heads, in.d.head_dim}, c.sd), k(c, a[11], {in.d.T, in.d.kv_heads, in.d.head_dim}, c.sd);
    void *pq = q.dense(c), *pk = k.dense(c);
    if (!c.ok) Py_RETURN_NONE;
    noble_status st;
    {
        NoGil nogil;
        const c10::DeviceGuard guard(c.dev);
        st = p_rope_fwd(&in.d, in.x, in.wq, in.wk, in.cos, in.sin, in.positions, pq, pk, c.stream());
    }
    return st == NOBLE_OK ? tuple({&q.t, &k.t}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// rope_bwd(dq, dk, 10 of RopeIn, dqkv) -> (dq_weight, dk_weight), into a given dqkv with qkv's row stride.
PyObject* rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 13 || a[12] == Py_None) Py_RETURN_NONE;
    Call c;
    const RopeIn in(c, a + 2);
    if (!c.ok || in.d.T == 0) Py_RETURN_NONE;
    const int64_t T = in.d.T, D = in.d.head_dim;
    const void *dq = c.dense(a[0], c.sd, {T, in.d.heads, D}), *dk = c.dense(a[1], c.sd, {T, in.d.kv_heads, D});
    const at::Tensor *g = c.tensor(a[12]), *x = c.tensor(a[2]);
    if (!c.ok || a[0] == Py_None || a[1] == Py_None || g->scalar_type() != c.sd || g->device() != c.dev ||
        !g->sizes().equals(x->sizes()) || !g->strides().equals(x->strides()))
        Py_RETURN_NONE;
    size_t bytes = 0;
    if (p_rope_size(&in.d, &bytes) != NOBLE_OK) Py_RETURN_NONE;
    noble_status st;
    at::Tensor wq, wk;
    {
        NoGil nogil;
        const c10::DeviceGuard guard(c.dev);
        at::Tensor scratch = c.work(in.wq ? bytes : 0);
        if (in.wq) {
            wq = c.empty({D}, at::kFloat);
            wk = c.empty({D}, at::kFloat);
        }
        st = p_rope_bwd(&in.d, dq, dk, in.x, in.wq, in.wk, in.cos, in.sin, in.positions, g->data_ptr(),
                        in.wq ? static_cast<float*>(wq.data_ptr()) : nullptr,
                        in.wq ? static_cast<float*>(wk.data_ptr()) : nullptr, scratch.data_ptr(),
                        (size_t)scratch.numel(), c.stream());
    }
    return st == NOBLE_OK ? tuple({&wq, &wk}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// append(10 of RopeIn, slots, cache, q) -> (q,).
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 13) Py_RETURN_NONE;
    Call c;
    const RopeIn in(c, a);
    const int64_t* slots = static_cast<int64_t*>(c.dense(a[10], at::kLong, {in.d.T}));
    const at::Tensor* t = c.tensor(a[11]);
    if (!c.ok || a[10] == Py_None || t->dim() != 5 || t->size(3) > 4096) Py_RETURN_NONE;
    noble_cache_desc cd{t->size(0), (int32_t)t->size(3), 0};
    void* cache = c.dense(a[11], c.sd, {t->size(0), 2, in.d.kv_heads, t->size(3), in.d.head_dim});
    const Output q(c, a[12], {in.d.T, in.d.heads, in.d.head_dim}, c.sd);
    void* pq = q.dense(c);
    if (!c.ok) Py_RETURN_NONE;
    noble_status st;
    {
        NoGil nogil;
        const c10::DeviceGuard guard(c.dev);
        st = p_append(&in.d, &cd, in.x, in.wq, in.wk, in.cos, in.sin, in.positions, slots, pq, cache, c.stream());
    }
    return st == NOBLE_OK ? tuple({&q.t}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// (q, k, v, key_lo, key_hi, slopes, causal, offset, scale, softcap) of the attention calls.
struct AttnIn {
    noble_attn_desc d{};
    noble_heads q{}, k{}, v{};
    int32_t *lo = nullptr, *hi = nullptr;
    float* slopes = nullptr;
    AttnIn(Call& c, PyObject* const* a) {
        const at::Tensor *tq = c.first(a[0]), *tk = c.tensor(a[1]);
        if (!c.ok || tq->dim() != 3 || tk->dim() != 3 || tq->size(1) > 4096 || tk->size(1) > 4096 || tq->size(2) > 4096) {
            c.ok = false;
            return;
        }
        const int64_t H = tq->size(1), K = tk->size(1), D = tq->size(2);
        d.Tq = tq->size(0);
        d.Tk = tk->size(0);
        d.heads = (int32_t)H;
        d.kv_heads = (int32_t)K;
        d.head_dim = (int32_t)D;
        d.dtype = c.dtype;
        q = c.heads(a[0], d.Tq, H, D);
        k = c.heads(a[1], d.Tk, K, D);
        v = c.heads(a[2], d.Tk, K, D);
        if ((a[3] == Py_None) != (a[4] == Py_None)) c.ok = false;
        lo = c.ints(a[3], {d.Tq});
        hi = c.ints(a[4], {d.Tq});
        slopes = c.floats(a[5], {H});
        d.causal = c.truth(a[6]);
        d.offset = a[7] == Py_None ? d.Tk - d.Tq : c.integer(a[7], INT32_MIN, INT32_MAX);
        d.scale = c.scale(a[8], D);
        d.softcap = c.number(a[9]);
    }
};

// attn_fwd(10 of AttnIn, o, lse) -> (o, lse).
PyObject* attn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    Call c;
    const AttnIn in(c, a);
    if (!c.ok) Py_RETURN_NONE;
    const Output o(c, a[10], {in.d.Tq, in.d.heads, in.d.head_dim}, c.sd), lse(c, a[11], {in.d.heads, in.d.Tq}, at::kFloat);
    const noble_heads oh = o.heads(c);
    float* pl = static_cast<float*>(lse.dense(c));
    if (!c.ok) Py_RETURN_NONE;
    noble_status st;
    {
        NoGil nogil;
        const c10::DeviceGuard guard(c.dev);
        st = p_attn_fwd(&in.d, &in.q, &in.k, &in.v, in.lo, in.hi, in.slopes, &oh, pl, c.stream());
    }
    return st == NOBLE_OK ? tuple({&o.t, &lse.t}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// attn_bwd(do, o, lse, 10 of AttnIn, dq, dk, dv) -> (dq, dk, dv).
PyObject* attn_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 16) Py_RETURN_NONE;
    Call c;
    const AttnIn in(c, a + 3);
    if (!c.ok) Py_RETURN_NONE;
    const int64_t Tq = in.d.Tq, Tk = in.d.Tk, H = in.d.heads, K = in.d.kv_heads, D = in.d.head_dim;
    const noble_heads g = c.heads(a[0], Tq, H, D), o = c.heads(a[1], Tq, H, D);
    const float* lse = c.floats(a[2], {H, Tq});
    const Output dq(c, a[13], {Tq, H, D}, c.sd), dk(c, a[14], {Tk, K, D}, c.sd), dv(c, a[15], {Tk, K, D}, c.sd);
    const noble_heads hq = dq.heads(c), hk = dk.heads(c), hv = dv.heads(c);
    size_t bytes = 0;
    if (!c.ok || a[2] == Py_None || p_bwd_size(&in.d, &bytes) != NOBLE_OK) Py_RETURN_NONE;
    noble_status st;
    {
        NoGil nogil;
        const c10::DeviceGuard guard(c.dev);
        const at::Tensor scratch = c.work(bytes);
        st = p_attn_bwd(&in.d, &g, &in.q, &in.k, &in.v, &o, lse, in.lo, in.hi, in.slopes, &hq, &hk, &hv,
                        scratch.data_ptr(), (size_t)scratch.numel(), c.stream());
    }
    return st == NOBLE_OK ? tuple({&dq.t, &dk.t, &dv.t}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// paged(q, cache, page_table, lengths, slopes, scale, softcap, window, o) -> (o,).
PyObject* paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 9) Py_RETURN_NONE;
    Call c;
    const at::Tensor *tq = c.first(a[0]), *tc = c.tensor(a[1]), *tt = c.tensor(a[2]);
    if (!c.ok || tq->dim() != 3 || tc->dim() != 5 || tt->dim() != 2 || tt->size(0) < 1 || tq->size(0) < tt->size(0) ||
        tq->size(0) % tt->size(0) || tq->size(0) / tt->size(0) > (1 << 20) || tq->size(1) > 4096 || tq->size(2) > 4096 ||
        tc->size(2) > 4096 || tc->size(3) > 4096)
        Py_RETURN_NONE;
    noble_paged_desc d{};
    const int64_t rows = tq->size(0), H = tq->size(1), D = tq->size(2);
    d.B = tt->size(0);
    d.table_row = tt->size(1);
    d.pages = tc->size(0);
    d.page = (int32_t)tc->size(3);
    d.new_tokens = (int32_t)(rows / d.B);
    d.heads = (int32_t)H;
    d.kv_heads = (int32_t)tc->size(2);
    d.head_dim = (int32_t)D;
    d.dtype = c.dtype;
    const noble_heads q = c.heads(a[0], rows, H, D);
    const void* cache = c.dense(a[1], c.sd, {d.pages, 2, d.kv_heads, d.page, D});
    const int32_t *table = c.ints(a[2], {d.B, d.table_row}), *lengths = c.ints(a[3], {d.B});
    const float* slopes = c.floats(a[4], {H});
    d.scale = c.scale(a[5], D);
    d.softcap = c.number(a[6]);
    d.window = (int32_t)c.integer(a[7], 0, INT32_MAX);
    const Output o(c, a[8], {rows, H, D}, c.sd);
    const noble_heads oh = o.heads(c);
    size_t bytes = 0;
    if (!c.ok || a[3] == Py_None || p_paged_size(&d, &bytes) != NOBLE_OK) Py_RETURN_NONE;
    noble_status st;
    {
        NoGil nogil;
        const c10::DeviceGuard guard(c.dev);
        at::Tensor scratch;
        if (bytes) scratch = c.work(bytes);
        st = p_paged(&d, &q, cache, table, lengths, slopes, &oh, bytes ? scratch.data_ptr() : nullptr, bytes, c.stream());
    }
    return st == NOBLE_OK ? tuple({&o.t}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// init(rope_fwd, rope_bwd, rope_scratch_size, append, attn_fwd, attn_bwd, attn_bwd_scratch_size, paged, paged_scratch_size):
// the library's entry points, as addresses.
PyObject* init(PyObject*, PyObject* args) {
    unsigned long long p[9];
    if (!PyArg_ParseTuple(args, "KKKKKKKKK", &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6], &p[7], &p[8])) return nullptr;
    p_rope_fwd = reinterpret_cast<decltype(p_rope_fwd)>(p[0]);
    p_rope_bwd = reinterpret_cast<decltype(p_rope_bwd)>(p[1]);
    p_rope_size = reinterpret_cast<decltype(p_rope_size)>(p[2]);
    p_append = reinterpret_cast<decltype(p_append)>(p[3]);
    p_attn_fwd = reinterpret_cast<decltype(p_attn_fwd)>(p[4]);
    p_attn_bwd = reinterpret_cast<decltype(p_attn_bwd)>(p[5]);
    p_bwd_size = reinterpret_cast<decltype(p_bwd_size)>(p[6]);
    p_paged = reinterpret_cast<decltype(p_paged)>(p[7]);
    p_paged_size = reinterpret_cast<decltype(p_paged_size)>(p[8]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"init", init, METH_VARARGS, nullptr},
                         NOBLE_FAST(rope_fwd),
                         NOBLE_FAST(rope_bwd),
                         NOBLE_FAST(append),
                         NOBLE_FAST(attn_fwd),
                         NOBLE_FAST(attn_bwd),
                         NOBLE_FAST(paged),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_noble_attn_torch", nullptr, -1, methods, nullptr, nullptr, nullptr,
                          nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__noble_attn_torch(void) { return PyModule_Create(&module_def); }
