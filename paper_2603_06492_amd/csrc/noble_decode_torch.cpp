// The decoding side's calls on torch tensors, in native code: argument checks, buffers and the library call of the functions
// of decoding.py.  As in noble_attn_torch.cpp, each serves the well-formed call on ordinary tensors and returns None for
// every other one, which the Python code then checks and runs; a status other than NOBLE_OK comes back as an int.  The
// library's entry points come in as addresses (init).
#include "noble_torch_call.hpp"

#include "noble_decode.h"

namespace {

decltype(&noble_tree_rows) p_tree_rows;
decltype(&noble_attn_tree) p_attn_tree;
decltype(&noble_attn_tree_scratch_size) p_tree_size;
decltype(&noble_cache_keep) p_keep;
decltype(&noble_page_means) p_means;
decltype(&noble_block_select) p_select;
decltype(&noble_block_select_scratch_size) p_select_size;
decltype(&noble_attn_blocks) p_attn_blocks;
decltype(&noble_attn_blocks_scratch_size) p_blocks_size;
decltype(&noble_attn_weigh) p_attn_weigh;
decltype(&noble_attn_weigh_scratch_size) p_weigh_size;
decltype(&noble_evict_select) p_evict;

// The cache's own fields of the descriptor, from the cache and the page table.
const void* cache_in(Call& c, PyObject* cache, PyObject* table, noble_paged_desc& d) {
    const at::Tensor *tc = c.tensor(cache), *tt = c.tensor(table);
    if (!c.ok || tc->dim() != 5 || tt->dim() != 2 || tc->size(2) > 4096 || tc->size(3) > 4096 || tc->size(4) > 4096) {
        c.ok = false;
        return nullptr;
    }
    d.B = tt->size(0);
    d.table_row = tt->size(1);
    d.pages = tc->size(0);
    d.page = (int32_t)tc->size(3);
    d.kv_heads = (int32_t)tc->size(2);
    d.head_dim = (int32_t)tc->size(4);
    d.dtype = c.dtype;
    return c.dense(cache, c.sd, {d.pages, 2, d.kv_heads, d.page, d.head_dim});
}
// An int32 array that has to be given.
int32_t* given(Call& c, PyObject* o, std::initializer_list<int64_t> shape) {
    if (o == Py_None) c.ok = false;
    return c.ints(o, shape);
}
// A given tensor's sizes, `dims` of them.
const at::Tensor* shaped(Call& c, PyObject* o, int64_t dims) {
    const at::Tensor* t = c.tensor(o);
    if (c.ok && t->dim() != dims) c.ok = false;
    return c.ok ? t : nullptr;
}

// (q, cache, page_table, lengths) and (slopes, scale, softcap) of the attention calls.
struct SequencesIn {
    noble_paged_desc d{};
    noble_heads q{};
    const void* cache = nullptr;
    int32_t *table = nullptr, *lengths = nullptr;
    float* slopes = nullptr;
    int64_t rows = 0, tokens = 0;
    SequencesIn(Call& c, PyObject* const* a, PyObject* const* how) {
        const at::Tensor* t = c.first(a[0]);
        if (!c.ok || t->dim() != 3 || t->size(1) > 4096) {
            c.ok = false;
            return;
        }
        cache = cache_in(c, a[1], a[2], d);
        rows = t->size(0);
        if (!c.ok || d.B < 1 || rows < d.B || rows % d.B || rows / d.B > (1 << 20)) {
            c.ok = false;
            return;
        }
        d.new_tokens = (int32_t)(rows / d.B);
        d.heads = (int32_t)t->size(1);
        tokens = d.table_row * d.page;
        q = c.heads(a[0], rows, d.heads, d.head_dim);
        table = given(c, a[2], {d.B, d.table_row});
        lengths = given(c, a[3], {d.B});
        slopes = c.floats(how[0], {d.heads});
        d.scale = c.scale(how[1], d.head_dim);
        d.softcap = c.number(how[2]);
    }
    c10::IntArrayRef shape() {
        sizes[0] = rows;
        sizes[1] = d.heads;
        sizes[2] = d.head_dim;
        return sizes;
    }
    int64_t sizes[3];
};

// Runs fn(scratch, its bytes, stream) on the call's device, without the GIL.
template <typename Fn>
noble_status on_device(const Call& c, size_t bytes, Fn&& fn) {
    NoGil nogil;
    const c10::DeviceGuard guard(c.dev);
    at::Tensor scratch;
    if (bytes) scratch = c.work(bytes);
    return fn(bytes ? scratch.data_ptr() : nullptr, bytes, c.stream());
}

// tree_rows(parents, lengths) -> (seen, depths, positions).
PyObject* tree_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 2) Py_RETURN_NONE;
    Call c;
    const at::Tensor* t = shaped(c, a[0], 2);
    if (!c.ok || t->size(1) < 1 || t->size(1) > NOBLE_TREE_MOST) Py_RETURN_NONE;
    c.dev = t->device();
    const int64_t B = t->size(0), nodes = t->size(1);
    const int32_t *parents = given(c, a[0], {B, nodes}), *lengths = given(c, a[1], {B});
    if (!c.ok) Py_RETURN_NONE;
    const at::Tensor seen = c.empty({B, nodes, NOBLE_TREE_WORDS(nodes)}, at::kInt), depths = c.empty({B, nodes}, at::kInt),
                     positions = c.empty({B, nodes}, at::kInt);
    const noble_status st = on_device(c, 0, [&](void*, size_t, void* s) {
        return p_tree_rows(B, (int32_t)nodes, parents, lengths, static_cast<int32_t*>(seen.data_ptr()),
                           static_cast<int32_t*>(depths.data_ptr()), static_cast<int32_t*>(positions.data_ptr()), s);
    });
    return st == NOBLE_OK ? tuple({&seen, &depths, &positions}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// attn_tree(q, cache, page_table, lengths, seen, depths, slopes, scale, softcap, o) -> (o,).
PyObject* attn_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 10) Py_RETURN_NONE;
    Call c;
    SequencesIn in(c, a, a + 6);
    if (!c.ok || in.d.new_tokens > NOBLE_TREE_MOST) Py_RETURN_NONE;
    const int64_t nodes = in.d.new_tokens;
    const int32_t *seen = given(c, a[4], {in.d.B, nodes, NOBLE_TREE_WORDS(nodes)}), *depths = given(c, a[5], {in.d.B, nodes});
    const Output o(c, a[9], in.shape(), c.sd);
    const noble_heads oh = o.heads(c);
    size_t bytes = 0;
    if (!c.ok || p_tree_size(&in.d, &bytes) != NOBLE_OK) Py_RETURN_NONE;
    const noble_status st = on_device(c, bytes, [&](void* w, size_t size, void* s) {
        return p_attn_tree(&in.d, &in.q, in.cache, in.table, in.lengths, seen, depths, in.slopes, &oh, w, size, s);
    });
    return st == NOBLE_OK ? tuple({&o.t}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// keep(cache, page_table, kept, start) -> True.
PyObject* keep(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 4) Py_RETURN_NONE;
    Call c;
    c.first(a[0]);
    noble_paged_desc d{};
    void* cache = const_cast<void*>(cache_in(c, a[0], a[1], d));
    const at::Tensor* t = shaped(c, a[2], 3);
    if (!c.ok || t->size(0) != d.B || (t->size(1) != 1 && t->size(1) != d.kv_heads)) Py_RETURN_NONE;
    const noble_keep_desc kd{d.B, d.table_row, d.pages, t->size(2), d.page, d.kv_heads, d.head_dim, (int32_t)t->size(1),
                             d.dtype, 0};
    const int32_t *table = given(c, a[1], {d.B, d.table_row}), *kept = given(c, a[2], {d.B, t->size(1), t->size(2)}),
                  *start = c.ints(a[3], {d.B});
    if (!c.ok) Py_RETURN_NONE;
    const noble_status st = on_device(c, 0, [&](void*, size_t, void* s) { return p_keep(&kd, cache, table, kept, start, s); });
    if (st != NOBLE_OK) return PyLong_FromLong(st);
    return tuple({});
    END_HANDLE_TH_ERRORS
}

// page_means(cache, page_table, lengths, new, means) -> (), into given means.
PyObject* page_means(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 5 || a[4] == Py_None) Py_RETURN_NONE;
    Call c;
    c.first(a[0]);
    noble_paged_desc d{};
    const void* cache = cache_in(c, a[0], a[1], d);
    const int32_t *table = given(c, a[1], {d.B, d.table_row}), *lengths = given(c, a[2], {d.B});
    d.new_tokens = (int32_t)c.integer(a[3], 1, INT32_MAX);
    void* means = c.dense(a[4], c.sd, {d.pages, d.kv_heads, d.head_dim});
    if (!c.ok) Py_RETURN_NONE;
    const noble_status st =
        on_device(c, 0, [&](void*, size_t, void* s) { return p_means(&d, cache, table, lengths, means, s); });
    if (st != NOBLE_OK) return PyLong_FromLong(st);
    return tuple({});
    END_HANDLE_TH_ERRORS
}

// block_select(q, means, page_table, lengths, count, page, sink, local, chosen) -> (chosen,).
PyObject* block_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 9) Py_RETURN_NONE;
    Call c;
    const at::Tensor *tq = c.first(a[0]), *tm = shaped(c, a[1], 3), *tt = shaped(c, a[2], 2);
    if (!c.ok || tq->dim() != 3 || tt->size(0) < 1 || tq->size(0) < tt->size(0) || tq->size(0) % tt->size(0) ||
        tq->size(0) / tt->size(0) > (1 << 20) || tq->size(1) > 4096 || tq->size(2) > 4096 || tm->size(1) > 4096)
        Py_RETURN_NONE;
    noble_paged_desc d{};
    d.B = tt->size(0);
    d.table_row = tt->size(1);
    d.pages = tm->size(0);
    d.page = (int32_t)c.integer(a[5], 1, 4096);
    d.new_tokens = (int32_t)(tq->size(0) / d.B);
    d.heads = (int32_t)tq->size(1);
    d.kv_heads = (int32_t)tm->size(1);
    d.head_dim = (int32_t)tq->size(2);
    d.dtype = c.dtype;
    d.scale = 1.f;
    const int64_t rows = tq->size(0);
    const noble_heads q = c.heads(a[0], rows, d.heads, d.head_dim);
    const void* means = c.dense(a[1], c.sd, {d.pages, d.kv_heads, d.head_dim});
    const int32_t *table = given(c, a[2], {d.B, d.table_row}), *lengths = given(c, a[3], {d.B});
    const noble_select_desc e{(int32_t)c.integer(a[4], 1, 65536), (int32_t)c.integer(a[6], 0, 65536),
                              (int32_t)c.integer(a[7], 1, 65536), 0};
    const Output chosen(c, a[8], {rows, d.kv_heads, e.count}, at::kInt);
    int32_t* pc = static_cast<int32_t*>(chosen.dense(c));
    size_t bytes = 0;
    if (!c.ok || p_select_size(&d, &e, &bytes) != NOBLE_OK) Py_RETURN_NONE;
    const noble_status st = on_device(c, bytes, [&](void* w, size_t size, void* s) {
        return p_select(&d, &e, &q, means, table, lengths, pc, w, size, s);
    });
    return st == NOBLE_OK ? tuple({&chosen.t}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// attn_blocks(q, cache, page_table, lengths, chosen, slopes, scale, softcap, o) -> (o,).
PyObject* attn_blocks(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 9) Py_RETURN_NONE;
    Call c;
    SequencesIn in(c, a, a + 5);
    const at::Tensor* t = shaped(c, a[4], 3);
    if (!c.ok || t->size(2) < 1 || t->size(2) > 65536) Py_RETURN_NONE;
    const int32_t count = (int32_t)t->size(2);
    const int32_t* chosen = given(c, a[4], {in.rows, in.d.kv_heads, count});
    const Output o(c, a[8], in.shape(), c.sd);
    const noble_heads oh = o.heads(c);
    size_t bytes = 0;
    if (!c.ok || p_blocks_size(&in.d, count, &bytes) != NOBLE_OK) Py_RETURN_NONE;
    const noble_status st = on_device(c, bytes, [&](void* w, size_t size, void* s) {
        return p_attn_blocks(&in.d, count, &in.q, in.cache, in.table, in.lengths, chosen, in.slopes, &oh, w, size, s);
    });
    return st == NOBLE_OK ? tuple({&o.t}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// attn_weigh(q, cache, page_table, lengths, weights, slopes, scale, softcap, o, out) -> (o, out), into a given out.
PyObject* attn_weigh(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 10 || a[9] == Py_None) Py_RETURN_NONE;
    Call c;
    SequencesIn in(c, a, a + 5);
    const float* weights = c.floats(a[4], {in.d.B, in.d.kv_heads, in.tokens});
    const Output o(c, a[8], in.shape(), c.sd), out(c, a[9], {in.d.B, in.d.kv_heads, in.tokens}, at::kFloat);
    const noble_heads oh = o.heads(c);
    float* po = static_cast<float*>(out.dense(c));
    size_t bytes = 0;
    if (!c.ok || p_weigh_size(&in.d, &bytes) != NOBLE_OK) Py_RETURN_NONE;
    const noble_status st = on_device(c, bytes, [&](void* w, size_t size, void* s) {
        return p_attn_weigh(&in.d, &in.q, in.cache, in.table, in.lengths, in.slopes, weights, po, &oh, w, size, s);
    });
    return st == NOBLE_OK ? tuple({&o.t, &out.t}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// evict_select(weights, lengths, keep, sink, recent, kept, kept_weights) -> (kept, kept_weights).
PyObject* evict_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 7) Py_RETURN_NONE;
    Call c;
    const at::Tensor* t = shaped(c, a[0], 3);
    if (!c.ok || t->size(1) < 1 || t->size(1) > 4096) Py_RETURN_NONE;
    c.dev = t->device();
    noble_evict_desc d{};
    d.B = t->size(0);
    d.heads = (int32_t)t->size(1);
    d.row = t->size(2);
    const float* weights = c.floats(a[0], {d.B, d.heads, d.row});
    const int32_t* lengths = given(c, a[1], {d.B});
    d.keep = (int32_t)c.integer(a[2], 1, INT32_MAX - 4095);
    d.sink = (int32_t)c.integer(a[3], 0, INT32_MAX);
    d.recent = (int32_t)c.integer(a[4], 0, INT32_MAX);
    const Output kept(c, a[5], {d.B, d.heads, d.keep}, at::kInt), kw(c, a[6], {d.B, d.heads, d.keep}, at::kFloat);
    int32_t* pk = static_cast<int32_t*>(kept.dense(c));
    float* pw = static_cast<float*>(kw.dense(c));
    if (!c.ok) Py_RETURN_NONE;
    const noble_status st =
        on_device(c, 0, [&](void*, size_t, void* s) { return p_evict(&d, weights, lengths, pk, pw, s); });
    return st == NOBLE_OK ? tuple({&kept.t, &kw.t}) : PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// init(the library's entry points, as addresses, in the order of the declarations above).
PyObject* init(PyObject*, PyObject* args) {
    unsigned long long p[12];
    if (!PyArg_ParseTuple(args, "KKKKKKKKKKKK", &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6], &p[7], &p[8], &p[9], &p[10],
                          &p[11]))
        return nullptr;
    p_tree_rows = reinterpret_cast<decltype(p_tree_rows)>(p[0]);
    p_attn_tree = reinterpret_cast<decltype(p_attn_tree)>(p[1]);
    p_tree_size = reinterpret_cast<decltype(p_tree_size)>(p[2]);
    p_keep = reinterpret_cast<decltype(p_keep)>(p[3]);
    p_means = reinterpret_cast<decltype(p_means)>(p[4]);
    p_select = reinterpret_cast<decltype(p_select)>(p[5]);
    p_select_size = reinterpret_cast<decltype(p_select_size)>(p[6]);
    p_attn_blocks = reinterpret_cast<decltype(p_attn_blocks)>(p[7]);
    p_blocks_size = reinterpret_cast<decltype(p_blocks_size)>(p[8]);
    p_attn_weigh = reinterpret_cast<decltype(p_attn_weigh)>(p[9]);
    p_weigh_size = reinterpret_cast<decltype(p_weigh_size)>(p[10]);
    p_evict = reinterpret_cast<decltype(p_evict)>(p[11]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"init", init, METH_VARARGS, nullptr},
                         NOBLE_FAST(tree_rows),
                         NOBLE_FAST(attn_tree),
                         NOBLE_FAST(keep),
                         NOBLE_FAST(page_means),
                         NOBLE_FAST(block_select),
                         NOBLE_FAST(attn_blocks),
                         NOBLE_FAST(attn_weigh),
                         NOBLE_FAST(evict_select),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_noble_decode_torch", nullptr, -1, methods, nullptr, nullptr, nullptr,
                          nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__noble_decode_torch(void) { return PyModule_Create(&module_def); }
