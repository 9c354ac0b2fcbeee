// The host side of the calls that a decoding loop makes once a step: argument checks, device pointers and the current stream in one
// C++ call each.  A launch costs the host 2 to 3 us; checked and marshalled in Python (nine tensors a call, an object for the
// stream, ctypes' conversions) a call took 10 to 13 us, longer than the kernels of a small batch run: acceptance of one sequence over 32 k
// tokens 11.4 us a call that way and 5 to 6 this way, a prompt of 300 tokens with reset and first draft (three calls) 24 and 19 us.
//
// The entry points of the C library come as addresses from _lib.load() (set_library), so that this module calls the build of the library
// that was loaded.  What a check refuses raises CachebackError with the text that it has in api.py; torch's own exceptions
// (a stride of a tensor without dimensions, a tensor without memory) pass through as they do there.
#include <Python.h>

#include <algorithm>
#include <initializer_list>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "cacheback.h"

namespace {

PyObject* g_error = nullptr;                                 // CachebackError
PyObject *s_cuda_stream, *s_tokens, *s_parent, *s_depth, *s_mask, *s_n_nodes, *s_n_accept, *s_accept_nodes, *s_out_tokens, *s_target_ids;

struct Library {
    decltype(&cb_reset) reset;
    decltype(&cb_update) update;
    decltype(&cb_update_bulk) update_bulk;
    decltype(&cb_draft_tree) draft_tree;
    decltype(&cb_update_draft_tree) update_draft_tree;
    decltype(&cb_tree_attn) tree_attn;
    decltype(&cb_accept) accept;
    decltype(&cb_accept_update_draft_tree) accept_update_draft_tree;
    decltype(&cb_kv_commit) kv_commit;
    decltype(&cb_chunk_append) chunk_append;
    decltype(&cb_chunk_attn) chunk_attn;
    decltype(&cb_tree_rope) tree_rope;
    decltype(&cb_logprobs) logprobs;
    decltype(&cb_accept_logprobs) accept_logprobs;
    decltype(&cb_status_str) status_str;
} g_lib;

struct Refused {};                                           // a Python exception is set

[[noreturn]] void refuse(const char* text) {
    PyErr_SetString(g_error, text);
    throw Refused();
}

const at::Tensor& tensor_of(PyObject* o) {
    if (!THPVariable_Check(o)) refuse("expected a contiguous CUDA tensor");
    return THPVariable_Unpack(o);
}

const char* type_name(at::ScalarType t) { return t == at::kInt ? "torch.int32" : t == at::kFloat ? "torch.float32" : "torch.bfloat16"; }

// The device pointer of a contiguous CUDA tensor of the given type; None: a null pointer.
template <typename T = int32_t>
T* ptr(PyObject* o, at::ScalarType want = at::kInt) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor_of(o);
    if (!t.is_cuda() || !t.is_contiguous()) refuse("expected a contiguous CUDA tensor");
    if (t.scalar_type() != want) {
        PyObject* d = PyObject_GetAttrString(o, "dtype");
        if (d) { PyErr_Format(g_error, "expected dtype %s, got %S", type_name(want), d); Py_DECREF(d); }
        throw Refused();
    }
    return static_cast<T*>(t.data_ptr());
}

struct Ref {                                                 // an owned reference
    PyObject* o;
    explicit Ref(PyObject* x) : o(x) { if (!x) throw Refused(); }
    Ref(const Ref&) = delete;
    ~Ref() { Py_DECREF(o); }
};
template <typename T = int32_t>
T* item(PyObject* mapping, PyObject* key) {
    Ref r(PyObject_GetItem(mapping, key));
    return ptr<T>(r.o);
}

void* stream_of(PyObject* o) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    Ref r(PyObject_GetAttr(o, s_cuda_stream));
    void* p = PyLong_AsVoidPtr(r.o);
    if (!p && PyErr_Occurred()) throw Refused();
    return p;
}

cb_ctx* ctx_of(PyObject* o) {
    if (o == Py_None) return nullptr;                         // a closed context: the library refuses it
    Ref r(PyObject_GetAttrString(o, "value"));
    if (r.o == Py_None) return nullptr;
    void* p = PyLong_AsVoidPtr(r.o);
    if (!p && PyErr_Occurred()) throw Refused();
    return static_cast<cb_ctx*>(p);
}

// The logits of all nodes: [batch, max_nodes, vocab] with one stride from row to row.
const void* logits_of(PyObject* o, int32_t* dtype, int64_t* stride) {
    const at::Tensor& t = tensor_of(o);
    if (t.scalar_type() == at::kFloat) *dtype = CB_DTYPE_F32;
    else if (t.scalar_type() == at::kBFloat16) *dtype = CB_DTYPE_BF16;
    else refuse("logits must be float32 or bfloat16");
    if (!(t.is_cuda() && t.dim() == 3 && t.stride(2) == 1 && t.stride(0) == t.size(1) * t.stride(1)))
        refuse("logits must be [batch, max_nodes, vocab] with a uniform row stride");
    *stride = t.stride(1);
    return t.data_ptr();
}

int64_t long_of(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    return v;
}

template <typename F>
void call(const char* what, F&& f) {
    cb_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    if (st != CB_OK) {
        PyErr_Format(g_error, "%s failed: %s", what, g_lib.status_str(st));
        throw Refused();
    }
}

// Python's entry: the number of arguments is fixed (api.py fills in the defaults)
template <int N, void (*F)(PyObject* const*)>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != N) { PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n); return nullptr; }
    try {
        F(a);
    } catch (const Refused&) {
        return nullptr;
    }
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// The token history [batch, columns]: its pointer and the columns that a row has.  The stride of a dimension of size one says nothing:
// the transpose of a [columns, 1] tensor is contiguous with a stride of 1.
template <typename T = int32_t>
T* history_of(PyObject* o, int64_t* row_stride) {
    T* p = ptr<T>(o);
    const at::Tensor& t = tensor_of(o);
    *row_stride = t.stride(0);
    if (t.dim() > 1 && t.size(0) == 1) *row_stride = std::max(*row_stride, t.numel());
    return p;
}

// handle, seq_mask, stream
void do_reset(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    const int32_t* m = ptr(a[1]);
    void* st = stream_of(a[2]);
    call("cb_reset", [&] { return g_lib.reset(c, m, st); });
}
// handle, tokens, n_old, n_new, stream
template <bool BULK>
void do_update(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    int64_t rs;
    const int32_t* tok = history_of(a[1], &rs);
    const int32_t *n0 = ptr(a[2]), *n1 = ptr(a[3]);
    void* st = stream_of(a[4]);
    call(BULK ? "cb_update_bulk" : "cb_update", [&] { return (BULK ? g_lib.update_bulk : g_lib.update)(c, tok, rs, n0, n1, st); });
}
struct Tree { int32_t *tok, *par, *dep; uint32_t* mask; int32_t* n; };
Tree tree_of(PyObject* t, bool mask) {
    Tree r;
    r.tok = item(t, s_tokens); r.par = item(t, s_parent); r.dep = item(t, s_depth);
    r.mask = mask ? item<uint32_t>(t, s_mask) : nullptr;
    r.n = item(t, s_n_nodes);
    return r;
}
// handle, tokens, seq_len, tree, stream
void do_draft(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    int64_t rs;
    const int32_t* tok = history_of(a[1], &rs);
    const int32_t* n = ptr(a[2]);
    const Tree t = tree_of(a[3], true);
    void* st = stream_of(a[4]);
    call("cb_draft_tree", [&] { return g_lib.draft_tree(c, tok, rs, n, t.tok, t.par, t.dep, t.mask, t.n, st); });
}
// handle, tokens, n_old, n_new, tree, stream
void do_update_draft(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    int64_t rs;
    const int32_t* tok = history_of(a[1], &rs);
    const int32_t *n0 = ptr(a[2]), *n1 = ptr(a[3]);
    const Tree t = tree_of(a[4], true);
    void* st = stream_of(a[5]);
    call("cb_update_draft_tree", [&] { return g_lib.update_draft_tree(c, tok, rs, n0, n1, t.tok, t.par, t.dep, t.mask, t.n, st); });
}
// handle, tree, logits, target_ids, res, stream
void do_accept(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    int32_t dtype = 0;
    int64_t rs = 0;
    const void* lg = a[2] == Py_None ? nullptr : logits_of(a[2], &dtype, &rs);
    const Tree t = tree_of(a[1], false);
    const int32_t* ids = ptr(a[3]);
    int32_t *na = item(a[4], s_n_accept), *an = item(a[4], s_accept_nodes), *ot = item(a[4], s_out_tokens), *ti = item(a[4], s_target_ids);
    void* st = stream_of(a[5]);
    call("cb_accept", [&] { return g_lib.accept(c, t.tok, t.par, t.dep, t.n, lg, dtype, rs, ids, na, an, ot, ti, st); });
}
// handle, tree, logits, tokens, seq_len, next_tree, res, stream
void do_accept_update_draft(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    cb_accept_draft_args x = {};
    x.logits = logits_of(a[2], &x.logits_dtype, &x.logits_row_stride);
    const Tree t = tree_of(a[1], false);
    x.tree_tokens = t.tok; x.tree_parent = t.par; x.tree_depth = t.dep; x.n_nodes = t.n;
    x.n_accept = item(a[6], s_n_accept); x.accept_nodes = item(a[6], s_accept_nodes);
    x.out_tokens = item(a[6], s_out_tokens); x.target_ids_out = item(a[6], s_target_ids);
    x.tokens = history_of(a[3], &x.row_stride);
    x.seq_len = ptr(a[4]);
    const Tree n = tree_of(a[5], true);
    x.next_tokens = n.tok; x.next_parent = n.par; x.next_depth = n.dep; x.next_mask = n.mask; x.next_n_nodes = n.n;
    void* st = stream_of(a[7]);
    call("cb_accept_update_draft_tree", [&] { return g_lib.accept_update_draft_tree(c, &x, st); });
}
// handle, q, k_pool, v_pool, block_table, ctx_len, k_tree, v_tree, tree_mask, n_nodes, out, lse, max_ctx, scale, stream
void do_attn(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    cb_attn_args x = {};
    const auto bf = at::kBFloat16;
    x.q = ptr<void>(a[1], bf); x.k_pool = ptr<void>(a[2], bf); x.v_pool = ptr<void>(a[3], bf);
    x.block_table = ptr(a[4]); x.ctx_len = ptr(a[5]);
    x.k_tree = ptr<void>(a[6], bf); x.v_tree = ptr<void>(a[7], bf);
    x.tree_mask = ptr<uint32_t>(a[8]); x.n_nodes = ptr(a[9]);
    x.out = ptr<void>(a[10], bf); x.lse = ptr<float>(a[11], at::kFloat);
    x.max_pages = (int32_t)tensor_of(a[4]).size(1);
    x.num_pages = (int32_t)tensor_of(a[2]).size(0);
    x.max_ctx = (int32_t)long_of(a[12]);
    const double sc = PyFloat_AsDouble(a[13]);
    if (sc == -1.0 && PyErr_Occurred()) throw Refused();
    x.scale = (float)sc;
    void* st = stream_of(a[14]);
    call("cb_tree_attn", [&] { return g_lib.tree_attn(c, &x, st); });
}
// handle, k_pool, v_pool, block_table, ctx_len, k_tree, v_tree, n_accept, accept_nodes, stream
void do_kv_commit(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    cb_kv_commit_args x = {};
    const auto bf = at::kBFloat16;
    x.k_pool = ptr<void>(a[1], bf); x.v_pool = ptr<void>(a[2], bf);
    x.block_table = ptr(a[3]); x.ctx_len = ptr(a[4]);
    x.k_tree = ptr<void>(a[5], bf); x.v_tree = ptr<void>(a[6], bf);
    x.n_accept = ptr(a[7]); x.accept_nodes = ptr(a[8]);
    x.max_pages = (int32_t)tensor_of(a[3]).size(1);
    x.num_pages = (int32_t)tensor_of(a[1]).size(0);
    void* st = stream_of(a[9]);
    call("cb_kv_commit", [&] { return g_lib.kv_commit(c, &x, st); });
}

// ---- the operators beside the step.  Their shapes are checked against the context's, which api.py hands over as a tuple.
struct Shape { int64_t device, B, T, Hq, Hkv, D, P, Dmax, V; };
Shape shape_of(PyObject* o) {
    int64_t v[9];
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 9) { PyErr_SetString(PyExc_TypeError, "expected the context's shape"); throw Refused(); }
    for (int k = 0; k < 9; ++k) v[k] = long_of(PyTuple_GET_ITEM(o, k));
    return {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8]};
}
[[noreturn]] void refuse_shape(const char* name, const char* want) {
    PyErr_Format(g_error, "%s must be %s", name, want);
    throw Refused();
}
// A CUDA tensor on the context's device, of the given type and shape (-1: any size).  Contiguous unless `rows` is set: then its first
// dimension may have any stride.
struct Arg { const at::Tensor* t; void* p; };
Arg arg(const Shape& s, PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> want, const char* text, bool rows = false) {
    const at::Tensor& t = tensor_of(o);
    if (!t.is_cuda()) refuse("expected a contiguous CUDA tensor");
    if (t.get_device() != s.device) refuse_shape(name, "on the context's device");
    if (t.scalar_type() != type) {
        PyObject* d = PyObject_GetAttrString(o, "dtype");
        if (d) { PyErr_Format(g_error, "%s: expected dtype %s, got %S", name, type_name(type), d); Py_DECREF(d); }
        throw Refused();
    }
    bool ok = t.dim() == (int64_t)want.size();
    int64_t k = 0;
    for (int64_t w : want) { ok = ok && (w < 0 || t.size(k) == w); ++k; }
    if (!ok) refuse_shape(name, text);
    if (!rows && !t.is_contiguous()) refuse("expected a contiguous CUDA tensor");
    return {&t, t.data_ptr()};
}
template <typename T>
T* opt(const Shape& s, PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> want, const char* text) {
    return o == Py_None ? nullptr : static_cast<T*>(arg(s, o, name, type, want, text).p);
}
// The stream to launch on: the one given, or the current one of the context's device, which is the current device for the call.
struct OnDevice {
    c10::cuda::CUDAGuard guard;
    void* stream;
    OnDevice(const Shape& s, PyObject* o) : guard((c10::DeviceIndex)s.device) {
        stream = o == Py_None ? c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)s.device).stream() : stream_of(o);
    }
};
int32_t int_of(PyObject* o, const char* name) {
    const int64_t v = long_of(o);
    if (v < INT32_MIN || v > INT32_MAX) refuse_shape(name, "a 32-bit number");
    return (int32_t)v;
}
float float_of(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused();
    return (float)v;
}
// q, k, v: [rows, heads, head_dim] with the heads of a row side by side, any stride from row to row
const void* heads_of(const Shape& s, PyObject* o, const char* name, int64_t rows, int64_t heads, int64_t* stride) {
    const Arg a = arg(s, o, name, at::kBFloat16, {rows, heads, s.D}, "[rows, heads, head_dim] of the context's heads, with a row per token", true);
    const at::Tensor& t = *a.t;
    if (t.numel() > 0 && (t.stride(2) != 1 || (heads > 1 && t.stride(1) != s.D))) refuse_shape(name, "contiguous within a row");
    *stride = t.size(0) > 1 ? t.stride(0) : heads * s.D;
    return a.p;
}
int64_t rows_of(PyObject* o) {
    const at::Tensor& t = tensor_of(o);
    if (t.dim() != 3 || t.size(0) > INT32_MAX) refuse_shape("q", "[rows, heads, head_dim]");
    return t.size(0);
}
// q, k, v, q_norm, k_norm, eps, rope, interleaved
cb_qkv_rows qkv_of(const Shape& s, PyObject* const* a, int64_t n) {
    const auto bf = at::kBFloat16;
    cb_qkv_rows r = {};
    r.q = heads_of(s, a[0], "q", n, s.Hq, &r.q_stride);
    r.k = heads_of(s, a[1], "k", n, s.Hkv, &r.k_stride);
    r.v = heads_of(s, a[2], "v", n, s.Hkv, &r.v_stride);
    r.q_norm = opt<void>(s, a[3], "q_norm", bf, {s.D}, "[head_dim]");
    r.k_norm = opt<void>(s, a[4], "k_norm", bf, {s.D}, "[head_dim]");
    r.eps = float_of(a[5]);
    if (a[6] != Py_None) {
        const Arg t = arg(s, a[6], "rope", at::kFloat, {-1, -1}, "[positions, rotary_dim]");
        r.rope = static_cast<const float*>(t.p);
        r.rope_len = (int32_t)std::min<int64_t>(t.t->size(0), INT32_MAX);
        r.rotary_dim = (int32_t)std::min<int64_t>(t.t->size(1), INT32_MAX);
        if (!r.rope) refuse_shape("rope", "[positions, rotary_dim] with at least one position");
    }
    const int inter = PyObject_IsTrue(a[7]);
    if (inter < 0) throw Refused();
    r.interleaved = inter;
    return r;
}
struct Cache { void *k, *v; int32_t* table; int32_t max_pages, num_pages; };
Cache cache_of(const Shape& s, PyObject* k, PyObject* v, PyObject* table) {
    const auto bf = at::kBFloat16;
    const Arg kp = arg(s, k, "k_pool", bf, {-1, s.P, s.Hkv, s.D}, "[pages, page_size, n_kv_heads, head_dim]");
    const Arg vp = arg(s, v, "v_pool", bf, {kp.t->size(0), s.P, s.Hkv, s.D}, "of k_pool's shape");
    const Arg bt = arg(s, table, "block_table", at::kInt, {s.B, -1}, "[batch, pages]");
    if (kp.t->size(0) > INT32_MAX || bt.t->size(1) > INT32_MAX) refuse_shape("k_pool", "of less than 2^31 pages");
    return {kp.p, vp.p, static_cast<int32_t*>(bt.p), (int32_t)bt.t->size(1), (int32_t)kp.t->size(0)};
}
// handle, shape, q, k, v, q_norm, k_norm, eps, rope, interleaved, q_start, ctx_len, k_pool, v_pool, block_table, q_out, stream
void do_chunk_append(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    const Shape s = shape_of(a[1]);
    cb_chunk_append_args x = {};
    const int64_t n = rows_of(a[2]);
    x.rows = qkv_of(s, a + 2, n);
    x.n_rows = (int32_t)n;
    x.q_start = static_cast<int32_t*>(arg(s, a[10], "q_start", at::kInt, {s.B + 1}, "[batch + 1]").p);
    x.ctx_len = static_cast<int32_t*>(arg(s, a[11], "ctx_len", at::kInt, {s.B}, "[batch]").p);
    const Cache k = cache_of(s, a[12], a[13], a[14]);
    x.k_pool = k.k; x.v_pool = k.v; x.block_table = k.table; x.max_pages = k.max_pages; x.num_pages = k.num_pages;
    x.q_out = arg(s, a[15], "q_out", at::kBFloat16, {n, s.Hq, s.D}, "[rows, n_q_heads, head_dim]").p;
    if (n == 0) return;                                       // tensors without elements have no memory
    const OnDevice on(s, a[16]);
    call("cb_chunk_append", [&] { return g_lib.chunk_append(c, &x, on.stream); });
}
// handle, shape, q, k, v, q_norm, k_norm, eps, rope, interleaved, tree, ctx_len, q_out, k_out, v_out, stream
void do_tree_rope(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    const Shape s = shape_of(a[1]);
    cb_tree_rope_args x = {};
    x.rows = qkv_of(s, a + 2, s.B * s.T);
    {
        Ref depth(PyObject_GetItem(a[10], s_depth)), n(PyObject_GetItem(a[10], s_n_nodes));
        x.tree_depth = static_cast<int32_t*>(arg(s, depth.o, "depth", at::kInt, {s.B, s.T}, "[batch, max_nodes]").p);
        x.n_nodes = static_cast<int32_t*>(arg(s, n.o, "n_nodes", at::kInt, {s.B}, "[batch]").p);
    }
    x.ctx_len = static_cast<int32_t*>(arg(s, a[11], "ctx_len", at::kInt, {s.B}, "[batch]").p);
    x.q_out = arg(s, a[12], "q_out", at::kBFloat16, {s.B, s.T, s.Hq, s.D}, "[batch, max_nodes, n_q_heads, head_dim]").p;
    x.k_out = arg(s, a[13], "k_out", at::kBFloat16, {s.B, s.T, s.Hkv, s.D}, "[batch, max_nodes, n_kv_heads, head_dim]").p;
    x.v_out = arg(s, a[14], "v_out", at::kBFloat16, {s.B, s.T, s.Hkv, s.D}, "[batch, max_nodes, n_kv_heads, head_dim]").p;
    const OnDevice on(s, a[15]);
    call("cb_tree_rope", [&] { return g_lib.tree_rope(c, &x, on.stream); });
}
// handle, shape, q, k_pool, v_pool, block_table, q_start, ctx_len, out, lse, max_chunk, max_ctx, scale, stream
void do_chunk_attn(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    const Shape s = shape_of(a[1]);
    cb_chunk_attn_args x = {};
    const int64_t n = rows_of(a[2]);
    const auto bf = at::kBFloat16;
    x.q = arg(s, a[2], "q", bf, {n, s.Hq, s.D}, "[rows, n_q_heads, head_dim]").p;
    x.n_rows = (int32_t)n;
    const Cache k = cache_of(s, a[3], a[4], a[5]);
    x.k_pool = k.k; x.v_pool = k.v; x.block_table = k.table; x.max_pages = k.max_pages; x.num_pages = k.num_pages;
    x.q_start = static_cast<int32_t*>(arg(s, a[6], "q_start", at::kInt, {s.B + 1}, "[batch + 1]").p);
    x.ctx_len = static_cast<int32_t*>(arg(s, a[7], "ctx_len", at::kInt, {s.B}, "[batch]").p);
    x.out = arg(s, a[8], "out", bf, {n, s.Hq, s.D}, "of q's shape").p;
    x.lse = opt<float>(s, a[9], "lse", at::kFloat, {n, s.Hq}, "[rows, n_q_heads]");
    x.max_chunk = int_of(a[10], "max_chunk");
    x.max_ctx = int_of(a[11], "max_ctx");
    x.scale = float_of(a[12]);
    if (n == 0) return;
    const OnDevice on(s, a[13]);
    call("cb_chunk_attn", [&] { return g_lib.chunk_attn(c, &x, on.stream); });
}
// The outputs of log probabilities: a dictionary with logprobs and entropy, and the alternatives where there are any.
void likely_of(const Shape& s, PyObject* res, PyObject* top, bool accept, int64_t n, cb_logprobs_args* x) {
    x->top_k = int_of(top, "top_k");
    if (x->top_k < 0 || x->top_k > CB_MAX_TOP) refuse_shape("top_k", "between 0 and 32");
    const char* text = accept ? "[batch, max_depth + 1], alternatives [batch, max_depth + 1, top_k]" : "[outputs], alternatives [outputs, top_k]";
    auto get = [&](const char* name, at::ScalarType t, bool many) -> void* {
        Ref r(PyMapping_GetItemString(res, name));
        if (accept) return many ? arg(s, r.o, name, t, {s.B, s.Dmax + 1, x->top_k}, text).p : arg(s, r.o, name, t, {s.B, s.Dmax + 1}, text).p;
        return many ? arg(s, r.o, name, t, {n, x->top_k}, text).p : arg(s, r.o, name, t, {n}, text).p;
    };
    x->logprobs = static_cast<float*>(get("logprobs", at::kFloat, false));
    x->entropy = static_cast<float*>(get("entropy", at::kFloat, false));
    if (x->top_k == 0) return;
    x->top_ids = static_cast<int32_t*>(get("top_ids", at::kInt, true));
    x->top_logprobs = static_cast<float*>(get("top_logprobs", at::kFloat, true));
}
int32_t logits_dtype_of(const Shape& s, const at::Tensor& t) {
    if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) refuse("logits must be float32 or bfloat16");
    if (!t.is_cuda() || t.get_device() != s.device) refuse_shape("logits", "on the context's device");
    return t.scalar_type() == at::kFloat ? CB_DTYPE_F32 : CB_DTYPE_BF16;
}
// handle, shape, logits, tokens, rows, top_k, res, stream
void do_logprobs(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    const Shape s = shape_of(a[1]);
    cb_logprobs_args x = {};
    const at::Tensor& t = tensor_of(a[2]);
    x.logits_dtype = logits_dtype_of(s, t);
    if (t.dim() != 2 || t.size(1) != s.V || t.size(0) > INT32_MAX || (t.numel() > 0 && s.V > 1 && t.stride(1) != 1))
        refuse_shape("logits", "[rows, vocab], contiguous within a row");
    x.n_rows = (int32_t)t.size(0);
    x.logits = t.data_ptr();
    x.logits_row_stride = t.size(0) > 1 ? t.stride(0) : s.V;
    const int64_t n = a[4] != Py_None ? tensor_of(a[4]).numel() : (a[3] != Py_None ? tensor_of(a[3]).numel() : t.size(0));
    if (n > INT32_MAX || (a[4] == Py_None && n > t.size(0))) refuse_shape("tokens", "at most one per row of logits");
    x.n_out = (int32_t)n;
    x.tokens = opt<int32_t>(s, a[3], "tokens", at::kInt, {n}, "[outputs]");
    x.rows = opt<int32_t>(s, a[4], "rows", at::kInt, {n}, "[outputs]");
    likely_of(s, a[6], a[5], false, n, &x);
    if (n == 0) return;
    if (t.size(0) == 0) refuse_shape("logits", "of at least one row");
    const OnDevice on(s, a[7]);
    call("cb_logprobs", [&] { return g_lib.logprobs(c, &x, on.stream); });
}
// handle, shape, logits, accepted, top_k, res, stream
void do_accept_logprobs(PyObject* const* a) {
    cb_ctx* c = ctx_of(a[0]);
    const Shape s = shape_of(a[1]);
    cb_logprobs_args x = {};
    const at::Tensor& t = tensor_of(a[2]);
    logits_dtype_of(s, t);
    x.logits = logits_of(a[2], &x.logits_dtype, &x.logits_row_stride);
    if (t.size(0) != s.B || t.size(1) != s.T || t.size(2) != s.V) refuse_shape("logits", "[batch, max_nodes, vocab]");
    Ref nodes(PyObject_GetItem(a[3], s_accept_nodes)), toks(PyObject_GetItem(a[3], s_out_tokens));
    const int32_t* an = static_cast<int32_t*>(arg(s, nodes.o, "accept_nodes", at::kInt, {s.B, s.Dmax}, "[batch, max_depth]").p);
    const int32_t* ot = static_cast<int32_t*>(arg(s, toks.o, "out_tokens", at::kInt, {s.B, s.Dmax + 1}, "[batch, max_depth + 1]").p);
    likely_of(s, a[5], a[4], true, 0, &x);
    const OnDevice on(s, a[6]);
    call("cb_accept_logprobs", [&] { return g_lib.accept_logprobs(c, an, ot, &x, on.stream); });
}

// set_library(CachebackError, {name: address})
PyObject* set_library(PyObject*, PyObject* args) {
    PyObject *err, *addr;
    if (!PyArg_ParseTuple(args, "OO!", &err, &PyDict_Type, &addr)) return nullptr;
    auto take = [&](const char* name, auto* f) {
        PyObject* o = PyDict_GetItemString(addr, name);
        if (!o) { PyErr_Format(PyExc_KeyError, "%s", name); return false; }
        void* p = PyLong_AsVoidPtr(o);
        if (!p) { if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "no address for %s", name); return false; }
        *f = reinterpret_cast<std::remove_reference_t<decltype(*f)>>(p);
        return true;
    };
    Library l;
    if (!(take("cb_reset", &l.reset) && take("cb_update", &l.update) && take("cb_update_bulk", &l.update_bulk) && take("cb_draft_tree", &l.draft_tree) &&
          take("cb_update_draft_tree", &l.update_draft_tree) && take("cb_tree_attn", &l.tree_attn) && take("cb_accept", &l.accept) &&
          take("cb_accept_update_draft_tree", &l.accept_update_draft_tree) && take("cb_kv_commit", &l.kv_commit) && take("cb_chunk_append", &l.chunk_append) &&
          take("cb_chunk_attn", &l.chunk_attn) && take("cb_tree_rope", &l.tree_rope) && take("cb_logprobs", &l.logprobs) &&
          take("cb_accept_logprobs", &l.accept_logprobs) && take("cb_status_str", &l.status_str)))
        return nullptr;
    g_lib = l;
    Py_INCREF(err);
    Py_XSETREF(g_error, err);
    Py_RETURN_NONE;
}

#define CB_FAST(name, n, f) {name, (PyCFunction)(void (*)(void))(entry<n, f>), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    {"set_library", set_library, METH_VARARGS, nullptr},
    CB_FAST("reset", 3, do_reset), CB_FAST("update", 5, do_update<false>), CB_FAST("update_bulk", 5, do_update<true>), CB_FAST("draft_tree", 5, do_draft),
    CB_FAST("update_draft_tree", 6, do_update_draft), CB_FAST("accept", 6, do_accept), CB_FAST("accept_update_draft_tree", 8, do_accept_update_draft),
    CB_FAST("tree_attn", 15, do_attn), CB_FAST("kv_commit", 10, do_kv_commit), CB_FAST("chunk_append", 17, do_chunk_append),
    CB_FAST("tree_rope", 16, do_tree_rope), CB_FAST("chunk_attn", 14, do_chunk_attn), CB_FAST("logprobs", 8, do_logprobs),
    CB_FAST("accept_logprobs", 7, do_accept_logprobs), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) {
    struct { PyObject** at; const char* text; } names[] = {
        {&s_cuda_stream, "cuda_stream"}, {&s_tokens, "tokens"}, {&s_parent, "parent"}, {&s_depth, "depth"}, {&s_mask, "mask"}, {&s_n_nodes, "n_nodes"},
        {&s_n_accept, "n_accept"}, {&s_accept_nodes, "accept_nodes"}, {&s_out_tokens, "out_tokens"}, {&s_target_ids, "target_ids"}};
    for (auto& n : names)
        if (!(*n.at = PyUnicode_InternFromString(n.text))) return nullptr;
    return PyModule_Create(&g_module);
}
