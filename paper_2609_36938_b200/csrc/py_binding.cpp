// Native half of binding.py: takes the tensors of a call apart, allocates its outputs and calls the C entry point.
//
// A pass over a short history is four calls of five or six launches; marshalling them in Python (some twenty tensor and stream
// queries and a ctypes conversion per call) took 65 to 75 us of host time per pass, longer than the kernels.  Positional
// arguments in the order of binding.py's signatures; checks and errors are the same, and so is the absence of any fallback.
#include <Python.h>

#include <dlfcn.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <initializer_list>
#include <string>
#include <vector>

#include "../../include/janus.h"

// read by build.py: the library is built again when torch or the interpreter is another
extern "C" __attribute__((used, visibility("default"))) const char janus_native_mark[] = JANUS_NATIVE_MARK;

namespace {

// ---- state set once by init(): the C entry points and the Python objects the calls need
struct Api {
    decltype(&janus_indexer_scores) indexer_scores;
    decltype(&janus_topk) topk;
    decltype(&janus_indexer_topk_workspace_size) indexer_topk_workspace_size;
    decltype(&janus_indexer_topk) indexer_topk;
    decltype(&janus_page_demand) page_demand;
    decltype(&janus_page_union) page_union;
    decltype(&janus_sparse_attn_prefill) sparse_attn_prefill;
    decltype(&janus_topk_entries) topk_entries;
    decltype(&janus_entry_pool_scores) entry_pool_scores;
    decltype(&janus_entry_expand) entry_expand;
    decltype(&janus_indexer_scores_batch) indexer_scores_batch;
    decltype(&janus_topk_batch) topk_batch;
    decltype(&janus_page_demand_batch) page_demand_batch;
    decltype(&janus_sparse_attn_decode) sparse_attn_decode;
    decltype(&janus_batch_plan) batch_plan;
    decltype(&janus_rope) rope;
    decltype(&janus_rope_append) rope_append;
    decltype(&janus_attn_decode_shared_workspace_size) attn_decode_shared_workspace_size;
    decltype(&janus_attn_decode_shared) attn_decode_shared;
    decltype(&janus_last_cuda_error) last_cuda_error;
} api;
PyObject* janus_error = nullptr;        // exception class
PyObject* status_tensor_fn = nullptr;   // binding.dev_status_tensor
auto& status_words = *new std::vector<at::Tensor>;   // by device, as binding.dev_status_tensor made them; never destroyed (outlives CUDA's own teardown)
PyObject *key_bitmap, *key_pages, *key_runs, *key_counts, *key_miss_pages, *key_miss_runs;
PyObject *key_row_offsets, *key_kv_lens, *key_table_offsets, *key_page_tables, *key_row_sessions, *key_positions, *key_slots, *key_key_rows;

struct PyError {};                      // a Python exception is set
[[noreturn]] void fail(PyObject* type, const std::string& what) {
    PyErr_SetString(type, what.c_str());
    throw PyError{};
}

// ---- arguments
const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a tensor");
    return THPVariable_Unpack(o);
}
void* ptr(const at::Tensor& t) {
    if (!t.is_cuda()) fail(janus_error, "expected a CUDA tensor (the library takes device pointers)");
    return t.data_ptr();
}
void* ptr_or_null(PyObject* o) { return o == Py_None ? nullptr : ptr(tensor(o)); }
int64_t integer(PyObject* o) {
    if (PyLong_CheckExact(o)) {
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) throw PyError{};
        return v;
    }
    PyObject* n = PyNumber_Long(o);
    if (n == nullptr) throw PyError{};
    const long long v = PyLong_AsLongLong(n);
    Py_DECREF(n);
    if (v == -1 && PyErr_Occurred()) throw PyError{};
    return v;
}
// A size of something this call allocates: whole numbers only, as for any tensor's shape.
int64_t size(PyObject* o) {
    PyObject* n = PyNumber_Index(o);
    if (n == nullptr) throw PyError{};
    const long long v = PyLong_AsLongLong(n);
    Py_DECREF(n);
    if (v == -1 && PyErr_Occurred()) throw PyError{};
    return v;
}
double number(PyObject* o) {
    PyObject* f = PyNumber_Float(o);
    if (f == nullptr) throw PyError{};
    const double v = PyFloat_AS_DOUBLE(f);
    Py_DECREF(f);
    return v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PyError{};
    return v != 0;
}
void want_dims(const at::Tensor& t, int64_t n, const char* name) {
    if (t.dim() != n) fail(PyExc_ValueError, std::string(name) + " must have " + std::to_string(n) + " dimensions, not " + std::to_string(t.dim()));
}
const at::Tensor& item(PyObject* dict, PyObject* key, at::Tensor& hold) {
    PyObject* o = PyObject_GetItem(dict, key);
    if (o == nullptr) throw PyError{};
    if (!THPVariable_Check(o)) {
        Py_DECREF(o);
        fail(PyExc_TypeError, "expected a tensor");
    }
    hold = THPVariable_Unpack(o);
    Py_DECREF(o);
    return hold;
}

// ---- what every call passes along
int32_t* status_word() {
    const int dev = c10::cuda::current_device();
    if (static_cast<size_t>(dev) >= status_words.size()) status_words.resize(dev + 1);
    if (!status_words[dev].defined()) {
        PyObject* t = PyObject_CallNoArgs(status_tensor_fn);
        if (t == nullptr) throw PyError{};
        status_words[dev] = THPVariable_Unpack(t);
        Py_DECREF(t);
    }
    return static_cast<int32_t*>(status_words[dev].data_ptr());
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

at::Tensor make(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) { return at::empty(shape, like.options().dtype(type)); }
PyObject* wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }
PyObject* none() { return Py_NewRef(Py_None); }

PyObject* triple(PyObject* a, const at::Tensor& b, const at::Tensor& c) {      // b, c undefined -> None; steals a
    PyObject* t = PyTuple_New(3);
    PyTuple_SET_ITEM(t, 0, a);
    PyTuple_SET_ITEM(t, 1, b.defined() ? wrap(b) : none());
    PyTuple_SET_ITEM(t, 2, c.defined() ? wrap(c) : none());
    return t;
}

void check(int rc, const char* what) {
    if (rc == JANUS_OK) return;
    static const char* names[] = {"", "JANUS_ERR_INVALID_ARG", "JANUS_ERR_UNSUPPORTED", "JANUS_ERR_WORKSPACE_TOO_SMALL", "JANUS_ERR_CUDA"};
    std::string text = std::string(what) + " failed: " + (rc >= 1 && rc <= 4 ? names[rc] : std::to_string(rc));
    if (rc == JANUS_ERR_CUDA) text += " (cudaError " + std::to_string(api.last_cuda_error()) + ")";
    fail(janus_error, text);
}

// Calls a C entry point without the GIL (a full launch queue blocks).
template <class F, class... A>
void call(const char* what, F f, A... a) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(a...);
    Py_END_ALLOW_THREADS
    check(rc, what);
}

int idx_dtype_code(const at::Tensor& t) {
    if (t.scalar_type() == at::kBFloat16) return JANUS_DTYPE_BF16;
    if (t.scalar_type() == at::kByte || t.scalar_type() == at::kFloat8_e4m3fn) return JANUS_DTYPE_FP8_E4M3;
    fail(janus_error, std::string("indexer operands must be bfloat16 or E4M3 bytes, got ") + c10::toString(t.scalar_type()));
}
struct IdxDtypes {
    int code;
    int64_t k_stride;
};
IdxDtypes idx_dtypes(const at::Tensor& q, const at::Tensor& k, bool fp4) {
    const int code = idx_dtype_code(q);
    if (fp4) {
        if (code != JANUS_DTYPE_FP8_E4M3 || k.scalar_type() != at::kByte) fail(janus_error, "FP4 keys are uint8 (two per byte) and go with E4M3 queries");
        return {JANUS_DTYPE_FP8_Q_FP4_K, k.stride(0) * 2};
    }
    if (idx_dtype_code(k) != code) fail(janus_error, "q_idx and k_idx must share a dtype");
    return {code, k.stride(0)};
}
int64_t q_scale_stride(PyObject* q_scale, int64_t H) { return q_scale != Py_None && tensor(q_scale).dim() == 2 ? H : 0; }
int i32(int64_t v) { return static_cast<int>(v); }
template <class T>
T* as(void* p) { return static_cast<T*>(p); }

// ---- the calls: (arguments in the order of binding.py) -> new reference
using Args = PyObject* const*;

PyObject* indexer_scores(Args a) {
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]);
    want_dims(q, 3, "q_idx");
    const int64_t M = q.size(0), H = q.size(1), D = q.size(2), n_keys = k.size(0);
    const IdxDtypes dt = idx_dtypes(q, k, truth(a[10]));
    at::Tensor scores = a[9] == Py_None ? make({M, (n_keys + 31) / 32 * 32}, at::kFloat, q) : tensor(a[9]);
    call("janus_indexer_scores", api.indexer_scores, ptr(q), q.stride(0), ptr(k), dt.k_stride, as<const float>(ptr_or_null(a[2])),
         as<const float>(ptr_or_null(a[3])), q_scale_stride(a[3], H), as<const float>(ptr_or_null(a[4])), as<const float>(ptr_or_null(a[5])),
         as<const float>(ptr_or_null(a[6])), i32(M), i32(H), i32(D), n_keys, integer(a[7]), i32(truth(a[8])), dt.code, as<float>(ptr(scores)),
         scores.stride(0), nullptr, size_t(0), status_word(), stream());
    return a[9] == Py_None ? wrap(scores) : Py_NewRef(a[9]);
}

PyObject* topk(Args a) {
    const at::Tensor& scores = tensor(a[0]);
    const int64_t M = scores.size(0), k = a[7] == Py_None ? size(a[2]) : integer(a[2]);
    at::Tensor idx = a[7] == Py_None ? make({M, k}, at::kInt, scores) : tensor(a[7]), count, kth;
    if (truth(a[5])) count = make({M}, at::kInt, scores);
    if (truth(a[6])) kth = make({M}, at::kFloat, scores);
    call("janus_topk", api.topk, as<const float>(ptr(scores)), scores.stride(0), i32(M), integer(a[1]), integer(a[3]), i32(truth(a[4])), i32(k),
         as<int32_t>(ptr(idx)), as<int32_t>(count.defined() ? ptr(count) : nullptr), as<float>(kth.defined() ? ptr(kth) : nullptr), nullptr, size_t(0),
         status_word(), stream());
    return triple(a[7] == Py_None ? wrap(idx) : Py_NewRef(a[7]), count, kth);
}

PyObject* indexer_topk(Args a) {
    const at::Tensor &q = tensor(a[0]), &k_idx = tensor(a[1]);
    want_dims(q, 3, "q_idx");
    const int64_t M = q.size(0), H = q.size(1), D = q.size(2), n_keys = k_idx.size(0), k = a[13] == Py_None ? size(a[3]) : integer(a[3]), q_pos0 = integer(a[8]);
    const IdxDtypes dt = idx_dtypes(q, k_idx, truth(a[14]));
    const int causal = i32(truth(a[9]));
    const size_t need = api.indexer_topk_workspace_size(i32(M), i32(H), i32(D), n_keys, q_pos0, causal, dt.code, i32(k));
    at::Tensor ws;
    if (a[12] != Py_None) ws = tensor(a[12]);
    if (!ws.defined() || ws.numel() < static_cast<int64_t>(need)) ws = make({static_cast<int64_t>(need > 16 ? need : 16)}, at::kByte, q);
    at::Tensor idx, count, kth;
    if (a[13] == Py_None) {
        idx = make({M, k}, at::kInt, q);
    } else {
        idx = tensor(a[13]);
        if (idx.dim() != 2 || idx.size(0) != M || idx.size(1) != k || number(a[3]) != static_cast<double>(k) || idx.scalar_type() != at::kInt || !idx.is_contiguous())
            fail(janus_error, "idx must be a contiguous [M, k] int32 tensor");
    }
    if (truth(a[10])) count = make({M}, at::kInt, q);
    if (truth(a[11])) kth = make({M}, at::kFloat, q);
    call("janus_indexer_topk", api.indexer_topk, ptr(q), q.stride(0), ptr(k_idx), dt.k_stride, as<const float>(ptr_or_null(a[2])),
         as<const float>(ptr_or_null(a[4])), q_scale_stride(a[4], H), as<const float>(ptr_or_null(a[5])), as<const float>(ptr_or_null(a[6])),
         as<const float>(ptr_or_null(a[7])), i32(M), i32(H), i32(D), n_keys, q_pos0, causal, dt.code, i32(k), as<int32_t>(ptr(idx)),
         as<int32_t>(count.defined() ? ptr(count) : nullptr), as<float>(kth.defined() ? ptr(kth) : nullptr), ptr(ws), static_cast<size_t>(ws.numel()),
         status_word(), stream());
    return triple(a[13] == Py_None ? wrap(idx) : Py_NewRef(a[13]), count, kth);
}

// Output buffers of a page-demand call: the dict of page_demand_buffers().
struct PageOut {
    at::Tensor bitmap, pages, runs, counts, miss_pages, miss_runs;
    int32_t *n_pages, *n_runs, *miss_p = nullptr, *n_miss = nullptr, *miss_r = nullptr, *n_miss_runs = nullptr;
    int64_t capacity;
    PageOut(PyObject* out, PyObject* cap, bool want_miss) {
        item(out, key_bitmap, bitmap);
        item(out, key_pages, pages);
        item(out, key_runs, runs);
        item(out, key_counts, counts);
        n_pages = as<int32_t>(counts.data_ptr());
        n_runs = n_pages + 1;
        const int has = want_miss ? PySequence_Contains(out, key_miss_pages) : 0;
        if (has < 0) throw PyError{};
        if (has) {
            miss_p = as<int32_t>(ptr(item(out, key_miss_pages, miss_pages)));
            n_miss = n_pages + 2;
            miss_r = as<int32_t>(ptr(item(out, key_miss_runs, miss_runs)));
            n_miss_runs = n_pages + 3;
        }
        capacity = cap == Py_None ? pages.numel() : integer(cap);
    }
};

PyObject* page_demand(Args a) {       // idx, demand_limit, page_size, page_table, n_phys_pages, predicted, capacity, want_miss, out
    const at::Tensor &idx = tensor(a[0]), &table = tensor(a[3]);
    want_dims(idx, 2, "idx");
    PageOut o(a[8], a[6], truth(a[7]));
    call("janus_page_demand", api.page_demand, as<const int32_t>(ptr(idx)), idx.size(0), i32(idx.size(1)), integer(a[1]), i32(integer(a[2])),
         as<const int32_t>(ptr(table)), table.numel(), integer(a[4]), as<const uint32_t>(ptr_or_null(a[5])), as<uint32_t>(ptr(o.bitmap)),
         as<int32_t>(ptr(o.pages)), o.n_pages, as<int32_t>(ptr(o.runs)), o.n_runs, o.miss_p, o.n_miss, o.miss_r, o.n_miss_runs, o.capacity, nullptr,
         size_t(0), status_word(), stream());
    return Py_NewRef(a[8]);
}

PyObject* page_demand_batch(Args a) { // idx, demand_limits, page_size, page_tables, table_offsets, n_phys_pages, predicted, capacity, want_miss, out
    const at::Tensor& idx = tensor(a[0]);
    want_dims(idx, 2, "idx");
    PageOut o(a[9], a[7], truth(a[8]));
    call("janus_page_demand_batch", api.page_demand_batch, as<const int32_t>(ptr(idx)), idx.size(0), i32(idx.size(1)),
         as<const int64_t>(ptr_or_null(a[1])), i32(integer(a[2])), as<const int32_t>(ptr_or_null(a[3])), as<const int64_t>(ptr_or_null(a[4])),
         integer(a[5]), as<const uint32_t>(ptr_or_null(a[6])), as<uint32_t>(ptr(o.bitmap)), as<int32_t>(ptr(o.pages)), o.n_pages,
         as<int32_t>(ptr(o.runs)), o.n_runs, o.miss_p, o.n_miss, o.miss_r, o.n_miss_runs, o.capacity, status_word(), stream());
    return Py_NewRef(a[9]);
}

PyObject* page_union(Args a) {        // dst, src, n_phys_pages
    call("janus_page_union", api.page_union, as<uint32_t>(ptr_or_null(a[0])), as<const uint32_t>(ptr_or_null(a[1])), integer(a[2]), stream());
    return Py_NewRef(a[0]);
}

// q, k_pool, v_pool, idx, page tables, table offsets (None: prefill), page_size, softmax_scale, d_v, want_lse, out
PyObject* sparse_attn(Args a) {
    const at::Tensor &q = tensor(a[0]), &kp = tensor(a[1]), &vp = tensor(a[2]), &idx = tensor(a[3]), &table = tensor(a[4]);
    want_dims(q, 3, "q");
    const bool batch = a[5] != Py_None;
    const int64_t M = q.size(0), H = q.size(1), d_qk = q.size(2), n_kv = kp.size(2), d_v = a[10] == Py_None ? size(a[8]) : integer(a[8]);
    at::Tensor out = a[10] == Py_None ? make({M, H, d_v}, at::kBFloat16, q) : tensor(a[10]), lse;
    if (truth(a[9])) lse = make({M, H}, at::kFloat, q);
    if (!batch && vp.data_ptr() != kp.data_ptr() && vp.strides() != kp.strides()) fail(janus_error, "k_pool and v_pool must share strides");
    float* lse_p = lse.defined() ? as<float>(ptr(lse)) : nullptr;
    if (batch)
        call("janus_sparse_attn_decode", api.sparse_attn_decode, ptr(q), i32(M), i32(H), i32(d_qk), ptr(kp), ptr(vp), kp.stride(0), kp.stride(1),
             kp.stride(2), i32(n_kv), i32(d_v), as<const int32_t>(ptr(idx)), i32(idx.size(1)), i32(integer(a[6])), as<const int32_t>(ptr(table)),
             as<const int64_t>(ptr_or_null(a[5])), static_cast<float>(number(a[7])), ptr(out), lse_p, status_word(), stream());
    else
        call("janus_sparse_attn_prefill", api.sparse_attn_prefill, ptr(q), i32(M), i32(H), i32(d_qk), ptr(kp), ptr(vp), kp.stride(0), kp.stride(1),
             kp.stride(2), i32(n_kv), i32(d_v), as<const int32_t>(ptr(idx)), i32(idx.size(1)), i32(integer(a[6])), as<const int32_t>(ptr(table)),
             table.numel(), static_cast<float>(number(a[7])), ptr(out), lse_p, nullptr, size_t(0), status_word(), stream());
    PyObject* t = PyTuple_New(2);
    PyTuple_SET_ITEM(t, 0, a[10] == Py_None ? wrap(out) : Py_NewRef(a[10]));
    PyTuple_SET_ITEM(t, 1, lse.defined() ? wrap(lse) : none());
    return t;
}

PyObject* topk_entries(Args a) {      // scores, n_entries, k, q_pos0, entry_size, want_count, want_kth
    const at::Tensor& scores = tensor(a[0]);
    const int64_t M = scores.size(0), k = size(a[2]);
    at::Tensor idx = make({M, k}, at::kInt, scores), count, kth;
    if (truth(a[5])) count = make({M}, at::kInt, scores);
    if (truth(a[6])) kth = make({M}, at::kFloat, scores);
    call("janus_topk_entries", api.topk_entries, as<const float>(ptr(scores)), scores.stride(0), i32(M), integer(a[1]), integer(a[3]),
         i32(integer(a[4])), i32(k), as<int32_t>(ptr(idx)), as<int32_t>(count.defined() ? ptr(count) : nullptr),
         as<float>(kth.defined() ? ptr(kth) : nullptr), status_word(), stream());
    return triple(wrap(idx), count, kth);
}

PyObject* entry_pool_scores(Args a) { // scores, n_keys, entry_size, q_pos0, causal
    const at::Tensor& scores = tensor(a[0]);
    const int64_t M = scores.size(0), n_keys = integer(a[1]), entry = size(a[2]);
    if (entry == 0) fail(PyExc_ZeroDivisionError, "entry_size is zero");
    const int64_t n_entries = (n_keys + entry - 1) / entry, ld = n_entries > 4 ? (n_entries + 3) / 4 * 4 : 4;
    at::Tensor out = make({M, ld}, at::kFloat, scores);
    call("janus_entry_pool_scores", api.entry_pool_scores, as<const float>(ptr(scores)), scores.stride(0), i32(M), n_keys, integer(a[3]),
         i32(truth(a[4])), i32(entry), as<float>(ptr(out)), ld, stream());
    return wrap(out);
}

PyObject* entry_expand(Args a) {      // idx_entries, q_pos0, entry_size
    const at::Tensor& e = tensor(a[0]);
    want_dims(e, 2, "idx_entries");
    const int64_t M = e.size(0), k_e = e.size(1), entry = size(a[2]);
    at::Tensor out = make({M, k_e * entry}, at::kInt, e);
    call("janus_entry_expand", api.entry_expand, as<const int32_t>(ptr(e)), i32(M), i32(k_e), i32(entry), integer(a[1]), as<int32_t>(ptr(out)), stream());
    return wrap(out);
}

PyObject* indexer_scores_batch(Args a) {      // q, k, w, key_offsets, max_keys, q_scale, k_scale, row_bias, col_bias, scores, keys_fp4
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]);
    want_dims(q, 3, "q_idx");
    const int64_t n = q.size(0), H = q.size(1), D = q.size(2), total = k.size(0);
    const bool fp4 = truth(a[10]);
    const int code = fp4 ? JANUS_DTYPE_FP8_Q_FP4_K : idx_dtype_code(q);
    at::Tensor scores = a[9] == Py_None ? make({total}, at::kFloat, q) : tensor(a[9]);
    call("janus_indexer_scores_batch", api.indexer_scores_batch, ptr(q), ptr(k), k.stride(0) * (fp4 ? 2 : 1), as<const float>(ptr_or_null(a[2])),
         as<const float>(ptr_or_null(a[5])), q_scale_stride(a[5], H), as<const float>(ptr_or_null(a[6])), as<const float>(ptr_or_null(a[7])),
         as<const float>(ptr_or_null(a[8])), i32(n), i32(H), i32(D), as<const int64_t>(ptr_or_null(a[3])), total, integer(a[4]), code,
         as<float>(ptr(scores)), status_word(), stream());
    return a[9] == Py_None ? wrap(scores) : Py_NewRef(a[9]);
}

PyObject* topk_batch(Args a) {        // scores, row_offsets, k, row_lengths, want_count, want_kth
    const at::Tensor &scores = tensor(a[0]), &off = tensor(a[1]);
    const int64_t n = off.numel() - 1, k = size(a[2]);
    at::Tensor idx = make({n, k}, at::kInt, scores), count, kth;
    if (truth(a[4])) count = make({n}, at::kInt, scores);
    if (truth(a[5])) kth = make({n}, at::kFloat, scores);
    call("janus_topk_batch", api.topk_batch, as<const float>(ptr(scores)), as<const int64_t>(ptr(off)), as<const int64_t>(ptr_or_null(a[3])), i32(n),
         i32(k), as<int32_t>(ptr(idx)), as<int32_t>(count.defined() ? ptr(count) : nullptr), as<float>(kth.defined() ? ptr(kth) : nullptr),
         status_word(), stream());
    return triple(wrap(idx), count, kth);
}

// ---- a step's plan, rotary positions and the cache, dense layers
void want(bool ok, const char* what) {
    if (!ok) fail(janus_error, what);
}
// One axis of the given type, elements adjacent, on the device; at least n of them (n < 0: any number).
template <class T>
T* vec(const at::Tensor& t, at::ScalarType type, int64_t n, const char* name) {
    if (t.scalar_type() != type || !t.is_contiguous() || t.numel() < n)
        fail(janus_error, std::string(name) + " must be a contiguous " + c10::toString(type) + " tensor" + (n >= 0 ? " of at least " + std::to_string(n) + " elements" : ""));
    return as<T>(ptr(t));
}
// Tensors whose memory lies on the current device, whose stream and status word the call takes.
void here(std::initializer_list<const at::Tensor*> list) {
    int current = -1;
    for (const at::Tensor* t : list)
        if (t->defined()) {
            if (!t->is_cuda()) fail(janus_error, "expected a CUDA tensor (the library takes device pointers)");
            if (current < 0) current = c10::cuda::current_device();      // (after the first look: without a device it is torch that fails)
            if (t->get_device() != current) fail(janus_error, "a tensor is not on the current device");
        }
}
int32_t* i32_vec(const at::Tensor& t, int64_t n, const char* name) { return vec<int32_t>(t, at::kInt, n, name); }
int64_t* i64_vec(const at::Tensor& t, int64_t n, const char* name) { return vec<int64_t>(t, at::kLong, n, name); }
at::Tensor optional(PyObject* o) { return o == Py_None ? at::Tensor() : tensor(o); }
// int arguments: what does not fit is refused, not cut
int small(PyObject* o, const char* name) {
    const int64_t v = size(o);
    if (v < INT32_MIN || v > INT32_MAX) fail(PyExc_OverflowError, std::string(name) + " is out of range");
    return static_cast<int>(v);
}

PyObject* batch_plan(Args a) {        // cached_lens, new_lens, block_tables, free_pages, page_size, n_phys_pages, max_rows, key_offsets, out
    const at::Tensor &cached = tensor(a[0]), &fresh = tensor(a[1]), &tables = tensor(a[2]), &free_pages = tensor(a[3]), key_offsets = optional(a[7]);
    want_dims(cached, 1, "cached_lens");
    want_dims(tables, 2, "block_tables");
    const int64_t n = cached.numel(), max_rows = size(a[6]);
    want(fresh.numel() == n && tables.size(0) == n, "cached_lens, new_lens and block_tables must agree in the number of sessions");
    want(tables.scalar_type() == at::kInt && (tables.size(1) <= 1 || tables.stride(1) == 1), "block_tables must be int32 with adjacent columns");
    at::Tensor row_offsets, kv_lens, table_offsets, page_tables, row_sessions, positions, slots, counts, key_rows;
    item(a[8], key_row_offsets, row_offsets); item(a[8], key_kv_lens, kv_lens); item(a[8], key_table_offsets, table_offsets);
    item(a[8], key_page_tables, page_tables); item(a[8], key_row_sessions, row_sessions); item(a[8], key_positions, positions);
    item(a[8], key_slots, slots); item(a[8], key_counts, counts);
    if (key_offsets.defined()) item(a[8], key_key_rows, key_rows);
    want(n <= INT32_MAX, "too many sessions");
    auto of = [](const at::Tensor& t, int64_t least, const char* name) { return t.defined() ? i64_vec(t, least, name) : nullptr; };
    const int64_t *cached_p = of(cached, n, "cached_lens"), *fresh_p = of(fresh, n, "new_lens"), *key_offsets_p = of(key_offsets, n, "key_offsets");
    int64_t *row_offsets_p = of(row_offsets, n + 1, "row_offsets"), *kv_lens_p = of(kv_lens, n, "kv_lens"), *table_offsets_p = of(table_offsets, n + 1, "table_offsets");
    int64_t *positions_p = of(positions, max_rows, "positions"), *slots_p = of(slots, max_rows, "slots"), *key_rows_p = of(key_rows, max_rows, "key_rows");
    int64_t* counts_p = of(counts, 3, "counts");
    const int32_t* free_p = i32_vec(free_pages, -1, "free_pages");
    int32_t *page_tables_p = i32_vec(page_tables, -1, "page_tables"), *row_sessions_p = i32_vec(row_sessions, max_rows, "row_sessions");
    here({&cached, &fresh, &tables, &free_pages, &key_offsets, &row_offsets, &kv_lens, &table_offsets, &page_tables, &row_sessions, &positions, &slots, &counts, &key_rows});
    call("janus_batch_plan", api.batch_plan, cached_p, fresh_p, i32(n), small(a[4], "page_size"), as<int32_t>(ptr(tables)),
         n > 1 ? tables.stride(0) : tables.size(1), tables.size(1), free_p, free_pages.numel(), size(a[5]), key_offsets_p, row_offsets_p, kv_lens_p, table_offsets_p,
         page_tables_p, page_tables.numel(), row_sessions_p, positions_p, slots_p, key_rows_p, max_rows, counts_p, status_word(), stream());
    return Py_NewRef(a[8]);
}

int elem_code(const at::Tensor& t, const char* name) {
    switch (t.scalar_type()) {
        case at::kBFloat16: return JANUS_ELEM_BF16;
        case at::kHalf: return JANUS_ELEM_FP16;
        case at::kFloat: return JANUS_ELEM_FP32;
        default: fail(janus_error, std::string(name) + " must be bfloat16, float16 or float32, got " + c10::toString(t.scalar_type()));
    }
}
void rows_of_heads(const at::Tensor& t, const char* name) {
    want_dims(t, 3, name);
    if (t.size(2) > 1 && t.stride(2) != 1) fail(janus_error, std::string(name) + ": the dims of a head must be adjacent");
}
// A tensor with `like`'s shape and type, its dims of a head adjacent.
bool same_form(const at::Tensor& t, const at::Tensor& like) { return t.sizes() == like.sizes() && t.scalar_type() == like.scalar_type(); }

PyObject* rope(Args a) {              // x, positions, freqs, rot_offset, interleaved, scale, inverse, out
    const at::Tensor &x = tensor(a[0]), &positions = tensor(a[1]), &freqs = tensor(a[2]);
    rows_of_heads(x, "x");
    const int type = elem_code(x, "x");
    at::Tensor out = a[7] == Py_None ? make(x.sizes(), x.scalar_type(), x) : tensor(a[7]);
    rows_of_heads(out, "out");
    want(same_form(out, x), "out must have x's shape and type");
    const int64_t *positions_p = i64_vec(positions, x.size(0), "positions"), *freqs_p = i64_vec(freqs, 1, "freqs");
    here({&x, &positions, &freqs, &out});
    call("janus_rope", api.rope, ptr(x), x.stride(0), x.stride(1), x.size(0), i32(x.size(1)), i32(x.size(2)), positions_p, reinterpret_cast<const uint64_t*>(freqs_p), small(a[3], "rot_offset"), i32(2 * freqs.numel()), i32(truth(a[4])), static_cast<float>(number(a[5])),
         i32(truth(a[6])), type, ptr(out), out.stride(0), out.stride(1), stream());
    return a[7] == Py_None ? wrap(out) : Py_NewRef(a[7]);
}

void bf16(const at::Tensor& t, const char* name) {
    if (t.scalar_type() != at::kBFloat16) fail(janus_error, std::string(name) + " must be bfloat16, got " + c10::toString(t.scalar_type()));
}
void pool_of_rows(const at::Tensor& t, const char* name) {
    want_dims(t, 4, name);
    bf16(t, name);
    if (t.size(3) > 1 && t.stride(3) != 1) fail(janus_error, std::string(name) + ": the dims of a row must be adjacent");
}

// k, v, positions, slots, freqs, k_pool, v_pool, rot_offset, interleaved, scale, q, q_out
PyObject* rope_append(Args a) {
    const at::Tensor &k = tensor(a[0]), &positions = tensor(a[2]), &slots = tensor(a[3]), &freqs = tensor(a[4]), &kp = tensor(a[5]);
    const at::Tensor v = optional(a[1]), vp = optional(a[6]), q = optional(a[10]);
    rows_of_heads(k, "k");
    bf16(k, "k");
    pool_of_rows(kp, "k_pool");
    want(v.defined() == vp.defined(), "v and v_pool go together");
    want(kp.size(2) == k.size(1) && kp.size(3) == k.size(2), "k and k_pool must agree in heads and dims");
    const int64_t T = k.size(0), d_qk = k.size(2);
    if (v.defined()) {
        rows_of_heads(v, "v");
        bf16(v, "v");
        pool_of_rows(vp, "v_pool");
        want(v.size(0) == T && v.size(1) == k.size(1), "k and v must agree in rows and heads");
        want(vp.size(0) == kp.size(0) && vp.size(1) == kp.size(1) && vp.size(2) == v.size(1) && vp.size(3) == v.size(2), "v_pool must have k_pool's pages and v's heads and dims");
    }
    at::Tensor q_out;
    if (q.defined()) {
        rows_of_heads(q, "q");
        bf16(q, "q");
        want(q.size(0) == T && q.size(2) == d_qk, "q and k must agree in rows and dims");
        q_out = a[11] == Py_None ? make(q.sizes(), at::kBFloat16, q) : tensor(a[11]);
        rows_of_heads(q_out, "q_out");
        want(same_form(q_out, q), "q_out must have q's shape and type");
    } else {
        want(a[11] == Py_None, "q_out goes with q");
    }
    const int64_t *positions_p = i64_vec(positions, T, "positions"), *slots_p = i64_vec(slots, T, "slots"), *freqs_p = i64_vec(freqs, 1, "freqs");
    here({&k, &v, &positions, &slots, &freqs, &kp, &vp, &q, &q_out});
    auto at_ = [](const at::Tensor& t) { return t.defined() ? ptr(t) : nullptr; };
    auto st = [](const at::Tensor& t, int d) { return t.defined() ? t.stride(d) : int64_t(0); };
    call("janus_rope_append", api.rope_append, at_(q), st(q, 0), st(q, 1), q.defined() ? i32(q.size(1)) : 0, ptr(k), k.stride(0), k.stride(1), i32(k.size(1)),
         i32(d_qk), at_(v), st(v, 0), st(v, 1), v.defined() ? i32(v.size(2)) : 0, T, positions_p, slots_p,
         reinterpret_cast<const uint64_t*>(freqs_p), small(a[7], "rot_offset"), i32(2 * freqs.numel()), i32(truth(a[8])), static_cast<float>(number(a[9])),
         at_(q_out), st(q_out, 0), st(q_out, 1), ptr(kp), kp.stride(0), kp.stride(1), kp.stride(2), at_(vp), st(vp, 0), st(vp, 1), st(vp, 2), i32(kp.size(1)),
         kp.size(0), status_word(), stream());
    if (!q.defined()) return none();
    return a[11] == Py_None ? wrap(q_out) : Py_NewRef(a[11]);
}

// q, k_pool, v_pool, prefix_table, prefix_len, page_tables, table_offsets, kv_lens, max_len, page_size, softmax_scale, d_v, want_lse, out, workspace
PyObject* attn_decode_shared(Args a) {
    const at::Tensor &q = tensor(a[0]), &kp = tensor(a[1]), &vp = tensor(a[2]), &lens = tensor(a[7]);
    const at::Tensor prefix = optional(a[3]), tables = optional(a[5]), offsets = optional(a[6]);
    want_dims(q, 3, "q");
    bf16(q, "q");
    pool_of_rows(kp, "k_pool");
    pool_of_rows(vp, "v_pool");
    const int64_t n = q.size(0), H = q.size(1), d_qk = q.size(2), n_kv = kp.size(2), d_v = size(a[11]), prefix_len = size(a[4]), max_len = size(a[8]);
    const int page = small(a[9], "page_size");
    want(q.is_contiguous(), "q must be contiguous");
    want(kp.size(1) == page && vp.size(1) == page && vp.size(0) == kp.size(0) && vp.size(2) == n_kv, "the pools must be [pages, page_size, kv heads, dims], both of the same pages");
    want(kp.size(3) == d_qk && vp.size(3) >= d_v && d_v > 0, "the rows of the pools are shorter than the heads");
    want(prefix_len >= 0 && page > 0, "prefix_len must not be negative, page_size is positive");
    if (prefix_len > 0 && (!prefix.defined() || prefix.numel() < (prefix_len + page - 1) / page)) fail(janus_error, "prefix_table must cover prefix_len tokens");
    at::Tensor out = a[13] == Py_None ? make({n, H, d_v}, at::kBFloat16, q) : tensor(a[13]), lse;
    want(out.sizes() == at::IntArrayRef({n, H, d_v}) && out.scalar_type() == at::kBFloat16 && out.is_contiguous(), "out must be a contiguous [B, H_q, d_v] bfloat16 tensor");
    if (truth(a[12])) lse = make({n, H}, at::kFloat, q);
    const size_t need = api.attn_decode_shared_workspace_size(i32(n), i32(H), i32(d_qk), i32(n_kv), i32(d_v), page, prefix_len, max_len);
    at::Tensor ws = optional(a[14]);
    if (ws.defined()) want(ws.scalar_type() == at::kByte && ws.is_contiguous(), "workspace must be a contiguous uint8 tensor");
    if (!ws.defined() || ws.numel() < static_cast<int64_t>(need)) ws = make({static_cast<int64_t>(need > 16 ? need : 16)}, at::kByte, q);
    const int32_t *prefix_p = prefix.defined() ? i32_vec(prefix, -1, "prefix_table") : nullptr, *tables_p = tables.defined() ? i32_vec(tables, -1, "page_tables") : nullptr;
    const int64_t *offsets_p = offsets.defined() ? i64_vec(offsets, n + 1, "table_offsets") : nullptr, *lens_p = i64_vec(lens, n, "kv_lens");
    here({&q, &kp, &vp, &lens, &prefix, &tables, &offsets, &out, &ws});
    call("janus_attn_decode_shared", api.attn_decode_shared, ptr(q), i32(n), i32(H), i32(d_qk), ptr(kp), kp.stride(0), kp.stride(1), kp.stride(2), ptr(vp), vp.stride(0),
         vp.stride(1), vp.stride(2), i32(n_kv), i32(d_v), page, kp.size(0), prefix_p, prefix_len, tables_p, offsets_p,
         lens_p, max_len, static_cast<float>(number(a[10])), ptr(out), lse.defined() ? as<float>(ptr(lse)) : nullptr, ptr(ws),
         static_cast<size_t>(ws.numel()), status_word(), stream());
    PyObject* t = PyTuple_New(2);
    PyTuple_SET_ITEM(t, 0, a[13] == Py_None ? wrap(out) : Py_NewRef(a[13]));
    PyTuple_SET_ITEM(t, 1, lse.defined() ? wrap(lse) : none());
    return t;
}

// ---- module
template <PyObject* (*F)(Args), int N>
PyObject* entry(PyObject*, Args args, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const PyError&) {
    } catch (...) {      // torch's own exceptions by their own names: out of memory, a dimension that is not there
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

PyObject* init(PyObject*, Args args, Py_ssize_t n) {      // path of libjanus.so, exception class, dev_status_tensor
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "init(path, error, dev_status_tensor)");
        return nullptr;
    }
    const char* path = PyUnicode_AsUTF8(args[0]);
    if (path == nullptr) return nullptr;
    void* lib = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (lib == nullptr) {
        PyErr_SetString(args[1], dlerror());
        return nullptr;
    }
    bool ok = true;
    auto find = [&](auto& f, const char* name) {
        f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(dlsym(lib, name));
        ok = ok && f != nullptr;
    };
    find(api.indexer_scores, "janus_indexer_scores");
    find(api.topk, "janus_topk");
    find(api.indexer_topk_workspace_size, "janus_indexer_topk_workspace_size");
    find(api.indexer_topk, "janus_indexer_topk");
    find(api.page_demand, "janus_page_demand");
    find(api.page_union, "janus_page_union");
    find(api.sparse_attn_prefill, "janus_sparse_attn_prefill");
    find(api.topk_entries, "janus_topk_entries");
    find(api.entry_pool_scores, "janus_entry_pool_scores");
    find(api.entry_expand, "janus_entry_expand");
    find(api.indexer_scores_batch, "janus_indexer_scores_batch");
    find(api.topk_batch, "janus_topk_batch");
    find(api.page_demand_batch, "janus_page_demand_batch");
    find(api.sparse_attn_decode, "janus_sparse_attn_decode");
    find(api.batch_plan, "janus_batch_plan");
    find(api.rope, "janus_rope");
    find(api.rope_append, "janus_rope_append");
    find(api.attn_decode_shared_workspace_size, "janus_attn_decode_shared_workspace_size");
    find(api.attn_decode_shared, "janus_attn_decode_shared");
    find(api.last_cuda_error, "janus_last_cuda_error");
    if (!ok) {
        PyErr_SetString(args[1], "libjanus.so lacks an entry point");
        return nullptr;
    }
    janus_error = Py_NewRef(args[1]);
    status_tensor_fn = Py_NewRef(args[2]);
    return Py_NewRef(Py_None);
}

#define JANUS_METHOD(name, n) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<&name, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"init", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&init)), METH_FASTCALL, nullptr},
    JANUS_METHOD(indexer_scores, 11),
    JANUS_METHOD(topk, 8),
    JANUS_METHOD(indexer_topk, 15),
    JANUS_METHOD(page_demand, 9),
    JANUS_METHOD(page_demand_batch, 10),
    JANUS_METHOD(page_union, 3),
    JANUS_METHOD(sparse_attn, 11),
    JANUS_METHOD(topk_entries, 7),
    JANUS_METHOD(entry_pool_scores, 5),
    JANUS_METHOD(entry_expand, 3),
    JANUS_METHOD(indexer_scores_batch, 11),
    JANUS_METHOD(topk_batch, 6),
    JANUS_METHOD(batch_plan, 9),
    JANUS_METHOD(rope, 8),
    JANUS_METHOD(rope_append, 12),
    JANUS_METHOD(attn_decode_shared, 15),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
    key_bitmap = PyUnicode_InternFromString("bitmap");
    key_pages = PyUnicode_InternFromString("pages");
    key_runs = PyUnicode_InternFromString("runs");
    key_counts = PyUnicode_InternFromString("counts");
    key_miss_pages = PyUnicode_InternFromString("miss_pages");
    key_miss_runs = PyUnicode_InternFromString("miss_runs");
    key_row_offsets = PyUnicode_InternFromString("row_offsets");
    key_kv_lens = PyUnicode_InternFromString("kv_lens");
    key_table_offsets = PyUnicode_InternFromString("table_offsets");
    key_page_tables = PyUnicode_InternFromString("page_tables");
    key_row_sessions = PyUnicode_InternFromString("row_sessions");
    key_positions = PyUnicode_InternFromString("positions");
    key_slots = PyUnicode_InternFromString("slots");
    key_key_rows = PyUnicode_InternFromString("key_rows");
    return PyModule_Create(&module);
}
