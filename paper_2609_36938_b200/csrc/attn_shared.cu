// Dense attention of one query token per session over a shared prefix and each session's own tokens: the entry point, and the route by
// listed tokens.
//
// Listed tokens.  The sparse attention kernels take any selection, so also all tokens: a kernel writes for every session one page table (pages
// of the prefix, then its own) and the list of its tokens.  That is the way of layouts whose work is bound by the matrix units for one session
// already, so that reading the prefix once for all gains nothing (latent: 128 heads read one row per token, 242 flops a byte), and of head
// dims without a kernel of their own.
#include "attn_shared.cuh"

namespace janus {

int sparse_attn_listed(const void* q, int M, int H_q, int d_qk, const void* k_pool, const void* v_pool, int64_t page_stride, int64_t tok_stride,
                       int64_t head_stride, int64_t v_page_stride, int64_t v_tok_stride, int64_t v_head_stride, int n_kv_heads, int d_v, const int32_t* idx, int k,
                       int page_size, const int32_t* page_tables, const int64_t* table_offsets, float softmax_scale, void* out, float* lse, int32_t* dev_status,
                       cudaStream_t stream);

constexpr int SL_THREADS = 256;

struct SlParams {
    const int32_t* prefix_table;
    const int32_t* page_tables;
    const int64_t* table_offsets;
    const int64_t* kv_lens;
    int64_t prefix, max_len, n_phys;
    int B, page_size, prefix_pages, first_own, width;      // first_own: page of a session's table that holds token `prefix`
    int k;
    int32_t* idx;              // [B, k]
    int32_t* tables;           // [B, width]
    int64_t* offsets;          // [B + 1]
    int32_t* dev_status;
};

// One block per session and stretch of its tokens and pages.
__global__ void __launch_bounds__(SL_THREADS) shared_list_kernel(const SlParams p) {
    grid_launch_next();
    grid_wait();
    const int b = blockIdx.y;
    int64_t len = ld_input(p.kv_lens + b);
    if (len > p.max_len || len < 0 || (len > 0 && len < p.prefix)) {
        if (threadIdx.x == 0 && blockIdx.x == 0) report(p.dev_status, JANUS_DEV_INDEX_OUT_OF_RANGE);
        len = len > p.max_len ? p.max_len : 0;
    }
    int64_t table = 0, entries = 0;
    if (p.max_len > p.prefix) {
        table = ld_input(p.table_offsets + b);
        entries = ld_input(p.table_offsets + b + 1) - table;
        if (table < 0) entries = 0;
    }
    // a page of the prefix that also holds a session's first own tokens is there twice: the tokens behind it are one page further on
    const int shift = p.prefix % p.page_size != 0 ? p.page_size : 0;
    const int64_t n = static_cast<int64_t>(p.k) > p.width ? p.k : p.width;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * SL_THREADS + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * SL_THREADS) {
        if (i < p.k) p.idx[static_cast<int64_t>(b) * p.k + i] = i < len ? static_cast<int32_t>(i + (i < p.prefix ? 0 : shift)) : -1;
        if (i < p.width) {
            int32_t id = -1;
            if (i < p.prefix_pages) {
                id = ld_input(p.prefix_table + i);
            } else {
                const int64_t j = i - p.prefix_pages + p.first_own;
                if (j < entries) id = ld_input(p.page_tables + table + j);
            }
            p.tables[static_cast<int64_t>(b) * p.width + i] = id < p.n_phys ? id : -1;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        p.offsets[b] = static_cast<int64_t>(b) * p.width;
        if (b == p.B - 1) p.offsets[p.B] = static_cast<int64_t>(p.B) * p.width;
    }
}

// Sizes of the lists; false where a token's number would pass 31 bits.
static bool sl_sizes(int page_size, int64_t prefix, int64_t max_len, int64_t* prefix_pages, int64_t* width) {
    *prefix_pages = (prefix + page_size - 1) / page_size;
    *width = *prefix_pages + (max_len + page_size - 1) / page_size - prefix / page_size;
    return max_len <= INT32_MAX - 2 * static_cast<int64_t>(page_size);
}

static size_t sl_bytes(int B, int page_size, int64_t prefix, int64_t max_len) {
    int64_t prefix_pages, width;
    if (!sl_sizes(page_size, prefix, max_len, &prefix_pages, &width)) return 0;
    auto round = [](size_t n) { return (n + 15) & ~static_cast<size_t>(15); };
    return round(sizeof(int64_t) * (static_cast<size_t>(B) + 1)) + round(sizeof(int32_t) * static_cast<size_t>(B) * width) + round(sizeof(int32_t) * static_cast<size_t>(B) * max_len);
}

}  // namespace janus

extern "C" size_t janus_attn_decode_shared_workspace_size(int B, int H_q, int d_qk, int n_kv_heads, int d_v, int page_size, int64_t prefix_len, int64_t max_len) {
    using namespace janus;
    if (B <= 0 || H_q <= 0 || d_qk <= 0 || n_kv_heads <= 0 || d_v <= 0 || page_size <= 0 || prefix_len < 0 || max_len < prefix_len) return 0;
    if (attn_shared_tc_supported(d_qk, d_v)) return attn_shared_tc_workspace(B, H_q, n_kv_heads, d_v, prefix_len, max_len);
    return sl_bytes(B, page_size, prefix_len, max_len);
}

extern "C" int janus_attn_decode_shared(const void* q, int B, int H_q, int d_qk, const void* k_pool, int64_t k_page_stride, int64_t k_tok_stride,
                                        int64_t k_head_stride, const void* v_pool, int64_t v_page_stride, int64_t v_tok_stride, int64_t v_head_stride,
                                        int n_kv_heads, int d_v, int page_size, int64_t n_phys_pages, const int32_t* prefix_table, int64_t prefix_len,
                                        const int32_t* page_tables, const int64_t* table_offsets, const int64_t* kv_lens, int64_t max_len,
                                        float softmax_scale, void* out, float* lse, void* ws, size_t ws_bytes, int32_t* dev_status, void* stream_) {
    using namespace janus;
    if (B < 0 || H_q <= 0 || d_qk <= 0 || d_v <= 0 || n_kv_heads <= 0 || page_size <= 0 || n_phys_pages < 0 || prefix_len < 0 || max_len < prefix_len)
        return JANUS_ERR_INVALID_ARG;
    if (H_q % n_kv_heads != 0 || !(softmax_scale > 0.f) || softmax_scale > 3.4e38f) return JANUS_ERR_INVALID_ARG;
    if ((d_qk % 8) != 0 || (d_v % 8) != 0 || d_qk > 576 || d_v > 512) return JANUS_ERR_UNSUPPORTED;
    if (n_phys_pages > INT32_MAX || page_size > (1 << 30) || max_len > INT32_MAX - 2 * static_cast<int64_t>(page_size)) return JANUS_ERR_UNSUPPORTED;
    if (B == 0) return JANUS_OK;
    if (B > 65535) return JANUS_ERR_UNSUPPORTED;
    if (!q || !k_pool || !v_pool || !out || !kv_lens) return JANUS_ERR_INVALID_ARG;
    if ((prefix_len > 0 && !prefix_table) || (max_len > prefix_len && (!page_tables || !table_offsets))) return JANUS_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(out) || !aligned16(ws)) return JANUS_ERR_INVALID_ARG;
    if (((k_page_stride | k_tok_stride | k_head_stride | v_page_stride | v_tok_stride | v_head_stride) % 8) != 0) return JANUS_ERR_INVALID_ARG;
    auto positive = [&](int64_t page, int64_t tok, int64_t head) { return (n_phys_pages <= 1 || page > 0) && (page_size <= 1 || tok > 0) && (n_kv_heads <= 1 || head > 0); };
    if (!positive(k_page_stride, k_tok_stride, k_head_stride) || !positive(v_page_stride, v_tok_stride, v_head_stride)) return JANUS_ERR_INVALID_ARG;
    if (n_phys_pages == 0 && max_len > 0) return JANUS_ERR_INVALID_ARG;
    const bool same_strides = k_page_stride == v_page_stride && k_tok_stride == v_tok_stride && (n_kv_heads == 1 || k_head_stride == v_head_stride);
    if (v_pool == k_pool && (d_v > d_qk || !same_strides)) return JANUS_ERR_INVALID_ARG;
    if (ws_bytes < janus_attn_decode_shared_workspace_size(B, H_q, d_qk, n_kv_heads, d_v, page_size, prefix_len, max_len)) return JANUS_ERR_WORKSPACE_TOO_SMALL;
    if (!ws) return JANUS_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (attn_shared_tc_supported(d_qk, d_v))
        return launch_attn_shared_tc({q, B, H_q, d_qk, k_pool, k_page_stride, k_tok_stride, k_head_stride, v_pool, v_page_stride, v_tok_stride, v_head_stride, n_kv_heads,
                                      d_v, page_size, n_phys_pages, prefix_table, prefix_len, page_tables, table_offsets, kv_lens, max_len, softmax_scale, out, lse, ws,
                                      dev_status}, stream);

    SlParams p;
    p.prefix_table = prefix_table; p.page_tables = page_tables; p.table_offsets = table_offsets; p.kv_lens = kv_lens;
    p.prefix = prefix_len; p.max_len = max_len; p.n_phys = n_phys_pages;
    p.B = B; p.page_size = page_size;
    int64_t prefix_pages, width;
    sl_sizes(page_size, prefix_len, max_len, &prefix_pages, &width);
    p.prefix_pages = static_cast<int>(prefix_pages); p.first_own = static_cast<int>(prefix_len / page_size); p.width = static_cast<int>(width);
    p.k = static_cast<int>(max_len);
    p.offsets = static_cast<int64_t*>(ws);
    p.tables = reinterpret_cast<int32_t*>(static_cast<unsigned char*>(ws) + ((sizeof(int64_t) * (B + 1) + 15) & ~static_cast<size_t>(15)));
    p.idx = p.tables + ((static_cast<size_t>(B) * width + 3) & ~static_cast<size_t>(3));
    p.dev_status = dev_status;
    const int64_t most = p.k > p.width ? p.k : p.width, blocks = (most + 4 * SL_THREADS - 1) / (4 * SL_THREADS);
    const dim3 grid(static_cast<unsigned>(blocks < 1 ? 1 : blocks < 64 ? blocks : 64), static_cast<unsigned>(B));
    JANUS_CUDA_CHECK(launch_kernel(shared_list_kernel, grid, SL_THREADS, 0, stream, 1, p));
    return sparse_attn_listed(q, B, H_q, d_qk, k_pool, v_pool, k_page_stride, k_tok_stride, k_head_stride, v_page_stride, v_tok_stride, v_head_stride, n_kv_heads, d_v, p.idx,
                              p.k, page_size, p.tables, p.offsets, softmax_scale, out, lse, dev_status, stream);
}
