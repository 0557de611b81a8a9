// Dense attention of one query token per session over a shared prefix and each session's own tokens: the entry point, and the route by
// listed tokens.
//
// Listed tokens.  The sparse attention kernels take any selection, so also all tokens: a kernel writes page tables (pages of the prefix, then the
// session's own) and lists of tokens.  That is the way of layouts whose work is bound by the matrix units for one session already, so that reading the
// prefix once for all gains nothing (latent: 128 heads read one row per token, 242 flops a byte), and of head dims without a kernel of their own.
//
// For the latent layout a session's keys are cut into pieces of equal length, each a row of the selection with an output of its own (fp32), so that every
// pair of SMs has work; the pieces that there are form a compact list, whose length the attention kernel reads from device
// memory, and a last kernel joins them by their log-sum-exp.
#include "attn_shared.cuh"

namespace janus {

int launch_sparse_attn_generic(const void* q, int M, int H_q, int d_qk, const void* k_pool, const void* v_pool, int64_t page_stride,
                               int64_t tok_stride, int64_t head_stride, int64_t v_page_stride, int64_t v_tok_stride, int64_t v_head_stride, int n_kv_heads,
                               int d_v, const int32_t* idx, int k, int page_size, const int32_t* page_table, int64_t n_logical_pages,
                               const int64_t* table_offsets, float softmax_scale, void* out, float* lse, int32_t* dev_status, cudaStream_t stream);
bool sparse_attn_latent_tc_supported(int M, int H_q, int d_qk, const void* k_pool, const void* v_pool, int64_t page_stride,
                                     int64_t tok_stride, int n_kv_heads, int d_v, int k);
int launch_latent_pieces(const void* q, int n_tokens, int max_rows, const int32_t* rows, const int32_t* token_of, const void* pool, int64_t page_stride,
                         int64_t tok_stride, const int32_t* idx, int k, int page_size, const int32_t* page_tables, const int64_t* table_offsets,
                         float softmax_scale, float* out, float* lse, int32_t* dev_status, cudaStream_t stream);

constexpr int SL_THREADS = 256;
constexpr int SL_HEADS = 128, SL_DV = 512;      // latent layout

struct SlParams {
    const int32_t* prefix_table;
    const int32_t* page_tables;
    const int64_t* table_offsets;
    const int64_t* kv_lens;
    int64_t prefix, max_len, n_phys;
    int B, page_size, prefix_pages, first_own, width;      // first_own: page of a session's table that holds token `prefix`; width: pages of a session
    int k, pieces;             // tokens of a row, rows of a session at most
    int32_t* idx;              // [rows, k]
    int row_width;             // table entries of a row: those of its own tokens where rows are compact
    int32_t* tables;           // [rows, row_width]
    int64_t* offsets;          // [rows + 1]
    int32_t* row_base;         // [B + 1]: rows of the sessions before
    int32_t* token_of;         // [rows]: session of a row
    bool compact;              // only rows that there are; else `pieces` (one) for every session
    int32_t* dev_status;
};

__device__ __forceinline__ int64_t sl_length(const SlParams& p, int b, bool& bad) {
    const int64_t len = ld_input(p.kv_lens + b);
    bad = len > p.max_len || len < 0 || (len > 0 && len < p.prefix);
    return len > p.max_len ? p.max_len : len < p.prefix ? 0 : len;
}

// A block per piece of a session.
__global__ void __launch_bounds__(SL_THREADS) shared_list_kernel(const SlParams p) {
    grid_launch_next();
    __shared__ int sums[SL_THREADS / 32];
    grid_wait();
    const int b = blockIdx.y, piece = blockIdx.x;
    bool bad;
    const int64_t len = sl_length(p, b, bad);
    if (bad && threadIdx.x == 0 && piece == 0) report(p.dev_status, JANUS_DEV_INDEX_OUT_OF_RANGE);
    int row = b * p.pieces + piece;
    if (p.compact) {           // rows of the sessions before this one
        int before = 0;
        for (int i = threadIdx.x; i < b; i += SL_THREADS) before += static_cast<int>((sl_length(p, i, bad) + p.k - 1) / p.k);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) before += __shfl_xor_sync(0xffffffffu, before, d);
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = before;
        __syncthreads();
        before = 0;
#pragma unroll
        for (int w = 0; w < SL_THREADS / 32; ++w) before += sums[w];
        const int here = static_cast<int>((len + p.k - 1) / p.k);
        row = before + piece;
        if (piece == 0 && threadIdx.x == 0) {
            p.row_base[b] = before;
            if (b == p.B - 1) p.row_base[p.B] = before + here;
        }
        if (piece >= here) {
            if (b == p.B - 1 && piece == here && threadIdx.x == 0) p.offsets[row] = static_cast<int64_t>(row) * p.row_width;
            return;
        }
        if (threadIdx.x == 0) p.token_of[row] = b;
    }
    int64_t table = 0, entries = 0;
    if (p.max_len > p.prefix) {
        table = ld_input(p.table_offsets + b);
        entries = ld_input(p.table_offsets + b + 1) - table;
        if (table < 0) entries = 0;
    }
    // a page of the prefix that also holds a session's first own tokens is there twice: the tokens behind it are one page further on
    const int shift = p.prefix % p.page_size != 0 ? p.page_size : 0;
    const int64_t first = static_cast<int64_t>(piece) * p.k;
    // the pages that the row's tokens lie in, where rows are compact no others: e0 .. e1 of the session's
    const int64_t last = first + p.k < len ? first + p.k : len;
    int e0 = 0, e1 = p.width;
    if (p.compact && last > first) {
        e0 = static_cast<int>((first + (first < p.prefix ? 0 : shift)) / p.page_size);
        e1 = static_cast<int>((last - 1 + (last - 1 < p.prefix ? 0 : shift)) / p.page_size) + 1;
    }
    const int64_t skipped = static_cast<int64_t>(e0) * p.page_size;
    for (int i = threadIdx.x; i < p.k; i += SL_THREADS) {
        const int64_t s = first + i;
        p.idx[static_cast<int64_t>(row) * p.k + i] = s < len ? static_cast<int32_t>(s + (s < p.prefix ? 0 : shift) - skipped) : -1;
    }
    for (int i = e0 + threadIdx.x; i < e1; i += SL_THREADS) {
        int32_t id = -1;
        if (i < p.prefix_pages) {
            id = ld_input(p.prefix_table + i);
        } else {
            const int64_t j = static_cast<int64_t>(i) - p.prefix_pages + p.first_own;
            if (j < entries) id = ld_input(p.page_tables + table + j);
        }
        p.tables[static_cast<int64_t>(row) * p.row_width + (i - e0)] = id < p.n_phys ? id : -1;
    }
    if (threadIdx.x == 0) {
        p.offsets[row] = static_cast<int64_t>(row) * p.row_width;
        if (b == p.B - 1 && piece == p.pieces - 1) p.offsets[row + 1] = static_cast<int64_t>(row + 1) * p.row_width;
    }
}

// Output of a session from those of its pieces, in fp32, and their log-sum-exps: 64 threads per head, eight dims each.
__global__ void __launch_bounds__(SL_THREADS) shared_join_kernel(const float* piece_out, const float* piece_lse, const int32_t* row_base, uint16_t* out, float* lse) {
    grid_launch_next();
    grid_wait();
    constexpr float LOG2E = 1.4426950408889634f;
    const int b = blockIdx.y, h = blockIdx.x * (SL_THREADS / 64) + threadIdx.x / 64, d = threadIdx.x % 64 * 8;
    const int r0 = ld_input(row_base + b), r1 = ld_input(row_base + b + 1);
    const float neg_inf = __int_as_float(0xff800000);
    float m = neg_inf, l = 0.f, acc[8] = {};
#pragma unroll 8
    for (int r = r0; r < r1; ++r) m = fmaxf(m, __ldcg(piece_lse + static_cast<int64_t>(r) * SL_HEADS + h));
    const float safe = m == neg_inf ? 0.f : m;
#pragma unroll 8
    for (int r = r0; r < r1; ++r) {
        const int64_t at = static_cast<int64_t>(r) * SL_HEADS + h;
        const float v = __ldcg(piece_lse + at), f = exp2f((v - safe) * LOG2E);
        const float4* src = reinterpret_cast<const float4*>(piece_out + at * SL_DV + d);
        const float4 x = __ldcg(src), y = __ldcg(src + 1);
        if (v == neg_inf) continue;
        const float w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        l += f;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = fmaf(f, w[j], acc[j]);
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;        // (a NaN is a sum)
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(acc[2 * j] * inv, acc[2 * j + 1] * inv);
        w[j] = *reinterpret_cast<const uint32_t*>(&v);
    }
    const int64_t at = static_cast<int64_t>(b) * SL_HEADS + h;
    *reinterpret_cast<uint4*>(out + at * SL_DV + d) = make_uint4(w[0], w[1], w[2], w[3]);
    if (lse != nullptr && d == 0) lse[at] = l != 0.f ? safe + logf(l) : neg_inf;
}

// Lists of the route by listed tokens, and where they lie in the workspace.  Sessions whose pieces could be more than SL_MOST_ROWS go so many at a time: outputs of
// pieces take 256 KB each, 2 GB then.
constexpr int64_t SL_MOST_ROWS = 8192;
struct SlLayout {
    int64_t prefix_pages, width, row_width, pieces, rows;
    int k, at_once;            // tokens of a row; sessions
    size_t offsets, row_base, token_of, tables, idx, lse, out, bytes;
};

static bool sl_latent(int H_q, int d_qk, int n_kv_heads, int d_v, int64_t max_len) {
    return H_q == SL_HEADS && d_qk == 576 && n_kv_heads == 1 && d_v == SL_DV && max_len > 0;
}

static SlLayout sl_layout(int B, bool latent, int page_size, int64_t prefix, int64_t max_len) {
    SlLayout l = {};
    l.prefix_pages = (prefix + page_size - 1) / page_size;
    l.width = l.prefix_pages + (max_len + page_size - 1) / page_size - prefix / page_size;
    l.k = static_cast<int>(max_len);
    if (latent) {
        // By a model in which a pair of SMs takes 1.5 us for 128 tokens (2.0 to 2.3 where all pairs are at work) and 0.6 us for a row, and the rows go to 74
        // pairs in turn, the length with the least time for sessions of max_len (24 sessions of 9216: 1024, 216 rows).  The lengths themselves are on the device, so a
        // loose bound costs time: 300 sessions of 1000 tokens 138 us with max_len 1024, 398 with 131072; 4 of 9000 32 and 72.
        double best = 0.;
        for (int k = 256; k <= 4096; k *= 2) {
            const int64_t rows = B * ((max_len + k - 1) / k), turns = (rows + 73) / 74;
            const double t = turns * (k / 128 * 1.5 + 0.6) + rows * 0.04;      // (and what the join reads)
            if (k == 256 || t < best) { best = t; l.k = k; }
        }
    }
    l.pieces = latent ? (max_len + l.k - 1) / l.k : 1;
    l.at_once = B;
    l.row_width = l.width;
    if (latent) {
        const int64_t most = l.pieces < SL_MOST_ROWS ? SL_MOST_ROWS / l.pieces : 1;
        if (most < B) l.at_once = static_cast<int>(most);
        // k consecutive tokens lie in ceil(k / page_size) + 1 pages at most, and one further where the page that the prefix ends in is there twice
        const int64_t own = (l.k + static_cast<int64_t>(page_size) - 1) / page_size + 2;
        if (own < l.row_width) l.row_width = own;
    }
    l.rows = l.at_once * l.pieces;
    size_t at = 0;
    auto take = [&](size_t n) { const size_t x = at; at += (n + 127) & ~static_cast<size_t>(127); return x; };
    l.offsets = take(sizeof(int64_t) * (l.rows + 1));
    l.row_base = take(latent ? sizeof(int32_t) * (static_cast<size_t>(l.at_once) + 1) : 0);
    l.token_of = take(latent ? sizeof(int32_t) * l.rows : 0);
    l.tables = take(sizeof(int32_t) * l.rows * l.row_width);
    l.idx = take(sizeof(int32_t) * l.rows * l.k);
    l.lse = take(latent ? sizeof(float) * l.rows * SL_HEADS : 0);
    l.out = take(latent ? sizeof(float) * l.rows * SL_HEADS * SL_DV : 0);
    l.bytes = at;
    return l;
}

}  // namespace janus

extern "C" size_t janus_attn_decode_shared_workspace_size(int B, int H_q, int d_qk, int n_kv_heads, int d_v, int page_size, int64_t prefix_len, int64_t max_len) {
    using namespace janus;
    if (B <= 0 || H_q <= 0 || d_qk <= 0 || n_kv_heads <= 0 || d_v <= 0 || page_size <= 0 || prefix_len < 0 || max_len < prefix_len) return 0;
    if (attn_shared_tc_supported(d_qk, d_v)) return attn_shared_tc_workspace(B, H_q, n_kv_heads, d_v, prefix_len, max_len);
    // (which of its two kernels the route takes also depends on the pools)
    const size_t listed = sl_layout(B, false, page_size, prefix_len, max_len).bytes;
    if (!sl_latent(H_q, d_qk, n_kv_heads, d_v, max_len)) return listed;
    const size_t pieces = sl_layout(B, true, page_size, prefix_len, max_len).bytes;
    return pieces > listed ? pieces : listed;
}

extern "C" int janus_attn_decode_shared(const void* q, int B, int H_q, int d_qk, const void* k_pool, int64_t k_page_stride, int64_t k_tok_stride,
                                        int64_t k_head_stride, const void* v_pool, int64_t v_page_stride, int64_t v_tok_stride, int64_t v_head_stride,
                                        int n_kv_heads, int d_v, int page_size, int64_t n_phys_pages, const int32_t* prefix_table, int64_t prefix_len,
                                        const int32_t* page_tables, const int64_t* table_offsets, const int64_t* kv_lens, int64_t max_len,
                                        float softmax_scale, void* out, float* lse, void* ws, size_t ws_bytes, int32_t* dev_status, void* stream_) {
    using namespace janus;
    if (B < 0 || H_q <= 0 || d_qk <= 0 || d_v <= 0 || n_kv_heads <= 0 || page_size <= 0 || n_phys_pages < 0 || prefix_len < 0 || max_len < prefix_len)
        return JANUS_ERR_INVALID_ARG;
    if (H_q % n_kv_heads != 0 || !(softmax_scale > 0.f) || softmax_scale > 2.3e38f) return JANUS_ERR_INVALID_ARG;
    if ((d_qk % 8) != 0 || (d_v % 8) != 0 || d_qk > 576 || d_v > 512) return JANUS_ERR_UNSUPPORTED;
    if (n_phys_pages > INT32_MAX || page_size > (1 << 30) || max_len > INT32_MAX - 2 * static_cast<int64_t>(page_size)) return JANUS_ERR_UNSUPPORTED;
    if (B == 0) return JANUS_OK;
    if (B > 65535 || H_q > 65535) return JANUS_ERR_UNSUPPORTED;      // (grids; fewer than 2^20 segments, as st_divide wants)
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

    // (the two kernels of this route: the latent one takes aliased values alone)
    const bool latent = sl_latent(H_q, d_qk, n_kv_heads, d_v, max_len) &&
                        sparse_attn_latent_tc_supported(B, H_q, d_qk, k_pool, v_pool, k_page_stride, k_tok_stride, n_kv_heads, d_v, 256);
    const SlLayout l = sl_layout(B, latent, page_size, prefix_len, max_len);
    if (l.rows > (1 << 30) / SL_HEADS || l.pieces > 0x7fffffff || l.width > INT32_MAX) return JANUS_ERR_UNSUPPORTED;
    unsigned char* base = static_cast<unsigned char*>(ws);
    SlParams p;
    p.prefix_table = prefix_table; p.page_tables = page_tables; p.table_offsets = table_offsets; p.kv_lens = kv_lens;
    p.prefix = prefix_len; p.max_len = max_len; p.n_phys = n_phys_pages;
    p.B = B; p.page_size = page_size;
    p.prefix_pages = static_cast<int>(l.prefix_pages); p.first_own = static_cast<int>(prefix_len / page_size); p.width = static_cast<int>(l.width);
    p.row_width = static_cast<int>(l.row_width);
    p.k = l.k; p.pieces = static_cast<int>(l.pieces);
    p.offsets = reinterpret_cast<int64_t*>(base + l.offsets);
    p.row_base = reinterpret_cast<int32_t*>(base + l.row_base);
    p.token_of = reinterpret_cast<int32_t*>(base + l.token_of);
    p.tables = reinterpret_cast<int32_t*>(base + l.tables);
    p.idx = reinterpret_cast<int32_t*>(base + l.idx);
    p.compact = latent;
    p.dev_status = dev_status;
    float* piece_out = reinterpret_cast<float*>(base + l.out);
    float* piece_lse = reinterpret_cast<float*>(base + l.lse);
    for (int b = 0; b < B; b += l.at_once) {
        p.B = B - b < l.at_once ? B - b : l.at_once;
        p.kv_lens = kv_lens + b;
        p.table_offsets = table_offsets != nullptr ? table_offsets + b : nullptr;
        JANUS_CUDA_CHECK(launch_kernel(shared_list_kernel, dim3(static_cast<unsigned>(l.pieces), static_cast<unsigned>(p.B)), SL_THREADS, 0, stream, 1, p));
        if (!latent)      // (all sessions at once)
            return launch_sparse_attn_generic(q, B, H_q, d_qk, k_pool, v_pool, k_page_stride, k_tok_stride, k_head_stride, v_page_stride, v_tok_stride, v_head_stride,
                                              n_kv_heads, d_v, p.idx, p.k, page_size, p.tables, 0, p.offsets, softmax_scale, out, lse, dev_status, stream);
        const int64_t at = static_cast<int64_t>(b) * SL_HEADS;
        const int rc = launch_latent_pieces(static_cast<const uint16_t*>(q) + at * d_qk, p.B, static_cast<int>(p.B * l.pieces), p.row_base + p.B, p.token_of, k_pool,
                                            k_page_stride, k_tok_stride, p.idx, p.k, page_size, p.tables, p.offsets, softmax_scale, piece_out, piece_lse, dev_status, stream);
        if (rc != JANUS_OK) return rc;
        JANUS_CUDA_CHECK(launch_kernel(shared_join_kernel, dim3(SL_HEADS / (SL_THREADS / 64), static_cast<unsigned>(p.B)), SL_THREADS, 0, stream, 1, piece_out, piece_lse,
                                       p.row_base, static_cast<uint16_t*>(out) + at * SL_DV, lse != nullptr ? lse + at : nullptr));
    }
    return JANUS_OK;
}
