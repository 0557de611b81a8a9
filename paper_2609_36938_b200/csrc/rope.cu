// Rotary positions on part of every head, and the write of new rows into the paged cache, rotated on the way.
//
//     angle a = position * f_i;   (y1, y2) = scale * (x1 cos a - x2 sin a, x1 sin a + x2 cos a)     for the pair i of a head
//
// (pairs are neighbours, or the two halves of the rotated part; `inverse` takes -a, which is also the gradient of the forward rotation).
//
// Angles.  f_i comes as turns per position in units of 2^-64, so the phase of a position is one 64-bit product: whole turns drop out of it
// by overflow, and what is left is rounded to 2^-32 turns: off by 2^-33 turns at most, beside position times what the entry is off by.  (An fp32 product
// of position and frequency is off by 0.06 rad at position 10^6.)  It is split into a quarter turn and an eighth of a turn either side, of which sine and cosine are taken in fp32.
//
// What bounds it: HBM; three flops per element.  A thread takes one 16-byte chunk of the head dimension (half layout: two, half the rotated
// part apart), works out the sines and cosines of its pairs once and applies them to the same chunk of up to RP_HEADS heads of its
// token.  Consecutive threads take consecutive chunks, then heads, then tokens.  Two heads a thread: 4096 tokens x 128 heads, 64 dims of 576: 37.8 us (134 MB of
// 128-byte pieces, 3.5 TB/s), 777 x 32 x 128 in fp32 4.7 us (5.4 TB/s), rows of 4096 tokens into the cache with 32 query heads 20.1 us; four heads 39.9, 5.1 and
// 26.8 (fewer warps); one 44.1, 5.6 and 23.2 (angles).  Sines and cosines of a block's tokens in shared memory, each worked out once: 82.9, 10.4
// and 38.8 (the barrier keeps loads and stores apart).  Loads ahead of the look at the position: 40.2, 5.1 and 21.1 (registers).  Two pairs at a time
// in packed registers, with shorter polynomials: 40.7, 4.8 and 23.0.  A plain copy of the same 128-byte pieces takes 28.8.
#include <cuda_fp16.h>

#include <algorithm>

#include "janus_common.cuh"
#include "memory_overlap.h"

namespace janus {

constexpr int RP_THREADS = 256;
constexpr int RP_HEADS = 2;
constexpr int RP_JOBS = 3;           // queries, keys, values

// Rows of one tensor: heads h of rows t from src to dst.  `rot` = 0: copied only.
struct RpJob {
    const unsigned char* src;
    unsigned char* dst;
    int64_t s_row, s_head;           // bytes
    int64_t d_row, d_head, d_page;   // bytes; paged: d_row is that of a token within its page
    int H;
    int head_bytes;                  // bytes of a head that are moved (copy chunks included), 0: only the rotated part
    int chunks;                      // per head
    int groups;                      // heads g, g + groups, ... are one thread's
    bool rotate, paged;
    uint32_t first_block, inv_row, inv_chunks;       // 2^32 / (groups * chunks), 2^32 / chunks
};

struct RpParams {
    RpJob job[RP_JOBS];
    int n_jobs;
    int64_t T;
    const int64_t* positions;
    const int64_t* slots;
    const uint64_t* freqs;
    int rot_offset, rot;             // elements
    float scale;
    bool inverse;
    int page_size, page_shift;
    int64_t n_slots;
    int32_t* dev_status;
};

// Sine and cosine of phase * 2^-64 turns, to which 2^31 has been added: the high word is then the phase rounded to 2^-32 turns.  The nearest quarter turn is
// taken off, and of what is left, at most an eighth, the Taylor series: the first terms left out, a^11 / 11! and a^12 / 12!, are below 2^-29.
__device__ __forceinline__ void rp_turn(uint64_t phase, float& s, float& c) {
    const uint32_t top = static_cast<uint32_t>(phase >> 32), q = (top + (1u << 29)) >> 30;
    const float a = static_cast<float>(static_cast<int32_t>(top - (q << 30))) * 1.4629180792671596e-9f, b = a * a;      // 2 pi 2^-32
    const float s0 = fmaf(a * b, fmaf(b, fmaf(b, fmaf(b, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), a);
    const float c0 = fmaf(b, fmaf(b, fmaf(b, fmaf(b, fmaf(b, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    s = (q & 1u) ? c0 : s0;
    c = (q & 1u) ? s0 : c0;
    if (q & 2u) s = -s;
    if ((q + 1u) & 2u) c = -c;
}

// u / d with m = 2^32 / d, rounded down: the estimate is at most two short.
__device__ __forceinline__ uint32_t rp_divide(uint32_t u, uint32_t d, uint32_t m) {
    uint32_t q = __umulhi(u, m), r = u - q * d;
    if (r >= d) { ++q; r -= d; }
    if (r >= d) ++q;
    return q;
}

template <class T>
__device__ __forceinline__ float rp_load(T x);
template <>
__device__ __forceinline__ float rp_load(uint16_t x) { return bf16_bits_to_float(x); }
template <>
__device__ __forceinline__ float rp_load(__half x) { return __half2float(x); }
template <>
__device__ __forceinline__ float rp_load(float x) { return x; }
template <class T>
__device__ __forceinline__ T rp_store(float x);
template <>
__device__ __forceinline__ uint16_t rp_store(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
template <>
__device__ __forceinline__ __half rp_store(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ float rp_store(float x) { return x; }

template <class T, int VEC>
struct alignas(VEC * sizeof(T) == 16 ? 16 : sizeof(T)) RpVec {
    T v[VEC];
};

// VEC: elements of a rotated chunk: 16 bytes, or one element (neighbours: a pair) where something does not lie on 16 bytes.  The rest of a
// head is copied in chunks of 16 bytes or of one element.
template <class T, int VEC, bool NEIGHBOURS>
__global__ void __launch_bounds__(RP_THREADS) rope_kernel(const RpParams p) {
    using V = RpVec<T, VEC>;
    grid_launch_next();
    grid_wait();
    int n = 0;
    while (n + 1 < p.n_jobs && blockIdx.x >= p.job[n + 1].first_block) ++n;
    const RpJob& job = p.job[n];
    const uint64_t unit = static_cast<uint64_t>(blockIdx.x - job.first_block) * RP_THREADS + threadIdx.x;
    const uint32_t per_row = static_cast<uint32_t>(job.groups * job.chunks);
    int64_t t;
    uint32_t in_row;
    if (unit >> 32) {
        t = static_cast<int64_t>(unit / per_row);
        in_row = static_cast<uint32_t>(unit - static_cast<uint64_t>(t) * per_row);
    } else {
        const uint32_t u = static_cast<uint32_t>(unit);
        t = rp_divide(u, per_row, job.inv_row);
        in_row = u - static_cast<uint32_t>(t) * per_row;
    }
    if (t >= p.T) return;
    const int g = static_cast<int>(rp_divide(in_row, job.chunks, job.inv_chunks)), chunk = static_cast<int>(in_row - g * job.chunks);

    // which bytes of a head this thread moves, and whether it turns them
    constexpr int CB = VEC * static_cast<int>(sizeof(T)), COPY_VEC = CB == 16 ? VEC : 1, COPY_BYTES = COPY_VEC * static_cast<int>(sizeof(T));
    using Copy = RpVec<T, COPY_VEC>;
    const int rot_bytes = p.rot * static_cast<int>(sizeof(T)), at = p.rot_offset * static_cast<int>(sizeof(T));
    const int turned = job.rotate ? rot_bytes / (NEIGHBOURS ? CB : 2 * CB) : 0;       // the first chunks of a head are the rotated ones
    const bool turn = chunk < turned;
    int off;
    if (turn) {
        off = at + chunk * CB;
    } else {
        off = (chunk - turned) * COPY_BYTES;
        if (job.rotate && off >= at) off += rot_bytes;
    }

    const int64_t pos = ld_input(p.positions + t);
    unsigned char* dst = job.dst;
    if (job.paged) {
        const int64_t slot = ld_input(p.slots + t);
        if (slot < 0) return;                                      // a padding row
        if (slot >= p.n_slots || pos < 0) {
            report(p.dev_status, JANUS_DEV_INDEX_OUT_OF_RANGE);
            return;
        }
        const int64_t page = p.page_shift >= 0 ? slot >> p.page_shift : slot / p.page_size;
        dst += page * job.d_page + (slot - page * p.page_size) * job.d_row;
    } else {
        if (pos < 0) return;
        dst += t * job.d_row;
    }
    const unsigned char* src = job.src + t * job.s_row;

    if (!turn) {
        Copy x[RP_HEADS];
#pragma unroll
        for (int i = 0; i < RP_HEADS; ++i)
            if (g + i * job.groups < job.H) x[i] = *reinterpret_cast<const Copy*>(src + (g + i * job.groups) * job.s_head + off);
#pragma unroll
        for (int i = 0; i < RP_HEADS; ++i)
            if (g + i * job.groups < job.H) *reinterpret_cast<Copy*>(dst + (g + i * job.groups) * job.d_head + off) = x[i];
        return;
    }
    constexpr int PAIRS = NEIGHBOURS ? VEC / 2 : VEC;
    const int half = rot_bytes / 2;
    V x[RP_HEADS], y[NEIGHBOURS ? 1 : RP_HEADS];
#pragma unroll
    for (int i = 0; i < RP_HEADS; ++i)
        if (g + i * job.groups < job.H) {
            const unsigned char* a = src + (g + i * job.groups) * job.s_head + off;
            x[i] = *reinterpret_cast<const V*>(a);
            if constexpr (!NEIGHBOURS) y[i] = *reinterpret_cast<const V*>(a + half);
        }
    float s[PAIRS], c[PAIRS];
#pragma unroll
    for (int e = 0; e < PAIRS; ++e) {
        rp_turn(static_cast<uint64_t>(pos) * ld_input(p.freqs + chunk * PAIRS + e) + (1ull << 31), s[e], c[e]);
        s[e] *= p.inverse ? -p.scale : p.scale;
        c[e] *= p.scale;
    }
#pragma unroll
    for (int i = 0; i < RP_HEADS; ++i)
        if (g + i * job.groups < job.H) {
            unsigned char* a = dst + (g + i * job.groups) * job.d_head + off;
#pragma unroll
            for (int e = 0; e < PAIRS; ++e) {
                T& p1 = NEIGHBOURS ? x[i].v[2 * e] : x[i].v[e];
                T& p2 = NEIGHBOURS ? x[i].v[(2 * e + 1) % VEC] : y[NEIGHBOURS ? 0 : i].v[e];
                const float x1 = rp_load(p1), x2 = rp_load(p2);
                p1 = rp_store<T>(x1 * c[e] - x2 * s[e]);
                p2 = rp_store<T>(x1 * s[e] + x2 * c[e]);
            }
            *reinterpret_cast<V*>(a) = x[i];
            if constexpr (!NEIGHBOURS) *reinterpret_cast<V*>(a + half) = y[i];
        }
}

// [rows, heads, dim] or [pages, tokens, heads, dim], strides in elements, as it lies in memory.
static MoTensor rp_memory(const void* at, int elem, int64_t dim, int64_t n0, int64_t stride0, int64_t n1, int64_t stride1, int64_t n2 = 1, int64_t stride2 = 0) {
    return {reinterpret_cast<uintptr_t>(at), dim * elem, {n0, n1, n2}, {stride0 * elem, stride1 * elem, stride2 * elem}};
}

template <class T, bool NEIGHBOURS>
static int rp_launch(RpParams& p, bool wide, cudaStream_t stream) {
    const int vec = wide ? 16 / static_cast<int>(sizeof(T)) : NEIGHBOURS ? 2 : 1, cb = vec * static_cast<int>(sizeof(T)), copy_bytes = wide ? 16 : static_cast<int>(sizeof(T));
    uint64_t blocks = 0;
    for (int n = 0; n < p.n_jobs; ++n) {
        RpJob& j = p.job[n];
        const int rot_bytes = j.rotate ? p.rot * static_cast<int>(sizeof(T)) : 0;
        j.chunks = rot_bytes / (NEIGHBOURS ? cb : 2 * cb) + (j.head_bytes > 0 ? (j.head_bytes - rot_bytes) / copy_bytes : 0);
        // one head per thread until those are more threads than the GPU holds at once
        const int64_t threads = p.T * j.H * j.chunks;
        int per = 1;
        while (per < RP_HEADS && threads / per > 148 * 2048) per *= 2;
        j.groups = (j.H + per - 1) / per;
        j.first_block = static_cast<uint32_t>(blocks);
        j.inv_row = static_cast<uint32_t>(std::min<uint64_t>((1ull << 32) / (static_cast<uint64_t>(j.groups) * j.chunks), UINT32_MAX));
        j.inv_chunks = static_cast<uint32_t>(std::min<uint64_t>((1ull << 32) / j.chunks, UINT32_MAX));
        blocks += (static_cast<uint64_t>(p.T) * j.groups * j.chunks + RP_THREADS - 1) / RP_THREADS;
        if (blocks > 0x7fffffffu || static_cast<int64_t>(j.groups) * j.chunks > INT32_MAX) return JANUS_ERR_UNSUPPORTED;
    }
    if (blocks == 0) return JANUS_OK;
    const dim3 grid(static_cast<unsigned>(blocks));
    if (wide) JANUS_CUDA_CHECK(launch_kernel(rope_kernel<T, 16 / static_cast<int>(sizeof(T)), NEIGHBOURS>, grid, RP_THREADS, 0, stream, 1, p));
    else JANUS_CUDA_CHECK(launch_kernel(rope_kernel<T, NEIGHBOURS ? 2 : 1, NEIGHBOURS>, grid, RP_THREADS, 0, stream, 1, p));
    return JANUS_OK;
}

// Every address on 16 bytes: bases, strides, and where the rotated part (half layout: its halves too) begins and ends.
static bool rp_wide(const RpParams& p, int elem, bool neighbours) {
    uint64_t all = static_cast<uint64_t>(p.rot_offset) * elem | static_cast<uint64_t>(p.rot) * elem / (neighbours ? 1 : 2);
    for (int n = 0; n < p.n_jobs; ++n) {
        const RpJob& j = p.job[n];
        all |= reinterpret_cast<uintptr_t>(j.src) | reinterpret_cast<uintptr_t>(j.dst) | static_cast<uint64_t>(j.head_bytes);
        all |= static_cast<uint64_t>(j.s_row) | static_cast<uint64_t>(j.s_head) | static_cast<uint64_t>(j.d_row) | static_cast<uint64_t>(j.d_head) | static_cast<uint64_t>(j.d_page);
    }
    return (all & 15u) == 0;
}

// Strides of an axis of one do not matter; 0 keeps them out of the alignment rule.
static RpJob rp_job(const void* src, int64_t s_row, int64_t s_head, void* dst, int64_t d_page, int64_t d_row, int64_t d_head, int64_t T, int H, int elem) {
    RpJob j = {};
    j.src = static_cast<const unsigned char*>(src);
    j.dst = static_cast<unsigned char*>(dst);
    j.s_row = T > 1 ? s_row * elem : 0; j.s_head = H > 1 ? s_head * elem : 0;
    j.d_row = d_row * elem; j.d_head = H > 1 ? d_head * elem : 0; j.d_page = d_page * elem;
    j.H = H;
    return j;
}

}  // namespace janus

extern "C" int janus_rope(const void* x, int64_t x_row_stride, int64_t x_head_stride, int64_t T, int H, int D, const int64_t* positions,
                          const uint64_t* freqs, int rot_offset, int rot_dim, int interleaved, float scale, int inverse, int dtype, void* out,
                          int64_t out_row_stride, int64_t out_head_stride, void* stream_) {
    using namespace janus;
    if (T < 0 || H < 0 || D <= 0 || rot_offset < 0 || rot_dim <= 0 || (rot_dim & 1) || rot_offset > D - rot_dim) return JANUS_ERR_INVALID_ARG;
    if (dtype != JANUS_ELEM_BF16 && dtype != JANUS_ELEM_FP16 && dtype != JANUS_ELEM_FP32) return JANUS_ERR_UNSUPPORTED;
    if (D > (1 << 28)) return JANUS_ERR_UNSUPPORTED;
    if (T == 0 || H == 0) return JANUS_OK;
    if (!x || !out || !positions || !freqs) return JANUS_ERR_INVALID_ARG;
    const int elem = dtype == JANUS_ELEM_FP32 ? 4 : 2;
    if (((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out)) & (elem - 1)) != 0) return JANUS_ERR_INVALID_ARG;
    if (x_row_stride < 0 || x_head_stride < 0 || out_row_stride < 0 || out_head_stride < 0) return JANUS_ERR_INVALID_ARG;
    const MoTensor out_memory = rp_memory(out, elem, D, T, out_row_stride, H, out_head_stride);
    if (!mo_apart(out_memory)) return JANUS_ERR_INVALID_ARG;
    const bool in_place = x == out;
    if (!in_place && mo_may_share(rp_memory(x, elem, D, T, x_row_stride, H, x_head_stride), out_memory)) return JANUS_ERR_INVALID_ARG;
    if (in_place && ((T > 1 && x_row_stride != out_row_stride) || (H > 1 && x_head_stride != out_head_stride))) return JANUS_ERR_INVALID_ARG;
    RpParams p = {};
    p.n_jobs = 1;
    p.job[0] = rp_job(x, x_row_stride, x_head_stride, out, 0, T > 1 ? out_row_stride : 0, out_head_stride, T, H, elem);
    p.job[0].rotate = true;
    p.job[0].head_bytes = in_place ? 0 : D * elem;
    p.T = T; p.positions = positions; p.freqs = freqs;
    p.rot_offset = rot_offset; p.rot = rot_dim; p.scale = scale; p.inverse = inverse != 0;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const bool wide = rp_wide(p, elem, interleaved != 0);
    if (dtype == JANUS_ELEM_BF16) return interleaved ? rp_launch<uint16_t, true>(p, wide, stream) : rp_launch<uint16_t, false>(p, wide, stream);
    if (dtype == JANUS_ELEM_FP16) return interleaved ? rp_launch<__half, true>(p, wide, stream) : rp_launch<__half, false>(p, wide, stream);
    return interleaved ? rp_launch<float, true>(p, wide, stream) : rp_launch<float, false>(p, wide, stream);
}

extern "C" int janus_rope_append(const void* q, int64_t q_row_stride, int64_t q_head_stride, int H_q, const void* k, int64_t k_row_stride,
                                 int64_t k_head_stride, int n_kv_heads, int d_qk, const void* v, int64_t v_row_stride, int64_t v_head_stride, int d_v,
                                 int64_t T, const int64_t* positions, const int64_t* slots, const uint64_t* freqs, int rot_offset, int rot_dim,
                                 int interleaved, float scale, void* q_out, int64_t q_out_row_stride, int64_t q_out_head_stride, void* k_pool,
                                 int64_t k_page_stride, int64_t k_tok_stride, int64_t k_pool_head_stride, void* v_pool, int64_t v_page_stride,
                                 int64_t v_tok_stride, int64_t v_pool_head_stride, int page_size, int64_t n_phys_pages, int32_t* dev_status, void* stream_) {
    using namespace janus;
    const bool has_q = q != nullptr || q_out != nullptr, has_v = v != nullptr || v_pool != nullptr;
    if (T < 0 || n_kv_heads <= 0 || d_qk <= 0 || page_size <= 0 || n_phys_pages < 0) return JANUS_ERR_INVALID_ARG;
    if (rot_offset < 0 || rot_dim <= 0 || (rot_dim & 1) || rot_offset > d_qk - rot_dim) return JANUS_ERR_INVALID_ARG;
    if (has_q && H_q <= 0) return JANUS_ERR_INVALID_ARG;
    if (has_v && d_v <= 0) return JANUS_ERR_INVALID_ARG;
    if ((d_qk % 8) != 0 || (has_v && (d_v % 8) != 0)) return JANUS_ERR_UNSUPPORTED;
    if (d_qk > (1 << 28) || (has_v && d_v > (1 << 28))) return JANUS_ERR_UNSUPPORTED;
    if (T == 0) return JANUS_OK;
    if (!k || !k_pool || !positions || !slots || !freqs || (has_q && (!q || !q_out)) || (has_v && (!v || !v_pool))) return JANUS_ERR_INVALID_ARG;
    if (n_phys_pages > INT64_MAX / page_size) return JANUS_ERR_INVALID_ARG;
    RpParams p = {};
    // the longest job first: its blocks are under way before the others'
    if (has_q) {
        p.job[p.n_jobs] = rp_job(q, q_row_stride, q_head_stride, q_out, 0, T > 1 ? q_out_row_stride : 0, q_out_head_stride, T, H_q, 2);
        p.job[p.n_jobs].rotate = true;
        p.job[p.n_jobs++].head_bytes = q == q_out ? 0 : d_qk * 2;
        if (q_row_stride < 0 || q_head_stride < 0 || q_out_row_stride < 0 || q_out_head_stride < 0) return JANUS_ERR_INVALID_ARG;
        if (q == q_out && ((T > 1 && q_row_stride != q_out_row_stride) || (H_q > 1 && q_head_stride != q_out_head_stride))) return JANUS_ERR_INVALID_ARG;
    }
    if (k_row_stride < 0 || k_head_stride < 0 || k_page_stride < 0 || k_tok_stride < 0 || k_pool_head_stride < 0) return JANUS_ERR_INVALID_ARG;
    const MoTensor k_pool_memory = rp_memory(k_pool, 2, d_qk, n_phys_pages, k_page_stride, page_size, k_tok_stride, n_kv_heads, k_pool_head_stride);
    if (!mo_apart(k_pool_memory)) return JANUS_ERR_INVALID_ARG;
    const MoTensor q_out_memory = rp_memory(q_out, 2, d_qk, T, q_out_row_stride, has_q ? H_q : 0, q_out_head_stride);
    if (has_q) {      // nothing that another thread still reads or also writes
        if (!mo_apart(q_out_memory) || mo_may_share(q_out_memory, k_pool_memory)) return JANUS_ERR_INVALID_ARG;
        if (mo_may_share(q_out_memory, rp_memory(k, 2, d_qk, T, k_row_stride, n_kv_heads, k_head_stride))) return JANUS_ERR_INVALID_ARG;
        if (q != q_out && mo_may_share(q_out_memory, rp_memory(q, 2, d_qk, T, q_row_stride, H_q, q_head_stride))) return JANUS_ERR_INVALID_ARG;
    }
    p.job[p.n_jobs] = rp_job(k, k_row_stride, k_head_stride, k_pool, k_page_stride, k_tok_stride, k_pool_head_stride, T, n_kv_heads, 2);
    p.job[p.n_jobs].rotate = true;
    p.job[p.n_jobs].paged = true;
    p.job[p.n_jobs++].head_bytes = d_qk * 2;
    if (has_v) {
        if (v_row_stride < 0 || v_head_stride < 0 || v_page_stride < 0 || v_tok_stride < 0 || v_pool_head_stride < 0) return JANUS_ERR_INVALID_ARG;
        const MoTensor v_pool_memory = rp_memory(v_pool, 2, d_v, n_phys_pages, v_page_stride, page_size, v_tok_stride, n_kv_heads, v_pool_head_stride);
        if (!mo_apart(v_pool_memory) || mo_may_share(k_pool_memory, v_pool_memory)) return JANUS_ERR_INVALID_ARG;      // two rows for one place
        if (has_q && (mo_may_share(q_out_memory, v_pool_memory) || mo_may_share(q_out_memory, rp_memory(v, 2, d_v, T, v_row_stride, n_kv_heads, v_head_stride))))
            return JANUS_ERR_INVALID_ARG;
        p.job[p.n_jobs] = rp_job(v, v_row_stride, v_head_stride, v_pool, v_page_stride, v_tok_stride, v_pool_head_stride, T, n_kv_heads, 2);
        p.job[p.n_jobs].paged = true;
        p.job[p.n_jobs++].head_bytes = d_v * 2;
    }
    // the rule of the attention calls: rows on 16 bytes; only the rotated part may begin elsewhere
    if (!rp_wide(p, 2, true)) return JANUS_ERR_INVALID_ARG;
    p.T = T; p.positions = positions; p.slots = slots; p.freqs = freqs;
    p.rot_offset = rot_offset; p.rot = rot_dim; p.scale = scale;
    p.page_size = page_size;
    p.page_shift = -1;
    if ((page_size & (page_size - 1)) == 0) {
        p.page_shift = 0;
        while ((1 << p.page_shift) < page_size) ++p.page_shift;
    }
    p.n_slots = n_phys_pages * page_size;
    p.dev_status = dev_status;
    const bool wide = rp_wide(p, 2, interleaved != 0);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    return interleaved ? rp_launch<uint16_t, true>(p, wide, stream) : rp_launch<uint16_t, false>(p, wide, stream);
}
