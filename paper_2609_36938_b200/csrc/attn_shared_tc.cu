// Dense attention of one query token per session over a shared prefix and each session's own tokens, on the tensor cores: keys of 64, 128 or
// 192 dims, values of 64 or 128, any grouping of heads.
//
//     out[b,h,:] = sum_s softmax_s(scale <q[b,h,:], K_s>) V_s     over the P shared tokens and session b's own ones
//
// Work.  Two kinds of segment, cut into tiles of KT keys:
//   prefix   per kv head and 256 rows: the rows are (session, head of the group) pairs, B * group of them, so that a tile of the prefix is read
//            once for 256 rows.  With 128 dims a tile is 16.8 MFLOP against 64 KB: the matrix units bound it;
//   own      per session and kv head: the group's heads are the rows, 8 or so; a tile is read for them alone: HBM bounds it, and the rows of an
//            MMA that stand empty cost nothing (a tile takes 1000 cycles of MMA, 2800 of an SM's share of HBM).
// All tiles form one line, and every CTA (one per SM, persistent) takes an equal stretch of it, whatever the sessions' lengths: each part of a
// segment within a stretch is a fragment that leaves its maximum, sum and unnormalised output in the workspace, and a second kernel merges the
// fragments of a row.  A fragment's place is (number of the CTA) + (number of the segment), which no two share and which the
// merge works out again from the same lengths; so there are no counters, and the result does not depend on timing.
//
// A CTA: two groups of four softmax warps (thread = row), a warp that copies, a warp that issues MMAs.  S of group w lies in tensor memory columns
// [128 w, ...), P (bf16) over it as the A operand of P . V, O of group w in [256 + 128 w, ...).  With more than 128 rows in a segment each group has 128
// rows and both work on every tile; with fewer, both have the same rows and take the tiles in turn, each with an output of its own.  Either way
// the MMAs of one group run while the other does its softmax.  K and V tiles come through one ring in boxes of TMA that lie within a page (the box
// height divides page and tile); boxes of pages that are not there, or of tokens past the end, are out of the map's bounds and arrive as zeros.
// Keys that do not count are masked by bits that the copying warp leaves; their rows of V are cleared, as 0 * NaN is not 0.
//
// The running maximum moves only when a tile exceeds it by more than 2^8, so O is rescaled a handful of times per fragment.  P is rounded to
// bf16 (half a step, 2^-8 relative, as the output itself); the row sum adds the probabilities as they were, so the log-sum-exp is exact to fp32.
// Every wait is bounded; on a timeout the CTA reports JANUS_DEV_WAIT_TIMEOUT and leaves when its copies have landed.
#include "attn_shared.cuh"
#include "sm100_ptx.cuh"

namespace janus {

using namespace ptx;

constexpr int ST_ROWS = 128;                        // rows of an MMA
constexpr int ST_SOFTMAX_WARPS = 8, ST_COPY_WARP = 8, ST_MMA_WARP = 9, ST_THREADS = 320;
constexpr int ST_INFO = 8;                          // tiles whose masks are kept
constexpr int ST_MAX_SLOTS = 8;
static_assert(ST_INFO >= ST_MAX_SLOTS / 2 + 2, "the copying warp is at most so many tiles ahead of a softmax");
constexpr int ST_MAX_SESSIONS = 1024;               // of one launch: their tile counts lie in shared memory
constexpr int ST_MAX_CTAS = 148;
constexpr uint32_t ST_COL_O = 256;

struct StShared {
    uint64_t full[ST_MAX_SLOTS], empty[ST_MAX_SLOTS];
    uint64_t info_full[ST_INFO];
    uint64_t s_full[2], p_full[2], o_done[2];       // by group: logits complete; P written, O rescaled; the fragment's last P . V done
    uint64_t q_full, drain;
    uint64_t left;                                  // both groups are through with a fragment
    uint32_t partial[ST_INFO];                      // whether some key of the tile does not count
    uint32_t mask[ST_INFO][4];
    uint32_t tmem_base, abort;
    int warp_sums[33];
    int32_t own_base[ST_MAX_SESSIONS + 1];          // tiles of the sessions before, per kv head
};

template <int DQK, int DV>
struct StShape {
    static constexpr int KT = DQK > 128 ? 64 : 128;                   // keys of a tile
    static constexpr int QA = DQK / 64, VA = DV / 64;                 // atoms of 64 dims
    static constexpr int Q_BYTES = 2 * ST_ROWS * DQK * 2, K_BYTES = KT * DQK * 2, V_BYTES = KT * DV * 2;
    static constexpr int SLOT = K_BYTES > V_BYTES ? K_BYTES : V_BYTES;
    static constexpr int ROOM = (227 * 1024 - static_cast<int>(sizeof(StShared)) - Q_BYTES) / SLOT;
    static constexpr int SLOTS = ROOM < ST_MAX_SLOTS ? ROOM : ST_MAX_SLOTS;
    static_assert(SLOTS >= 4, "K and V of a tile, and of the next");
    static constexpr int SMEM = Q_BYTES + SLOTS * SLOT + static_cast<int>(sizeof(StShared));
};

struct StParams {
    const uint16_t* q;
    int B, H_q, n_kv, group;
    int own_rows, own_parts;             // rows of an own segment, and how many cover a group
    int page_size, page_shift, box, n_phys;
    const int32_t* prefix_table;
    const int32_t* page_tables;
    const int64_t* table_offsets;
    const int64_t* kv_lens;
    int64_t prefix, own_start, max_len;  // own_start: where the tiles of the own tokens begin, prefix rounded down to a box
    int64_t prefix_tiles, prefix_units;  // of a segment; of all segments
    int prefix_segments, heavy_segments; // the first ones have more than 128 rows
    float scale_log2e;
    float *pre_o, *own_o;                // [place][256][d_v], [place][2][own_rows][d_v]
    float2 *pre_ml, *own_ml;             // maximum and sum, in the same places
    int32_t* own_base;                   // for the merge
    int n_ctas;
    uint16_t* out;
    float* lse;
    int32_t* dev_status;
};

// The line of tiles counts units: two for a tile of more than 128 rows, whose MMAs take twice the time.
constexpr int ST_HEAVY_UNITS = 2;

struct StFragment {
    bool prefix, heavy;
    int h;                 // kv head
    int row0;              // first row: of all rows (prefix), of the group (own)
    int rows;
    int b;                 // session (own)
    int64_t t0, t1;        // tiles of the segment
    int64_t place;
};

// First tile of a segment of `w` units a tile that belongs to the stretch from unit u on; u0: the segment's first unit.
__device__ __forceinline__ int64_t st_tile(int64_t u, int64_t u0, int w) { return (u - u0 + w - 1) / w; }

__device__ __forceinline__ void st_prefix_segment(const StParams& p, int s, int64_t& u0, int& w) {
    const int64_t heavy_units = p.prefix_tiles * ST_HEAVY_UNITS;
    w = s < p.heavy_segments ? ST_HEAVY_UNITS : 1;
    u0 = s < p.heavy_segments ? s * heavy_units : p.heavy_segments * heavy_units + (s - p.heavy_segments) * p.prefix_tiles;
}

// Next fragment of the stretch [u, end) of CTA `cta`; false when there is none.
__device__ __forceinline__ bool st_next(const StParams& p, const int32_t* own_base, int cta, int64_t& u, int64_t end, StFragment& f) {
    while (u < end) {
        if (u < p.prefix_units) {
            const int64_t heavy_units = p.prefix_tiles * ST_HEAVY_UNITS, all_heavy = p.heavy_segments * heavy_units;
            const int s = static_cast<int>(u < all_heavy ? u / heavy_units : p.heavy_segments + (u - all_heavy) / p.prefix_tiles);
            int64_t u0;
            int w;
            st_prefix_segment(p, s, u0, w);
            const int64_t u1 = u0 + w * p.prefix_tiles, stop = end < u1 ? end : u1;
            f.prefix = true;
            f.heavy = w == ST_HEAVY_UNITS;
            f.h = s % p.n_kv;
            f.row0 = s / p.n_kv * 2 * ST_ROWS;
            f.rows = min(2 * ST_ROWS, p.B * p.group - f.row0);
            f.b = 0;
            f.t0 = st_tile(u, u0, w);
            f.t1 = st_tile(stop, u0, w);
            f.place = static_cast<int64_t>(cta) + s;
            u = stop;
            if (f.t0 < f.t1) return true;
        } else {
            const int parts = p.n_kv * p.own_parts;
            const int64_t v = u - p.prefix_units;
            int lo = 0, hi = p.B;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (static_cast<int64_t>(own_base[mid]) * parts <= v) lo = mid;
                else hi = mid;
            }
            const int tiles = own_base[lo + 1] - own_base[lo];
            const int64_t rest = v - static_cast<int64_t>(own_base[lo]) * parts;
            const int part = static_cast<int>(rest / tiles);
            f.prefix = f.heavy = false;
            f.h = part / p.own_parts;
            f.row0 = part % p.own_parts * ST_ROWS;
            f.rows = min(ST_ROWS, p.group - f.row0);
            f.b = lo;
            f.t0 = rest - static_cast<int64_t>(part) * tiles;
            f.t1 = min(static_cast<int64_t>(tiles), f.t0 + (end - u));
            f.place = static_cast<int64_t>(cta) + static_cast<int64_t>(lo) * parts + part;
            u += f.t1 - f.t0;
            return true;
        }
    }
    return false;
}

// Length of session b as it counts: 0 where the entry is empty or refused.
__device__ __forceinline__ int64_t st_length(const StParams& p, int b, bool& bad) {
    const int64_t len = ld_input(p.kv_lens + b);
    bad = len < 0 || (len > 0 && len < p.prefix) || len > p.max_len;
    return len > p.max_len ? p.max_len : len < p.prefix ? 0 : len;
}

__device__ __forceinline__ float st_exp2(float x) {   // ex2.approx: 2 ulp, exp2(-inf) = 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t st_pack_bf16x2(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}

template <int DQK, int DV>
__global__ void __launch_bounds__(ST_THREADS, 1) attn_shared_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                                                                    const __grid_constant__ StParams p) {
    using C = StShape<DQK, DV>;
    constexpr int KT = C::KT, SLOTS = C::SLOTS;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* q_smem = smem;                             // 2 x atoms of [128 rows x 128 B]
    unsigned char* ring = smem + C::Q_BYTES;                  // slots of atoms of [KT keys x 128 B]
    StShared* sh = reinterpret_cast<StShared*>(ring + SLOTS * C::SLOT);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float neg_inf = __int_as_float(0xff800000);

    if (threadIdx.x == 0) {
        for (int i = 0; i < SLOTS; ++i) { mbar_init(smem_u32(&sh->full[i]), 1); mbar_init(smem_u32(&sh->empty[i]), 1); }
        for (int i = 0; i < ST_INFO; ++i) mbar_init(smem_u32(&sh->info_full[i]), 1);
        for (int w = 0; w < 2; ++w) { mbar_init(smem_u32(&sh->s_full[w]), 1); mbar_init(smem_u32(&sh->p_full[w]), 4); mbar_init(smem_u32(&sh->o_done[w]), 1); }
        mbar_init(smem_u32(&sh->q_full), ST_SOFTMAX_WARPS);
        mbar_init(smem_u32(&sh->left), ST_SOFTMAX_WARPS);
        mbar_init(smem_u32(&sh->drain), 1);
        fence_mbar_init();
        prefetch_tensormap(&tmap_k);
        prefetch_tensormap(&tmap_v);
    }
    grid_wait();
    // tiles of every session's own tokens
    const int per = (p.B + ST_THREADS - 1) / ST_THREADS, b0 = min(static_cast<int>(threadIdx.x) * per, p.B), b1 = min(b0 + per, p.B);
    int mine = 0;
    for (int b = b0; b < b1; ++b) {
        bool bad;
        const int64_t len = st_length(p, b, bad);
        const int tiles = len > p.prefix ? static_cast<int>((len - p.own_start + KT - 1) / KT) : 0;
        sh->own_base[b] = tiles;
        mine += tiles;
        if (bad && blockIdx.x == 0) report(p.dev_status, JANUS_DEV_INDEX_OUT_OF_RANGE);
    }
    int own_tiles;
    int at = block_exclusive_scan<ST_THREADS>(mine, sh->warp_sums, &own_tiles);
    for (int b = b0; b < b1; ++b) {
        const int tiles = sh->own_base[b];
        sh->own_base[b] = at;
        if (blockIdx.x == 0) p.own_base[b] = at;
        at += tiles;
    }
    if (threadIdx.x == 0) {
        sh->own_base[p.B] = own_tiles;
        if (blockIdx.x == 0) p.own_base[p.B] = own_tiles;
        // misaligned shared memory, or an earlier CTA that gave up on a wait
        uint32_t flag = (smem_u32(smem) & 1023u) != 0u ? 1u : 0u;
        if (flag != 0u) report(p.dev_status, JANUS_DEV_WAIT_TIMEOUT);
        if (p.dev_status != nullptr && *reinterpret_cast<volatile int32_t*>(p.dev_status) == JANUS_DEV_WAIT_TIMEOUT) flag = 1u;
        sh->abort = flag;
    }
    __syncwarp();
    if (warp == ST_MMA_WARP) { tmem_alloc(smem_u32(&sh->tmem_base), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem_base;
    const int64_t units = p.prefix_units + static_cast<int64_t>(own_tiles) * p.n_kv * p.own_parts;
    const int cta = blockIdx.x;
    int64_t u = units * cta / p.n_ctas;
    const int64_t end = units * (cta + 1) / p.n_ctas;
    auto wait_warp = [](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(smem_u32(bar), parity)) != 0; };
    bool ok = true;
    StFragment f;

    if (sh->abort != 0u) {
        // nothing to do
    } else if (warp == ST_COPY_WARP) {
        // ================================================================== copies
        // Lane l sees to boxes l, l + 32, ... of a tile.  The pages of a tile are looked up while the one before is copied.
        constexpr int MOST = KT / 32;                       // boxes of a lane: a box of one key at least
        const int boxes = KT / p.box;
        uint32_t unit = 0u, tc = 0u;
        while (ok && st_next(p, sh->own_base, cta, u, end, f)) {
            int64_t len = p.prefix, base = 0, entries = 0;
            const int32_t* table = p.prefix_table;
            if (f.prefix) {
                entries = (p.prefix + p.page_size - 1) / p.page_size;
            } else {
                bool bad;
                len = st_length(p, f.b, bad);
                base = p.own_start;
                const int64_t t = ld_input(p.table_offsets + f.b);
                entries = t < 0 ? 0 : ld_input(p.table_offsets + f.b + 1) - t;
                table = p.page_tables + (t < 0 ? 0 : t);
            }
            int id[MOST], row[MOST];
            bool wanted[MOST];                               // some key of the box lies in the segment
            auto look_up = [&](int64_t t) {
#pragma unroll
                for (int j = 0; j < MOST; ++j) {
                    const int i = lane + 32 * j;
                    const int64_t pos = base + t * KT + static_cast<int64_t>(i) * p.box;
                    id[j] = -1;
                    row[j] = 0;
                    wanted[j] = i < boxes && t < f.t1 && pos < len && (f.prefix || pos + p.box > p.prefix);
                    if (wanted[j]) {
                        const uint32_t x = static_cast<uint32_t>(pos), e = p.page_shift >= 0 ? x >> p.page_shift : x / static_cast<uint32_t>(p.page_size);
                        row[j] = static_cast<int>(x - e * static_cast<uint32_t>(p.page_size));
                        if (static_cast<int64_t>(e) < entries) id[j] = ld_input(table + e);
                    }
                }
            };
            look_up(f.t0);
            for (int64_t t = f.t0; t < f.t1 && ok; ++t, ++tc) {
                int page[MOST], page_row[MOST];              // of this tile's boxes; a page past the last where there is nothing to read
                bool missing = false;
                const int64_t p0 = base + t * KT;
                const int lo = !f.prefix && p.prefix > p0 ? static_cast<int>(p.prefix - p0) : 0, hi = len - p0 < KT ? static_cast<int>(len - p0) : KT;
                uint32_t words[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int j = 0; j < MOST; ++j) {
                    const int i = lane + 32 * j;
                    const bool there = wanted[j] && id[j] >= 0 && id[j] < p.n_phys;
                    missing |= wanted[j] && !there;
                    page[j] = there ? id[j] : p.n_phys;
                    page_row[j] = row[j];
                    if (there)
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const int from = max(max(i * p.box, lo) - 32 * w, 0), to = min(min((i + 1) * p.box, hi) - 32 * w, 32);
                            if (from < to) words[w] |= (to - from == 32 ? 0xffffffffu : ((1u << (to - from)) - 1u) << from);
                        }
                }
                bool whole = true;
#pragma unroll
                for (int w = 0; w < KT / 32; ++w) {
                    words[w] = __reduce_or_sync(0xffffffffu, words[w]);
                    whole = whole && words[w] == 0xffffffffu;
                }
                if (missing) report(p.dev_status, JANUS_DEV_INDEX_OUT_OF_RANGE);
                if (lane == 0) {
                    const uint32_t n = tc % ST_INFO;
                    sh->partial[n] = whole ? 0u : 1u;
#pragma unroll
                    for (int w = 0; w < 4; ++w) sh->mask[n][w] = words[w];
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->info_full[tc % ST_INFO]));
                look_up(t + 1);
#pragma unroll
                for (int kv = 0; kv < 2 && ok; ++kv, ++unit) {
                    const uint32_t slot = unit % SLOTS;
                    ok = wait_warp(&sh->empty[slot], ((unit / SLOTS) & 1u) ^ 1u);
                    if (!ok) break;
                    const uint32_t dst = smem_u32(ring) + slot * C::SLOT, bar = smem_u32(&sh->full[slot]);
                    if (lane == 0) mbar_expect_tx(bar, kv == 0 ? C::K_BYTES : C::V_BYTES);
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < MOST; ++j) {
                        const int i = lane + 32 * j;
                        if (i >= boxes) continue;
#pragma unroll
                        for (int a = 0; a < (kv == 0 ? C::QA : C::VA); ++a)
                            tma_load_4d(dst + a * KT * 128 + i * p.box * 128, kv == 0 ? &tmap_k : &tmap_v, a * 64, page_row[j], f.h, page[j], bar);
                    }
                    __syncwarp();
                }
            }
        }
        // Nothing may be on its way into shared memory when the CTA leaves, also after a wait somewhere gave up.
        for (uint32_t n = unit > SLOTS ? unit - SLOTS : 0u; n < unit; ++n)
            if (!wait_warp(&sh->full[n % SLOTS], (n / SLOTS) & 1u)) break;
    } else if (warp == ST_MMA_WARP) {
        // ================================================================== MMA issue
        constexpr uint32_t idesc_qk = umma_idesc_major(1u, ST_ROWS, KT, 0u, 0u), idesc_pv = umma_idesc_major(1u, ST_ROWS, DV, 0u, 1u);
        const uint32_t q_lo = umma_desc_lo(smem_u32(q_smem), 16), k_lo = umma_desc_lo(smem_u32(ring), 16), v_lo = umma_desc_lo(smem_u32(ring), KT * 128);
        uint32_t tc = 0u, n_frag = 0u, n_p[2] = {0u, 0u};
        while (ok && st_next(p, sh->own_base, cta, u, end, f)) {
            const int64_t tiles = f.t1 - f.t0, steps = f.heavy ? 2 * tiles : tiles;
            ok = wait_warp(&sh->q_full, n_frag & 1u);
            if (!ok) break;
            tc_fence_after();
            // logits of step n: the group n & 1, tile n or n / 2
            auto logits = [&](int64_t n) {
                const uint32_t w = static_cast<uint32_t>(n & 1), un = 2 * (tc + static_cast<uint32_t>(f.heavy ? n >> 1 : n)), slot = un % SLOTS;
                if (!f.heavy || w == 0u) {
                    ok = wait_warp(&sh->full[slot], (un / SLOTS) & 1u);
                    if (!ok) return;
                    tc_fence_after();
                }
                if (elect_one()) {
                    const uint32_t a = q_lo + (f.heavy ? w * (C::QA * ST_ROWS * 128 >> 4) : 0u), b = k_lo + slot * (C::SLOT >> 4);
#pragma unroll
                    for (int i = 0; i < DQK / 16; ++i)
                        umma_bf16_ss(tmem + w * 128u, a + (i >> 2) * (ST_ROWS * 128 >> 4) + (i & 3) * 2, b + (i >> 2) * (KT * 128 >> 4) + (i & 3) * 2, idesc_qk, i > 0 ? 1u : 0u);
                    if (!f.heavy || w == 1u) umma_commit(smem_u32(&sh->empty[slot]));
                    umma_commit(smem_u32(&sh->s_full[w]));
                }
                __syncwarp();
            };
            logits(0);
            if (ok && steps > 1) logits(1);
            for (int64_t n = 0; n < steps && ok; ++n) {
                const uint32_t w = static_cast<uint32_t>(n & 1), un = 2 * (tc + static_cast<uint32_t>(f.heavy ? n >> 1 : n)) + 1, slot = un % SLOTS;
                ok = wait_warp(&sh->p_full[w], n_p[w] & 1u);
                if (ok && (!f.heavy || w == 0u)) ok = wait_warp(&sh->full[slot], (un / SLOTS) & 1u);
                if (!ok) break;
                ++n_p[w];
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t b = v_lo + slot * (C::SLOT >> 4);
#pragma unroll
                    for (int i = 0; i < KT / 16; ++i)
                        umma_bf16_ts(tmem + ST_COL_O + w * 128u, tmem + w * 128u + 8 * i, b + i * (2048 >> 4), idesc_pv, n > 1 || i > 0 ? 1u : 0u);
                    if (!f.heavy || w == 1u) umma_commit(smem_u32(&sh->empty[slot]));
                    if (n + 2 >= steps) umma_commit(smem_u32(&sh->o_done[w]));
                }
                __syncwarp();
                if (n + 2 < steps) logits(n + 2);
            }
            tc += static_cast<uint32_t>(tiles);
            ++n_frag;
        }
        if (!ok) {                                    // what was issued must be through before tensor memory is given back
            if (elect_one()) umma_commit(smem_u32(&sh->drain));
            __syncwarp();
            (void)wait_warp(&sh->drain, 0u);
        }
    } else {
        // ================================================================== softmax, output
        const uint32_t w = static_cast<uint32_t>(warp) >> 2;              // group
        const int r = threadIdx.x & 127;                                  // row of the group, lane of tensor memory
        const uint32_t lane_addr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16), s_col = lane_addr + w * 128u, o_col = lane_addr + ST_COL_O + w * 128u;
        uint32_t tc = 0u, n_s = 0u, n_o = 0u, n_frag = 0u;
        while (ok && st_next(p, sh->own_base, cta, u, end, f)) {
            const int64_t tiles = f.t1 - f.t0;
            const int rows = f.heavy ? min(max(f.rows - static_cast<int>(w) * ST_ROWS, 0), ST_ROWS) : f.rows;      // of this group
            // ---- queries: those of 128 rows by this group (by the first group where both have the same)
            if (f.heavy || w == 0u) {
                constexpr int CH = DQK / 8;                               // 16-byte chunks of a row
                for (int c = r; c < rows * CH; c += ST_ROWS) {
                    const int row = c / CH, col = c % CH;
                    int64_t src;
                    if (f.prefix) {
                        const int x = f.row0 + static_cast<int>(w) * ST_ROWS + row, b = x / p.group;
                        src = static_cast<int64_t>(b) * p.H_q + f.h * p.group + (x - b * p.group);
                    } else {
                        src = static_cast<int64_t>(f.b) * p.H_q + f.h * p.group + f.row0 + row;
                    }
                    const uint4 v = __ldcg(reinterpret_cast<const uint4*>(p.q + src * DQK) + col);
                    *reinterpret_cast<uint4*>(q_smem + (w * C::QA + (col >> 3)) * (ST_ROWS * 128) + row * 128 + (((col & 7) ^ (row & 7)) << 4)) = v;
                }
                fence_proxy_async();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->q_full));

            const int64_t first = f.heavy ? 0 : w, step = f.heavy ? 1 : 2;
            const bool busy = (warp & 3) * 32 < rows;                     // some row of this warp counts
            float m_ref = neg_inf, l_sum = 0.f;                           // reference maximum (scaled, log2) and sum of this row
            for (int64_t t = first; t < tiles; t += step) {
                const uint32_t tile = tc + static_cast<uint32_t>(t), n = tile % ST_INFO;
                // (the mask was left before the copies of the tile began: the second wait only makes it visible here)
                ok = wait_warp(&sh->s_full[w], n_s & 1u) && wait_warp(&sh->info_full[n], (tile / ST_INFO) & 1u);
                if (!ok) break;
                ++n_s;
                tc_fence_after();
                const bool partial = sh->partial[n] != 0u;
                if (busy) {
                    uint32_t x[KT / 32][32];
#pragma unroll
                    for (int c = 0; c < KT / 32; ++c) tmem_ld32_issue(s_col + 32 * c, x[c]);
#pragma unroll
                    for (int c = 0; c < KT / 32; ++c) tmem_ld_wait(x[c]);
                    if (partial) {
#pragma unroll
                        for (int c = 0; c < KT / 32; ++c) {
                            const uint32_t bits = sh->mask[n][c];
#pragma unroll
                            for (int j = 0; j < 32; ++j) x[c][j] = (bits >> j) & 1u ? x[c][j] : 0xff800000u;
                        }
                    }
                    float mx[4] = {neg_inf, neg_inf, neg_inf, neg_inf};
#pragma unroll
                    for (int j = 0; j < KT; j += 2) mx[(j >> 1) & 3] = fmax3(mx[(j >> 1) & 3], __uint_as_float(x[j >> 5][j & 31]), __uint_as_float(x[j >> 5][(j & 31) + 1]));
                    const float tile_max = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2e;
                    float corr = 1.f;
                    bool moved = false;
                    if (tile_max > m_ref + 8.f) {
                        moved = m_ref != neg_inf;
                        corr = moved ? st_exp2(m_ref - tile_max) : 1.f;
                        l_sum *= corr;
                        m_ref = tile_max;
                    }
                    // O is at rest: s_full stands for all MMAs issued before it, the last P . V of this group among them
                    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll 1
                        for (int c = 0; c < DV / 32; ++c) {
                            uint32_t o[32];
                            tmem_ld32_wait(o_col + 32 * c, o);
#pragma unroll
                            for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * corr);
                            tmem_st32_wait(o_col + 32 * c, o);
                        }
                    }
                    const float neg_m = m_ref == neg_inf ? 0.f : -m_ref;
                    const float2 sc2 = make_float2(p.scale_log2e, p.scale_log2e), nm2 = make_float2(neg_m, neg_m);
                    float2 sum[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                    for (int c = 0; c < KT / 64; ++c) {
                        uint32_t pk[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const float2 e = ffma2(make_float2(__uint_as_float(x[2 * c + (j >> 4)][2 * j & 31]), __uint_as_float(x[2 * c + (j >> 4)][(2 * j & 31) + 1])), sc2, nm2);
                            const float2 pr = make_float2(st_exp2(e.x), st_exp2(e.y));
                            pk[j] = st_pack_bf16x2(pr.x, pr.y);
                            sum[j & 3] = fadd2(sum[j & 3], pr);
                        }
                        tmem_st32_wait(s_col + 32 * c, pk);
                    }
                    const float2 s4 = fadd2(fadd2(sum[0], sum[1]), fadd2(sum[2], sum[3]));
                    l_sum += s4.x + s4.y;
                }
                if (partial) {
                    // rows of V that do not count: zeros, once they have landed
                    const uint32_t un = 2 * tile + 1, slot = un % SLOTS;
                    ok = wait_warp(&sh->full[slot], (un / SLOTS) & 1u);
                    if (!ok) break;
                    if (r < KT && ((sh->mask[n][r >> 5] >> (r & 31)) & 1u) == 0u)
#pragma unroll
                        for (int c = 0; c < C::VA * 8; ++c) *reinterpret_cast<uint4*>(ring + slot * C::SLOT + (c >> 3) * KT * 128 + r * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                    fence_proxy_async();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_full[w]));
            }
            if (!ok) break;
            // ---- what this fragment leaves
            const bool some = first < tiles;
            if (some) {
                ok = wait_warp(&sh->o_done[w], n_o & 1u);
                if (!ok) break;
                ++n_o;
                tc_fence_after();
            }
            const int64_t place = f.prefix ? f.place * 2 * ST_ROWS + w * ST_ROWS + r : (f.place * 2 + w) * p.own_rows + r;
            if (some && busy) {
                float4* dst = reinterpret_cast<float4*>((f.prefix ? p.pre_o : p.own_o) + place * DV);
#pragma unroll 1
                for (int c = 0; c < DV / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32_wait(o_col + 32 * c, o);
                    if (r < rows)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            dst[8 * c + j] = make_float4(__uint_as_float(o[4 * j]), __uint_as_float(o[4 * j + 1]), __uint_as_float(o[4 * j + 2]), __uint_as_float(o[4 * j + 3]));
                }
            }
            if (r < rows) (f.prefix ? p.pre_ml : p.own_ml)[place] = make_float2(m_ref, l_sum);
            tc += static_cast<uint32_t>(tiles);
            // a group without a tile in a fragment would run ahead and arrive on q_full for two fragments before the other has for one
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->left));
            ok = wait_warp(&sh->left, n_frag++ & 1u);
        }
    }
    if (!ok && lane == 0) report(p.dev_status, JANUS_DEV_WAIT_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == ST_MMA_WARP) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// ---- merge: a block per row, its warps take the row's fragments in turn
constexpr int SM_WARPS = 4;

template <int DV>
__global__ void __launch_bounds__(32 * SM_WARPS) attn_shared_merge_kernel(const __grid_constant__ StParams p) {
    constexpr int PER = DV / 32;
    grid_launch_next();
    grid_wait();
    __shared__ float acc_s[SM_WARPS][DV];
    __shared__ float red[SM_WARPS], l_s[SM_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row = blockIdx.x;
    const int b = static_cast<int>(row / p.H_q), hq = static_cast<int>(row - static_cast<int64_t>(b) * p.H_q), h = hq / p.group, g = hq - h * p.group;
    const float neg_inf = __int_as_float(0xff800000);
    bool bad;
    const int64_t len = st_length(p, b, bad);
    const int base0 = ld_input(p.own_base + b), base1 = ld_input(p.own_base + b + 1), all = ld_input(p.own_base + p.B);
    const int parts = p.n_kv * p.own_parts;
    const int64_t units = p.prefix_units + static_cast<int64_t>(all) * parts;
    // CTA whose stretch holds unit x
    auto cta_of = [&](int64_t x) {
        int64_t i = x * p.n_ctas / units;
        while (i + 1 < p.n_ctas && units * (i + 1) / p.n_ctas <= x) ++i;
        while (i > 0 && units * i / p.n_ctas > x) --i;
        return static_cast<int>(i);
    };
    // fragments of the prefix segment, then of the own one: the first CTA of each, how many, and groups with an output of this row
    int pre_cta = 0, n_pre = 0, pre_groups = 1, own_cta = 0, n_own = 0, seg = 0, pre_row = 0;
    int64_t own_seg = 0, seg_u0 = 0;
    int seg_w = 1;
    if (len > 0 && p.prefix > 0) {
        const int x = b * p.group + g;
        seg = x / (2 * ST_ROWS) * p.n_kv + h;
        pre_row = x % (2 * ST_ROWS);
        st_prefix_segment(p, seg, seg_u0, seg_w);
        pre_groups = seg_w == ST_HEAVY_UNITS ? 1 : 2;
        pre_cta = cta_of(seg_u0);
        n_pre = cta_of(seg_u0 + seg_w * p.prefix_tiles - 1) - pre_cta + 1;
    }
    if (base1 > base0) {
        const int part = h * p.own_parts + g / ST_ROWS;
        own_seg = static_cast<int64_t>(b) * parts + part;
        const int64_t u0 = p.prefix_units + static_cast<int64_t>(base0) * parts + static_cast<int64_t>(part) * (base1 - base0);
        own_cta = cta_of(u0);
        n_own = cta_of(u0 + (base1 - base0) - 1) - own_cta + 1;
    }
    const int n_a = n_pre * pre_groups, n = n_a + 2 * n_own;
    // maximum and sum of output i of the row (-inf, 0: none), and where it lies
    auto fragment = [&](int i, const float*& o) {
        if (i < n_a) {
            const int f = i / pre_groups, w = i - f * pre_groups, cta = pre_cta + f;
            int64_t from = units * cta / p.n_ctas, to = units * (cta + 1) / p.n_ctas;
            from = from > seg_u0 ? from : seg_u0;
            to = to < seg_u0 + seg_w * p.prefix_tiles ? to : seg_u0 + seg_w * p.prefix_tiles;
            if (st_tile(from, seg_u0, seg_w) >= st_tile(to, seg_u0, seg_w)) return make_float2(neg_inf, 0.f);      // no tile begins in its stretch
            const int64_t place = (static_cast<int64_t>(cta) + seg) * 2 * ST_ROWS + w * ST_ROWS + pre_row;
            o = p.pre_o + place * DV;
            return __ldcg(p.pre_ml + place);
        }
        const int f = (i - n_a) >> 1, w = (i - n_a) & 1, cta = own_cta + f;
        if (units * cta / p.n_ctas == units * (cta + 1) / p.n_ctas) return make_float2(neg_inf, 0.f);               // more CTAs than tiles
        const int64_t place = ((cta + own_seg) * 2 + w) * p.own_rows + g % ST_ROWS;
        o = p.own_o + place * DV;
        return __ldcg(p.own_ml + place);
    };
    float m = neg_inf;
    const float* o = nullptr;
    for (int i = threadIdx.x; i < n; i += 32 * SM_WARPS) m = fmaxf(m, fragment(i, o).x);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if (lane == 0) red[warp] = m;
    __syncthreads();
    m = red[0];
#pragma unroll
    for (int i = 1; i < SM_WARPS; ++i) m = fmaxf(m, red[i]);
    const float safe = m == neg_inf ? 0.f : m;
    float acc[PER] = {}, l = 0.f;
#pragma unroll 4
    for (int i = warp; i < n; i += SM_WARPS) {
        const float2 ml = fragment(i, o);
        if (ml.x == neg_inf && ml.y == 0.f) continue;      // nothing there (a sum that is not a number counts)
        const float f = st_exp2(ml.x - safe);
        l = fmaf(f, ml.y, l);
        if constexpr (PER == 4) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(o) + lane);
            acc[0] = fmaf(f, v.x, acc[0]); acc[1] = fmaf(f, v.y, acc[1]); acc[2] = fmaf(f, v.z, acc[2]); acc[3] = fmaf(f, v.w, acc[3]);
        } else {
            const float2 v = __ldcg(reinterpret_cast<const float2*>(o) + lane);
            acc[0] = fmaf(f, v.x, acc[0]); acc[1] = fmaf(f, v.y, acc[1]);
        }
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) acc_s[warp][lane * PER + e] = acc[e];
    if (lane == 0) l_s[warp] = l;
    __syncthreads();
    if (warp == 0) {
        l = 0.f;
#pragma unroll
        for (int i = 0; i < SM_WARPS; ++i) l += l_s[i];
        const float inv = l != 0.f ? 1.f / l : 0.f;        // (a NaN is a sum)
        uint32_t wd[PER / 2];
#pragma unroll
        for (int e = 0; e < PER; e += 2) {
            float x = 0.f, y = 0.f;
#pragma unroll
            for (int i = 0; i < SM_WARPS; ++i) { x += acc_s[i][lane * PER + e]; y += acc_s[i][lane * PER + e + 1]; }
            wd[e / 2] = st_pack_bf16x2(x * inv, y * inv);
        }
        if constexpr (PER == 4) *reinterpret_cast<uint2*>(p.out + row * DV + lane * PER) = make_uint2(wd[0], wd[1]);
        else *reinterpret_cast<uint32_t*>(p.out + row * DV + lane * PER) = wd[0];
        if (p.lse != nullptr && lane == 0) p.lse[row] = l != 0.f ? (safe + log2f(l)) * 0.6931471805599453f : neg_inf;
    }
}

// ---- host
bool attn_shared_tc_supported(int d_qk, int d_v) { return (d_qk == 64 || d_qk == 128 || d_qk == 192) && (d_v == 64 || d_v == 128); }

// Places of the fragments, and what they take of the workspace.
struct StLayout {
    int64_t row_tiles, prefix_segments, pre_places, own_places;
    int own_rows, own_parts;
    size_t own_base, pre_ml, own_ml, pre_o, own_o, bytes;      // byte offsets
};

static StLayout st_layout(int B, int H_q, int n_kv, int d_v, int64_t prefix, int64_t max_len) {
    StLayout l;
    const int group = H_q / n_kv;
    l.own_rows = group < ST_ROWS ? group : ST_ROWS;
    l.own_parts = (group + ST_ROWS - 1) / ST_ROWS;
    l.row_tiles = (static_cast<int64_t>(B) * group + 2 * ST_ROWS - 1) / (2 * ST_ROWS);
    l.prefix_segments = prefix > 0 ? l.row_tiles * n_kv : 0;
    l.pre_places = prefix > 0 ? l.prefix_segments + ST_MAX_CTAS : 0;
    l.own_places = max_len > prefix ? static_cast<int64_t>(B) * n_kv * l.own_parts + ST_MAX_CTAS : 0;
    size_t at = 0;
    auto take = [&](size_t n) { const size_t x = at; at += (n + 127) & ~static_cast<size_t>(127); return x; };
    l.own_base = take(sizeof(int32_t) * (static_cast<size_t>(B) + 1));
    l.pre_ml = take(sizeof(float2) * l.pre_places * 2 * ST_ROWS);
    l.own_ml = take(sizeof(float2) * l.own_places * 2 * l.own_rows);
    l.pre_o = take(sizeof(float) * l.pre_places * 2 * ST_ROWS * d_v);
    l.own_o = take(sizeof(float) * l.own_places * 2 * l.own_rows * d_v);
    l.bytes = at;
    return l;
}

size_t attn_shared_tc_workspace(int B, int H_q, int n_kv, int d_v, int64_t prefix, int64_t max_len) {
    return st_layout(B < ST_MAX_SESSIONS ? B : ST_MAX_SESSIONS, H_q, n_kv, d_v, prefix, max_len).bytes;
}

// Pool [pages, page_size, heads, d] as a 4-D tensor (d, token, head, page); boxes of 64 dims x `box` tokens.
static bool st_tmap(CUtensorMap* map, const void* base, int d, int page_size, int heads, int64_t pages, int64_t page_stride, int64_t tok_stride, int64_t head_stride, int box) {
    PFN_encodeTiled enc = get_encode_tiled();
    if (enc == nullptr) return false;
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(page_size), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(pages > 0 ? pages : 1)};
    // (the stride of an axis of one does not matter, but is looked at)
    const cuuint64_t strides[3] = {static_cast<cuuint64_t>(page_size > 1 ? tok_stride * 2 : 16), static_cast<cuuint64_t>(heads > 1 ? head_stride * 2 : 16),
                                   static_cast<cuuint64_t>(pages > 1 ? page_stride * 2 : 16)};
    const cuuint32_t boxes[4] = {64, static_cast<cuuint32_t>(box), 1, 1}, estr[4] = {1, 1, 1, 1};
    if (current_context_id() == 0) {      // the encoder is a driver call and wants a context on this thread
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || cudaSetDevice(dev) != cudaSuccess) return false;
    }
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, boxes, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DQK, int DV>
static int st_launch(const SharedAttnArgs& a, StParams p, cudaStream_t stream) {
    using C = StShape<DQK, DV>;
    static_assert(C::SMEM <= 227 * 1024, "shared memory");
    static once_per_context larger;
    JANUS_CUDA_CHECK(larger.run([] { return cudaFuncSetAttribute(attn_shared_kernel<DQK, DV>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM); }));
    int dev = 0, sms = 0;
    JANUS_CUDA_CHECK(cudaGetDevice(&dev));
    JANUS_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    // the tallest box that lies within a page and within a tile
    int box = 1;
    while (box < C::KT && p.page_size % (2 * box) == 0) box *= 2;
    p.box = box;
    CUtensorMap map_k, map_v;
    if (!st_tmap(&map_k, a.k_pool, DQK, p.page_size, p.n_kv, p.n_phys, a.k_page_stride, a.k_tok_stride, a.k_head_stride, box) ||
        !st_tmap(&map_v, a.v_pool, DV, p.page_size, p.n_kv, p.n_phys, a.v_page_stride, a.v_tok_stride, a.v_head_stride, box))
        return JANUS_ERR_CUDA;
    p.own_start = p.prefix / box * box;
    p.prefix_tiles = (p.prefix + C::KT - 1) / C::KT;
    const int64_t own_most = p.max_len > p.prefix ? (p.max_len - p.own_start + C::KT - 1) / C::KT : 0;
    for (int b = 0; b < a.B; b += ST_MAX_SESSIONS) {
        p.B = a.B - b < ST_MAX_SESSIONS ? a.B - b : ST_MAX_SESSIONS;
        if (own_most * p.B > INT32_MAX) return JANUS_ERR_UNSUPPORTED;
        const StLayout l = st_layout(p.B, p.H_q, p.n_kv, DV, p.prefix, p.max_len);
        unsigned char* ws = static_cast<unsigned char*>(a.ws);
        p.own_base = reinterpret_cast<int32_t*>(ws + l.own_base);
        p.pre_ml = reinterpret_cast<float2*>(ws + l.pre_ml);
        p.own_ml = reinterpret_cast<float2*>(ws + l.own_ml);
        p.pre_o = reinterpret_cast<float*>(ws + l.pre_o);
        p.own_o = reinterpret_cast<float*>(ws + l.own_o);
        p.own_rows = l.own_rows;
        p.own_parts = l.own_parts;
        p.prefix_segments = static_cast<int>(l.prefix_segments);
        const int64_t last_rows = static_cast<int64_t>(p.B) * p.group - (l.row_tiles - 1) * 2 * ST_ROWS;
        p.heavy_segments = p.prefix > 0 ? static_cast<int>((l.row_tiles - (last_rows > ST_ROWS ? 0 : 1)) * p.n_kv) : 0;
        p.prefix_units = (static_cast<int64_t>(p.heavy_segments) * ST_HEAVY_UNITS + (p.prefix_segments - p.heavy_segments)) * p.prefix_tiles;
        const int64_t most = p.prefix_units + own_most * p.B * p.n_kv * p.own_parts;
        const int ctas = sms < ST_MAX_CTAS ? sms : ST_MAX_CTAS;
        p.n_ctas = static_cast<int>(most < 1 ? 1 : most < ctas ? most : ctas);
        p.q = static_cast<const uint16_t*>(a.q) + static_cast<int64_t>(b) * p.H_q * DQK;
        p.out = static_cast<uint16_t*>(a.out) + static_cast<int64_t>(b) * p.H_q * DV;
        p.lse = a.lse != nullptr ? a.lse + static_cast<int64_t>(b) * p.H_q : nullptr;
        p.kv_lens = a.kv_lens + b;
        p.table_offsets = a.table_offsets != nullptr ? a.table_offsets + b : nullptr;
        JANUS_CUDA_CHECK(launch_kernel(attn_shared_kernel<DQK, DV>, dim3(p.n_ctas), ST_THREADS, C::SMEM, stream, 1, map_k, map_v, p));
        JANUS_CUDA_CHECK(launch_kernel(attn_shared_merge_kernel<DV>, dim3(static_cast<unsigned>(p.B) * p.H_q), 32 * SM_WARPS, 0, stream, 1, p));
    }
    return JANUS_OK;
}

int launch_attn_shared_tc(const SharedAttnArgs& a, cudaStream_t stream) {
    StParams p = {};
    p.H_q = a.H_q; p.n_kv = a.n_kv_heads; p.group = a.H_q / a.n_kv_heads;
    p.page_size = a.page_size;
    p.page_shift = -1;
    if ((a.page_size & (a.page_size - 1)) == 0) {
        p.page_shift = 0;
        while ((1 << p.page_shift) < a.page_size) ++p.page_shift;
    }
    p.n_phys = static_cast<int>(a.n_phys_pages);
    p.prefix_table = a.prefix_table; p.page_tables = a.page_tables;
    p.prefix = a.prefix_len; p.max_len = a.max_len;
    p.scale_log2e = a.softmax_scale * 1.4426950408889634f;
    p.dev_status = a.dev_status;
    if (a.d_v == 64) {
        if (a.d_qk == 64) return st_launch<64, 64>(a, p, stream);
        if (a.d_qk == 128) return st_launch<128, 64>(a, p, stream);
        return st_launch<192, 64>(a, p, stream);
    }
    if (a.d_qk == 64) return st_launch<64, 128>(a, p, stream);
    if (a.d_qk == 128) return st_launch<128, 128>(a, p, stream);
    return st_launch<192, 128>(a, p, stream);
}

}  // namespace janus
