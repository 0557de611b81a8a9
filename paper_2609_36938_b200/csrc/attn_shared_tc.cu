// Dense attention of one query token per session over a shared prefix and each session's own tokens, on the tensor cores: keys of 64, 128 or
// 192 dims, values of 64 or 128, any grouping of heads.
//
//     out[b,h,:] = sum_s softmax_s(scale <q[b,h,:], K_s>) V_s     over the P shared tokens and session b's own ones
//
// Work.  The query heads of a session that share a kv head are a chunk of rows.  Two kinds of segment, cut into tiles of KT keys:
//   prefix   per kv head and up to 256 rows, whole chunks of several sessions: a tile of the prefix is read once for all of them.  With 128 dims and 256
//            rows a tile is 16.8 MFLOP against 64 KB and 2048 cycles of MMAs;
//   own      per session and kv head: one chunk, eight rows or so; a tile is read for it alone: HBM bounds it, and the rows of an MMA that stand empty
//            cost nothing (a tile takes 1000 cycles of MMAs, 2800 of an SM's share of HBM).
// All tiles form one line, and every CTA (one per SM, persistent) takes an equal stretch of it by weight, whatever the sessions' lengths: each part
// of a segment within a stretch is a fragment that leaves maxima, sums and unnormalised outputs in the workspace, and a second kernel merges the
// fragments of a row.  A fragment's place is (number of the CTA) + (number of the segment), which no two share and which
// follows from the lengths alone; so there are no counters, and the result does not depend on timing.
//
// A CTA: two groups of four softmax warps (thread = row), and a warp each that copies K and V, issues Q . K, issues P . V, and works out fragments and
// fetches their queries, ahead of the others.  With more than 128 rows each group has 128 of them and both work on every tile; with fewer,
// both have the same rows and take the tiles in turn, each with an output of its own.  Where rows are so few that there are lanes for four of each (32; two
// with tiles of 64 keys), each lane takes a slice of a tile's keys, and the lanes' outputs join through shared memory when the fragment ends.  K and V
// tiles come through one ring, in boxes of TMA that lie within a page (the box height divides page and tile); boxes of pages that are not there, or
// of tokens past the end, are out of the map's bounds and arrive as zeros.  Keys that do not count are masked by bits that the copying warp leaves; their
// rows of V are cleared, as 0 * NaN is not 0.
//
// The running maximum moves only when a tile exceeds it by more than 2^8, so O is rescaled a handful of times per fragment.  P is rounded to
// bf16 (half a step, 2^-8 relative, as the output itself); the row sum adds the probabilities as they were, so the log-sum-exp is exact to fp32.  Every
// wait is bounded; on a timeout the CTA reports JANUS_DEV_WAIT_TIMEOUT and leaves when its copies have landed.
//
// What bounds it now.  More than 128 rows: 4100 cycles a tile.  Tensor memory has room for one S beside both P and both O, so the logits of a group wait until
// the other has taken its own into registers (MMAs 900, as P . V of the other group runs between them, news of them 450, the load and news of that 660);
// softmax 2400 beside it.  96 sessions x 32 heads in 4 groups over 65536 tokens: 116 us (890 TFLOP/s), 130 in a row of thousands, as the power limit takes the
// clock from 1965 to some 1850 MHz.  Tiles of 80 keys, with room for two S and two P, cost the same handshakes more often: 162-174 us.  Logits handed over 64
// keys at a time, half of S computed while the other half is read: 116 us too, as an MMA of half the keys reads all of Q again.  One warp for all MMAs, with one S
// as here: 4100 cycles a tile as well; with each group's P over an S of its own: 3865, but own tokens at 5.3 TB/s (below).
// Fewer rows: HBM, 6.0 TB/s while tiles run (96 sessions' own tokens from 2048 to 4096: 67 us for 403 MB; P over S, an S for each group: 5.3), less with
// small pages, as a box costs the copying some 100 cycles (8192 own tokens of 37 sessions, 8 heads of their own: pages of 64 226 us, of 16 314, of 8 445).
// A fragment costs two to three us besides: the softmax of its last tile, P . V and the join are 1400 + 1000 + 2900 cycles.  One session of 3000 tokens: 14 us,
// of which this kernel 8, mostly the latencies of lengths, pages, first tile and instructions not yet in the cache, one after the other.
#include <type_traits>

#include "attn_shared.cuh"
#include "sm100_ptx.cuh"

namespace janus {

using namespace ptx;

constexpr int ST_ROWS = 128;                        // rows of an MMA
constexpr int ST_SOFTMAX_WARPS = 8, ST_COPY_WARP = 8, ST_QK_WARP = 9, ST_PV_WARP = 10, ST_QUERY_WARP = 11, ST_THREADS = 384;
constexpr int ST_READERS = ST_SOFTMAX_WARPS + 3;    // warps that fragments are worked out for
constexpr int ST_INFO = 8;                          // tiles whose masks are kept
constexpr int ST_MAX_SLOTS = 8;
static_assert(ST_INFO >= ST_MAX_SLOTS / 2 + 2, "the copying warp is at most so many tiles ahead of a softmax");
constexpr int ST_MAX_SESSIONS = 1024;               // of one launch: their tile counts lie in shared memory
constexpr int ST_MAX_CTAS = 148;
// Tensor memory: one S in columns [0, 128), P of group w in [128 + 64 w, ...), its O in [256 + 128 w, ...).  A group takes S into registers at once, so
// that the other group's logits are computed while it still works on these.
constexpr uint32_t ST_COL_S = 0, ST_COL_P = 128, ST_COL_O = 256;

constexpr int ST_FRAGMENTS = 4;                     // fragments that are worked out ahead
struct StFragment {
    int prefix, heavy, last;       // last: there is no further one, and this is none either
    int h;                 // kv head
    int c0;                // first chunk
    int rows;              // of the first 128, of the second
    int rows2;
    int b;                 // session (own)
    int t0, t1;            // tiles of the segment
    int64_t place;
};

constexpr int ST_JOIN = 20;                         // floats of a lane: 16 dims and a pad of 16 bytes, or more dims of fewer lanes

struct StShared {
    uint64_t full[ST_MAX_SLOTS], empty[ST_MAX_SLOTS];
    uint64_t info_full[ST_INFO];
    uint64_t s_full[2], s_free[2];                  // by group: logits complete; in registers
    uint64_t p_full[2], pv_done[2];                 // P written, O rescaled; P . V done
    uint64_t q_full[2], q_empty[2];                 // queries of 128 rows are there / their place is no longer needed
    uint64_t f_full[ST_FRAGMENTS], f_empty[ST_FRAGMENTS];      // fragment worked out / taken over by the warps that work on it
    uint64_t meet[2];                               // the warps of a group wait for one another
    uint64_t drain[2];
    uint32_t partial[ST_INFO];                      // whether some key of the tile does not count
    uint32_t mask[ST_INFO][4];
    StFragment fragment[ST_FRAGMENTS];
    uint32_t tmem_base;
    float2 ml[2][ST_ROWS];                          // by group: maxima and sums of the copies, to be joined,
    alignas(16) float join[2][ST_ROWS * ST_JOIN];   // and their outputs, some dims at a time
    int32_t own_base[ST_MAX_SESSIONS + 1];          // tiles of the sessions before, per kv head
};

template <int DQK, int DV>
struct StShape {
    static constexpr int KT = DQK > 128 ? 64 : 128;                   // keys of a tile
    static constexpr int QA = DQK / 64, VA = DV / 64;                 // atoms of 64 dims
    static constexpr int Q_BYTES = 2 * ST_ROWS * DQK * 2, K_BYTES = KT * DQK * 2, V_BYTES = KT * DV * 2;
    static constexpr int SLOT = K_BYTES > V_BYTES ? K_BYTES : V_BYTES;
    static constexpr int ROOM = (227 * 1024 - static_cast<int>(sizeof(StShared)) - Q_BYTES) / SLOT;
    // A multiple of four: K follows K in a slot, and V follows V of the group's own.  A barrier tells its phase from the one before only, so whoever waits
    // for a tile must have seen the last one in its slot land (with five slots, which keys of 64 and values of 128 have room for, K would follow a V
    // that the warp of Q . K never waits for).
    static constexpr int SLOTS = (ROOM < ST_MAX_SLOTS ? ROOM : ST_MAX_SLOTS) / 4 * 4;
    static_assert(SLOTS >= 4 && SLOTS % 4 == 0, "K and V of a tile, and of the next");
    static constexpr int Q_PLACE = Q_BYTES / 2;
    static constexpr int COPIES = KT / 32;                            // a row's keys are shared by so many lanes at most
    static constexpr int SMEM = Q_BYTES + SLOTS * SLOT + static_cast<int>(sizeof(StShared));
};

// A row's outputs in a segment: one from every fragment (more than 128 rows), or one from each group of every fragment.
struct alignas(8) SmPart {
    int n, row, step, unused;
    int64_t place;                       // of the first, in groups; step to the next
};

constexpr int SM_ROWS = 8, SM_THREADS = 256;      // rows of a block of the merge, its threads

struct StParams {
    const uint16_t* q;
    int B, H_q, n_kv, group;
    // The query heads of a session that share a kv head are a chunk of rows; more than 128 of them are several (parts).  128 rows of a prefix segment
    // hold so many whole chunks (per_tile).
    int chunk_rows, parts, per_tile, chunks;
    int page_size, page_shift, box, n_phys;
    const int32_t* prefix_table;
    const int32_t* page_tables;
    const int64_t* table_offsets;
    const int64_t* kv_lens;
    const uint16_t* v_pool;
    int64_t v_page_stride, v_tok_stride, v_head_stride;
    int64_t prefix, own_start, max_len;  // own_start: where the tiles of the own tokens begin, prefix rounded down to a box
    int prefix_tiles, prefix_units;      // tiles of a segment, units of all segments
    int heavy_segments;                  // the first ones have more than 128 rows
    float scale_log2e;
    float *pre_o, *own_o;                // [place][2][d_v / 4][rows][4], rows: 128, chunk_rows
    float2 *pre_ml, *own_ml;             // [place][2][rows]: maximum and sum
    SmPart* places;                      // for the merge: [kv head][row, filled up to SM_ROWS][prefix, own]
    int n_ctas;
    uint16_t* out;
    float* lse;
    int32_t* dev_status;
};

// The line counts units: so many for a tile of more than 128 rows, for one of fewer, and for what a segment costs besides its tiles.
constexpr int ST_HEAVY = 8, ST_LIGHT = 8, ST_SEGMENT = 6;

// Lanes that share the keys of a row: where rows are so few that there are lanes for `most` of each, every one takes a slice of a tile's keys, with a
// maximum, a sum and an output of its own until the fragment ends.  Lane i holds copy i / (128 / copies), row i % (128 / copies).
__device__ __forceinline__ int st_copies(bool heavy, int rows, int most) { return !heavy && rows <= ST_ROWS / most ? most : 1; }

__device__ __forceinline__ int st_units(int tiles, int w) { return tiles * w + ST_SEGMENT; }
// Tiles of a segment that begin before its unit x.
__device__ __forceinline__ int st_tiles(int x, int w) { return x <= ST_SEGMENT ? 0 : (x - ST_SEGMENT + w - 1) / w; }

// x / d for d > 0 and a quotient below 2^20; inv = 1 / d, rounded.
__device__ __forceinline__ int st_divide(int x, int d, float inv) {
    int q = __float2int_rd(__int2float_rn(x) * inv);
    const int r = x - q * d;
    if (r < 0) --q;
    if (r >= d) ++q;
    return q;
}

// First unit of prefix segment s, and the units of its tiles.
__device__ __forceinline__ int st_prefix_segment(const StParams& p, int s, int& w) {
    const int heavy = st_units(p.prefix_tiles, ST_HEAVY), light = st_units(p.prefix_tiles, ST_LIGHT);
    w = s < p.heavy_segments ? ST_HEAVY : ST_LIGHT;
    return s < p.heavy_segments ? s * heavy : p.heavy_segments * heavy + (s - p.heavy_segments) * light;
}

// Units that a CTA takes of `units` in all: a tile at least.
__device__ __forceinline__ int st_share(const StParams& p, int units) { return max(units > 0 ? (units - 1) / p.n_ctas + 1 : 1, p.heavy_segments > 0 ? ST_HEAVY : ST_LIGHT); }

// Next fragment of the stretch [u, end) of CTA `cta`; false when there is none.  It may be without a tile (none of the segment begins in the stretch).
__device__ __forceinline__ bool st_next(const StParams& p, const int32_t* own_base, int cta, int& u, int end, StFragment& f) {
    if (u < end) {
        int u0, w, tiles;
        if (u < p.prefix_units) {
            const int heavy = st_units(p.prefix_tiles, ST_HEAVY), all_heavy = p.heavy_segments * heavy;
            const int each = u < all_heavy ? heavy : st_units(p.prefix_tiles, ST_LIGHT), from = u < all_heavy ? 0 : all_heavy;
            const int s = st_divide(u - from, each, __frcp_rn(static_cast<float>(each))) + (u < all_heavy ? 0 : p.heavy_segments);
            const int tile = st_divide(s, p.n_kv, __frcp_rn(static_cast<float>(p.n_kv)));
            u0 = st_prefix_segment(p, s, w);
            tiles = p.prefix_tiles;
            f.prefix = true;
            f.heavy = s < p.heavy_segments;
            f.h = s - tile * p.n_kv;
            f.c0 = tile * 2 * p.per_tile;
            f.rows = min(p.per_tile, p.chunks - f.c0) * p.chunk_rows;
            f.rows2 = f.heavy ? min(p.per_tile, p.chunks - f.c0 - p.per_tile) * p.chunk_rows : 0;
            f.b = 0;
            f.place = static_cast<int64_t>(cta) + s;
        } else {
            const int parts = p.n_kv * p.parts, v = u - p.prefix_units;
            int lo = 0, hi = p.B;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (own_base[mid] * parts <= v) lo = mid;
                else hi = mid;
            }
            const int seg = own_base[lo + 1] - own_base[lo], part = st_divide(v - own_base[lo] * parts, seg, __frcp_rn(static_cast<float>(seg)));
            u0 = p.prefix_units + own_base[lo] * parts + part * seg;
            w = ST_LIGHT;
            tiles = (seg - ST_SEGMENT) / ST_LIGHT;
            f.prefix = f.heavy = false;
            f.h = p.parts == 1 ? part : part / p.parts;
            f.c0 = lo * p.parts + (part - f.h * p.parts);
            f.rows = p.chunk_rows;
            f.rows2 = 0;
            f.b = lo;
            f.place = static_cast<int64_t>(cta) + static_cast<int64_t>(lo) * parts + part;
        }
        const int stop = min(end, u0 + st_units(tiles, w));
        f.t0 = st_tiles(u - u0, w);
        f.t1 = st_tiles(stop - u0, w);
        u = stop;
        return true;
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
                                                                    const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_q_own,
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
        for (int w = 0; w < 2; ++w) { mbar_init(smem_u32(&sh->s_full[w]), 1); mbar_init(smem_u32(&sh->s_free[w]), 4); mbar_init(smem_u32(&sh->p_full[w]), 4); mbar_init(smem_u32(&sh->pv_done[w]), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&sh->q_full[i]), 1); mbar_init(smem_u32(&sh->q_empty[i]), 1); mbar_init(smem_u32(&sh->meet[i]), 4); mbar_init(smem_u32(&sh->drain[i]), 1); }
        for (int i = 0; i < ST_FRAGMENTS; ++i) { mbar_init(smem_u32(&sh->f_full[i]), 1); mbar_init(smem_u32(&sh->f_empty[i]), ST_READERS); }
        fence_mbar_init();
        prefetch_tensormap(&tmap_k);
        prefetch_tensormap(&tmap_v);
        prefetch_tensormap(&tmap_q_own);
    }
    grid_wait();
    if (warp == ST_QK_WARP) { tmem_alloc(smem_u32(&sh->tmem_base), 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    grid_launch_next();      // (tensor memory is allocated)
    tc_fence_after();
    const uint32_t tmem = sh->tmem_base;
    const int cta = blockIdx.x;
    auto wait_warp = [](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(smem_u32(bar), parity)) != 0; };
    bool ok = true;
    StFragment f;
    uint32_t n_fragment = 0u;
    // The next fragment, as the query warp has worked it out.
    auto next_fragment = [&]() {
        const uint32_t i = n_fragment % ST_FRAGMENTS;
        ok = wait_warp(&sh->f_full[i], (n_fragment / ST_FRAGMENTS) & 1u);
        if (!ok) return false;
        f = sh->fragment[i];
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh->f_empty[i]));
        ++n_fragment;
        return f.last == 0;
    };

    // registers: 256 x 208 + 128 x 88 = 384 x 168, what the block was launched with; a raise waits until so many have been given up
    auto more_registers = [] { asm volatile("setmaxnreg.inc.sync.aligned.u32 208;"); };
    auto fewer_registers = [] { asm volatile("setmaxnreg.dec.sync.aligned.u32 88;"); };
    if (warp >= ST_SOFTMAX_WARPS) {
    fewer_registers();      // all four warps: the softmax warps wait for what they give up
    if (warp == ST_COPY_WARP) {
        // ================================================================== copies
        // Lane l sees to boxes l, l + 32, ... of a tile.  The pages of the next tile, be it of the next fragment, are looked up between the copies of
        // K and of V.
        constexpr int MOST = KT / 32;                       // boxes of a lane: a box of one key at least
        const int boxes = KT / p.box;
        uint32_t unit = 0u, tc = 0u;
        int64_t len = 0, base = 0, entries = 0;             // of the fragment of the tile that was looked up last
        const int32_t* table = nullptr;
        int t = 0;
        bool more = true;
        int id[MOST], row[MOST];
        bool wanted[MOST];                                  // some key of the box lies in the segment
        f.t1 = 0;
        auto look_up = [&]() {                              // the tile after the last one
            if (++t >= f.t1) {
                do {
                    more = next_fragment();
                    if (!more) return;
                } while (f.t0 >= f.t1);
                t = f.t0;
                if (f.prefix) {
                    len = p.prefix;
                    base = 0;
                    entries = (p.prefix + p.page_size - 1) / p.page_size;
                    table = p.prefix_table;
                } else {
                    bool bad;
                    const int64_t from = ld_input(p.table_offsets + f.b), to = ld_input(p.table_offsets + f.b + 1);
                    len = st_length(p, f.b, bad);
                    base = p.own_start;
                    entries = from < 0 ? 0 : to - from;
                    table = p.page_tables + (from < 0 ? 0 : from);
                }
            }
#pragma unroll
            for (int j = 0; j < MOST; ++j) {
                const int i = lane + 32 * j;
                const int64_t pos = base + static_cast<int64_t>(t) * KT + static_cast<int64_t>(i) * p.box;
                id[j] = -1;
                row[j] = 0;
                wanted[j] = i < boxes && pos < len && (f.prefix || pos + p.box > p.prefix);
                if (wanted[j]) {
                    const uint32_t x = static_cast<uint32_t>(pos), e = p.page_shift >= 0 ? x >> p.page_shift : x / static_cast<uint32_t>(p.page_size);
                    row[j] = static_cast<int>(x - e * static_cast<uint32_t>(p.page_size));
                    if (static_cast<int64_t>(e) < entries) id[j] = ld_input(table + e);
                }
            }
        };
        look_up();
        for (; more && ok; ++tc) {
            int page[MOST], page_row[MOST];                 // of this tile's boxes; a page past the last where there is nothing to read
            bool missing = false;
            const int head = f.h;
            const int64_t p0 = base + static_cast<int64_t>(t) * KT;
            const int lo = !f.prefix && p.prefix > p0 ? static_cast<int>(p.prefix - p0) : 0, hi = len - p0 < KT ? static_cast<int>(len - p0) : KT;
            bool there[MOST], whole = lo == 0 && hi == KT;
#pragma unroll
            for (int j = 0; j < MOST; ++j) {
                there[j] = wanted[j] && id[j] >= 0 && id[j] < p.n_phys;
                missing |= wanted[j] && !there[j];
                page[j] = there[j] ? id[j] : p.n_phys;
                page_row[j] = row[j];
                whole = whole && (there[j] || lane + 32 * j >= boxes);
            }
            whole = __all_sync(0xffffffffu, whole) != 0;
            uint32_t words[KT / 32];
            if (!whole) {
#pragma unroll
                for (int w = 0; w < KT / 32; ++w) {
                    uint32_t bits = 0u;
#pragma unroll
                    for (int j = 0; j < MOST; ++j) {
                        const int i = lane + 32 * j, from = max(max(i * p.box, lo) - 32 * w, 0), to = min(min((i + 1) * p.box, hi) - 32 * w, 32);
                        if (there[j] && from < to) bits |= to - from == 32 ? 0xffffffffu : ((1u << (to - from)) - 1u) << from;
                    }
                    words[w] = __reduce_or_sync(0xffffffffu, bits);
                }
            }
            if (missing) report(p.dev_status, JANUS_DEV_INDEX_OUT_OF_RANGE);
            if (lane == 0) {
                const uint32_t n = tc % ST_INFO;
                sh->partial[n] = whole ? 0u : 1u;
                if (!whole)
#pragma unroll
                    for (int w = 0; w < KT / 32; ++w) sh->mask[n][w] = words[w];
                mbar_arrive(smem_u32(&sh->info_full[n]));
            }
            __syncwarp();
#pragma unroll
            for (int kv = 0; kv < 2 && ok; ++kv) {
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
                        tma_load_4d(dst + a * KT * 128 + i * p.box * 128, kv == 0 ? &tmap_k : &tmap_v, a * 64, page_row[j], head, page[j], bar);
                }
                __syncwarp();
                ++unit;
                if (kv == 0) look_up();
            }
        }
        // Nothing may be on its way into shared memory when the CTA leaves, also after a wait somewhere gave up.
        for (uint32_t n = unit > SLOTS ? unit - SLOTS : 0u; n < unit; ++n)
            if (!wait_warp(&sh->full[n % SLOTS], (n / SLOTS) & 1u)) break;
    } else if (warp == ST_QK_WARP) {
        // ================================================================== MMA issue: logits
        // Two warps issue MMAs, one Q . K and one P . V, each in the order of its own tiles (a wait costs a warp some 270 cycles, ready or not; one warp for
        // both took the same time a tile).  What they need of one another goes by barriers.
        constexpr uint32_t idesc = umma_idesc_major(1u, ST_ROWS, KT, 0u, 0u);
        const uint32_t q_lo = umma_desc_lo(smem_u32(q_smem), 16), k_lo = umma_desc_lo(smem_u32(ring), 16);
        uint32_t tc = 0u, n_q = 0u, n_free[2] = {0u, 0u}, light = 0u;       // phases of s_free by group; steps of fragments of 128 rows at most
        int before = -1;                                                    // group of the step before
        while (ok && next_fragment()) {
            const int tiles = f.t1 - f.t0, steps = f.heavy ? 2 * tiles : tiles;
            if (tiles == 0) continue;
            const uint32_t turn = f.heavy ? 0u : light & 1u;      // the group that has the first tile: they take turns across fragments
            for (int n = 0; n < steps && ok; ++n) {       // step n: group n & 1, tile n / 2; or group (n + turn) & 1, tile n
                const uint32_t w = static_cast<uint32_t>(n + turn) & 1u, un = 2 * (tc + static_cast<uint32_t>(f.heavy ? n >> 1 : n)), slot = un % SLOTS;
                const uint32_t use = n_q + (f.heavy ? w : 0u);
                if (n == 0 || (f.heavy && n == 1)) ok = wait_warp(&sh->q_full[use & 1u], (use >> 1) & 1u);
                if (ok && (!f.heavy || w == 0u)) ok = wait_warp(&sh->full[slot], (un / SLOTS) & 1u);
                if (ok && before >= 0) ok = wait_warp(&sh->s_free[before], n_free[before]++ & 1u);      // the logits before are in registers
                before = static_cast<int>(w);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t a = q_lo + (use & 1u) * (C::QA * ST_ROWS * 128 >> 4), b = k_lo + slot * (C::SLOT >> 4), d = tmem + ST_COL_S;
#pragma unroll
                    for (int i = 0; i < DQK / 16; ++i)
                        umma_bf16_ss(d, a + (i >> 2) * (ST_ROWS * 128 >> 4) + (i & 3) * 2, b + (i >> 2) * (KT * 128 >> 4) + (i & 3) * 2, idesc, i > 0 ? 1u : 0u);
                    if (!f.heavy || w == 1u) umma_commit(smem_u32(&sh->empty[slot]));
                    umma_commit(smem_u32(&sh->s_full[w]));
                    if (f.heavy ? n + 2 >= steps : n + 1 == steps) umma_commit(smem_u32(&sh->q_empty[use & 1u]));
                }
                __syncwarp();
            }
            light += f.heavy ? 0u : static_cast<uint32_t>(steps);
            tc += static_cast<uint32_t>(tiles);
            n_q += f.heavy ? 2u : 1u;
        }
        if (!ok) {                                    // what was issued must be through before tensor memory is given back
            if (elect_one()) umma_commit(smem_u32(&sh->drain[0]));
            __syncwarp();
            (void)wait_warp(&sh->drain[0], 0u);
        }
    } else if (warp == ST_PV_WARP) {
        // ================================================================== MMA issue: outputs
        constexpr uint32_t idesc = umma_idesc_major(1u, ST_ROWS, DV, 0u, 1u);
        const uint32_t v_lo = umma_desc_lo(smem_u32(ring), KT * 128);
        uint32_t tc = 0u, n_p[2] = {0u, 0u}, light = 0u;
        while (ok && next_fragment()) {
            const int tiles = f.t1 - f.t0, steps = f.heavy ? 2 * tiles : tiles;
            const uint32_t turn = f.heavy ? 0u : light & 1u;
            for (int n = 0; n < steps && ok; ++n) {
                const uint32_t w = static_cast<uint32_t>(n + turn) & 1u, un = 2 * (tc + static_cast<uint32_t>(f.heavy ? n >> 1 : n)) + 1, slot = un % SLOTS;
                if (!f.heavy || w == 0u) ok = wait_warp(&sh->full[slot], (un / SLOTS) & 1u);
                ok = ok && wait_warp(&sh->p_full[w], n_p[w]++ & 1u);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t b = v_lo + slot * (C::SLOT >> 4), a = tmem + ST_COL_P + w * 64u, d = tmem + ST_COL_O + w * 128u;
#pragma unroll
                    for (int i = 0; i < KT / 16; ++i) umma_bf16_ts(d, a + 8 * i, b + i * (2048 >> 4), idesc, n > 1 || i > 0 ? 1u : 0u);
                    if (!f.heavy || w == 1u) umma_commit(smem_u32(&sh->empty[slot]));
                    umma_commit(smem_u32(&sh->pv_done[w]));
                }
                __syncwarp();
            }
            light += f.heavy ? 0u : static_cast<uint32_t>(tiles);
            tc += static_cast<uint32_t>(tiles);
        }
        if (!ok) {
            if (elect_one()) umma_commit(smem_u32(&sh->drain[1]));
            __syncwarp();
            (void)wait_warp(&sh->drain[1], 0u);
        }
    } else if (warp == ST_QUERY_WARP) {
        // ================================================================== fragments, and their queries, ahead of the other warps
        // Two places of 128 rows: a fragment of more rows takes both, others take them in turn.  Rows that a chunk or a segment does not have hold
        // whatever comes; nothing is read of what becomes of them.
        uint32_t n_q = 0u;
        // units of every session's own tokens, per part of its heads: a lane adds up its own consecutive sessions, then the lanes' sums are scanned
        const int per = (p.B + 31) / 32, b0 = min(lane * per, p.B), b1 = min(b0 + per, p.B);
        // (nothing is done where shared memory is misaligned, or an earlier CTA of the launch gave up on a wait)
        const int32_t status = p.dev_status != nullptr ? *reinterpret_cast<volatile int32_t*>(p.dev_status) : 0;
        int sum = 0;
        for (int b = b0; b < b1; ++b) {
            bool bad;
            const int64_t len = st_length(p, b, bad);
            const int n = len > p.prefix ? st_units(static_cast<int>((len - p.own_start + KT - 1) / KT), ST_LIGHT) : 0;
            sh->own_base[b] = n;
            sum += n;
            if (bad && blockIdx.x == 0) report(p.dev_status, JANUS_DEV_INDEX_OUT_OF_RANGE);
        }
        bool give_up = (smem_u32(smem) & 1023u) != 0u;
        if (give_up) report(p.dev_status, JANUS_DEV_WAIT_TIMEOUT);
        give_up = give_up || status == JANUS_DEV_WAIT_TIMEOUT;
        int before = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, before, d);
            if (lane >= d) before += y;
        }
        const int own_units = __shfl_sync(0xffffffffu, before, 31);
        before -= sum;
        for (int b = b0; b < b1; ++b) {
            const int n = sh->own_base[b];
            sh->own_base[b] = before;
            before += n;
        }
        if (lane == 0) sh->own_base[p.B] = own_units;
        __syncwarp();
        const int units = p.prefix_units + own_units * p.n_kv * p.parts, share = st_share(p, units);
        int u = min(static_cast<int64_t>(share) * cta, static_cast<int64_t>(units));
        const int end = __any_sync(0xffffffffu, give_up) ? u : min(static_cast<int64_t>(u) + share, static_cast<int64_t>(units));
        auto publish = [&]() {
            const bool more = st_next(p, sh->own_base, cta, u, end, f);
            const uint32_t i = n_fragment % ST_FRAGMENTS;
            ok = wait_warp(&sh->f_empty[i], ((n_fragment / ST_FRAGMENTS) & 1u) ^ 1u);
            if (!ok) return false;
            ++n_fragment;
            f.last = more ? 0 : 1;
            if (lane == 0) {
                sh->fragment[i] = f;
                mbar_arrive(smem_u32(&sh->f_full[i]));
            }
            __syncwarp();
            return more;
        };
        while (ok && publish()) {
            if (f.t0 >= f.t1) continue;
            const int copies = st_copies(f.heavy, f.rows, C::COPIES);
            for (int w = 0; w < (f.heavy ? 2 : 1) && ok; ++w, ++n_q) {
                ok = wait_warp(&sh->q_empty[n_q & 1u], ((n_q >> 1) & 1u) ^ 1u);
                if (!ok) break;
                const uint32_t dst = smem_u32(q_smem) + (n_q & 1u) * C::Q_PLACE, bar = smem_u32(&sh->q_full[n_q & 1u]);
                const int c = f.c0 + w * p.per_tile, b = c / p.parts, y = f.h * p.group + (c - b * p.parts) * ST_ROWS;
                if (f.prefix && copies == 1) {                // one box of 128 rows, as far as whole chunks go
                    if (elect_one()) {
                        mbar_expect_tx(bar, static_cast<uint32_t>(C::QA * 128 * p.chunk_rows * p.per_tile));
#pragma unroll
                        for (int a = 0; a < C::QA; ++a) tma_load_3d(dst + a * (ST_ROWS * 128), &tmap_q, a * 64, y, b, bar);
                    }
                } else {                                      // chunk by chunk, every copy
                    const int chunks = f.rows / p.chunk_rows;
                    if (lane == 0) mbar_expect_tx(bar, static_cast<uint32_t>(C::QA * 128 * f.rows * copies));
                    __syncwarp();
                    for (int i = lane; i < chunks * copies; i += 32) {
                        const int copy = i / chunks, j = i - copy * chunks;
#pragma unroll
                        for (int a = 0; a < C::QA; ++a)
                            tma_load_3d(dst + a * (ST_ROWS * 128) + (copy * (ST_ROWS / copies) + j * p.chunk_rows) * 128, &tmap_q_own, a * 64, y, b + j, bar);
                    }
                }
                __syncwarp();
            }
        }
        // Meanwhile, for the merge: where the outputs of the rows lie.  Every CTA takes some rows; a lane for a row's prefix segment, one for its own.
        const int x_rows = p.B * p.group, blocks = (x_rows + SM_ROWS - 1) / SM_ROWS, all = blocks * SM_ROWS * p.n_kv * 2;
        const float inv_share = __frcp_rn(static_cast<float>(share)), inv_group = __frcp_rn(static_cast<float>(p.group)), inv_rows = __frcp_rn(static_cast<float>(blocks * SM_ROWS));
        for (int i = cta * 32 + lane; i < all; i += p.n_ctas * 32) {
            SmPart part = {};
            const int h = st_divide(i >> 1, blocks * SM_ROWS, inv_rows), x = (i >> 1) - h * blocks * SM_ROWS, b = st_divide(x, p.group, inv_group), g = x - b * p.group;
            bool bad;
            if (x < x_rows && st_length(p, b, bad) > 0) {
                const int segments = p.n_kv * p.parts, sub = g / ST_ROWS, c = b * p.parts + sub;
                if ((i & 1) == 0 && p.prefix > 0) {
                    const int tile = st_divide(c, 2 * p.per_tile, __frcp_rn(static_cast<float>(2 * p.per_tile))), in_tile = c - tile * 2 * p.per_tile;
                    const int half = in_tile >= p.per_tile ? 1 : 0, s = tile * p.n_kv + h;
                    int w;
                    const int u0 = st_prefix_segment(p, s, w), first = st_divide(u0, share, inv_share);
                    part.n = st_divide(u0 + st_units(p.prefix_tiles, w) - 1, share, inv_share) - first + 1;
                    part.place = 2 * (static_cast<int64_t>(first) + s) + half;
                    part.step = 2;
                    if (s >= p.heavy_segments) { part.n *= 2; part.step = 1; }
                    part.row = (in_tile - half * p.per_tile) * p.chunk_rows + (g - sub * ST_ROWS);
                }
                const int base = sh->own_base[b], seg = sh->own_base[b + 1] - base;
                if ((i & 1) != 0 && seg > 0) {
                    const int k = h * p.parts + sub, u0 = p.prefix_units + base * segments + k * seg, first = st_divide(u0, share, inv_share);
                    part.n = 2 * (st_divide(u0 + seg - 1, share, inv_share) - first + 1);
                    part.place = 2 * (static_cast<int64_t>(first) + static_cast<int64_t>(b) * segments + k);
                    part.step = 1;
                    part.row = g - sub * ST_ROWS;
                }
            }
            p.places[i] = part;
        }
        // (what is on its way has landed before the CTA leaves, also after a wait somewhere gave up)
        for (uint32_t n = n_q > 2u ? n_q - 2u : 0u; n < n_q; ++n)
            if (!wait_warp(&sh->q_full[n & 1u], (n >> 1) & 1u)) break;
    }
    } else {
        // ================================================================== softmax, output
        more_registers();
        const uint32_t w = static_cast<uint32_t>(warp) >> 2;              // group
        const int r = threadIdx.x & 127;                                  // row of the group, lane of tensor memory
        const uint32_t lane_addr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16), o_col = lane_addr + ST_COL_O + w * 128u;
        uint32_t tc = 0u, n_s = 0u, n_pv = 0u, n_meet = 0u, light = 0u;
        auto meet = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->meet[w]));
            return wait_warp(&sh->meet[w], n_meet++ & 1u);
        };
        while (ok && next_fragment()) {
            const int tiles = f.t1 - f.t0, first = f.heavy ? 0 : static_cast<int>((w + light) & 1u), step = f.heavy ? 1 : 2;
            light += f.heavy ? 0u : static_cast<uint32_t>(tiles);
            const int rows = f.heavy && w == 1u ? f.rows2 : f.rows;                // of this group
            const int copies = st_copies(f.heavy, f.rows, C::COPIES), apart = ST_ROWS / copies, copy = r / apart, row = r - copy * apart;
            const bool busy = ((warp & 3) * 32) % apart < rows;           // some row of this warp counts
            const uint32_t s_col = lane_addr + ST_COL_S, p_col = lane_addr + ST_COL_P + w * 64u;
            float m_ref = neg_inf, l_sum = 0.f;                           // reference maximum (scaled, log2) and sum of this lane
            // One tile.  N: lanes that share a row's keys; this one has KT / N of them.  P is rounded to bf16, half a step (a second term costs
            // 512 cycles of MMAs a tile and the room for P beside S: 10 % of the time of own tokens).
            auto softmax = [&](auto copies_, bool rested, uint32_t info) {
                constexpr int N = decltype(copies_)::value, KEYS = KT / N, CHUNKS = KEYS / 32, COLS = KEYS / 2;
                uint32_t x[CHUNKS][32];
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) tmem_ld32_issue(s_col + copy * KEYS + 32 * c, x[c]);
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) tmem_ld_wait(x[c]);
                tc_fence_before();  // the logits are in registers: the next may be computed
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->s_free[w]));
                if (sh->partial[info] != 0u) {
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c) {
                        const uint32_t bits = sh->mask[info][copy * CHUNKS + c];
#pragma unroll
                        for (int j = 0; j < 32; ++j) x[c][j] = (bits >> j) & 1u ? x[c][j] : 0xff800000u;
                    }
                }
                float mx[4] = {neg_inf, neg_inf, neg_inf, neg_inf};
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int j = 0; j < 16; ++j) mx[j & 3] = fmax3(mx[j & 3], __uint_as_float(x[c][2 * j]), __uint_as_float(x[c][2 * j + 1]));
                const float tile_max = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2e;
                float corr = 1.f;
                bool moved = false;
                if (tile_max > m_ref + 8.f) {
                    moved = m_ref != neg_inf;
                    corr = moved ? st_exp2(m_ref - tile_max) : 1.f;
                    l_sum *= corr;
                    m_ref = tile_max;
                }
                const float neg_m = m_ref == neg_inf ? 0.f : -m_ref;
                const float2 sc2 = make_float2(p.scale_log2e, p.scale_log2e), nm2 = make_float2(neg_m, neg_m);
                float2 sum[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                constexpr int ST = COLS < 32 ? COLS : 32;                 // columns of a store
#pragma unroll
                for (int c = 0; c < COLS / ST; ++c) {
                    uint32_t pk[ST];
#pragma unroll
                    for (int j = 0; j < ST; ++j) {
                        const int k = 2 * (c * ST + j);
                        const float2 e = ffma2(make_float2(__uint_as_float(x[k >> 5][k & 31]), __uint_as_float(x[k >> 5][(k & 31) + 1])), sc2, nm2);
                        const float2 pr = make_float2(st_exp2(e.x), st_exp2(e.y));
                        pk[j] = st_pack_bf16x2(pr.x, pr.y);
                        sum[j & 3] = fadd2(sum[j & 3], pr);
                    }
                    if (c == 0) {
                        // the group's last P . V is done: its P may be overwritten, and O is at rest
                        if (!rested) ok = wait_warp(&sh->pv_done[w], n_pv++ & 1u);
                        if (!ok) return;
                        tc_fence_after();
                        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll 1
                            for (int d = 0; d < DV / 32; ++d) {
                                uint32_t o[32];
                                tmem_ld32_wait(o_col + 32 * d, o);
#pragma unroll
                                for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * corr);
                                tmem_st32_wait(o_col + 32 * d, o);
                            }
                        }
                    }
                    tmem_st_issue(p_col + copy * COLS + ST * c, pk);
                }
                if constexpr (N > 1) {
                    // the keys of the other copies do not count for this lane (0 * inf is NaN: the merge sees to that)
                    uint32_t zero[COLS];
#pragma unroll
                    for (int j = 0; j < COLS; ++j) zero[j] = 0u;
#pragma unroll
                    for (int i = 1; i < N; ++i) tmem_st_issue(p_col + ((copy + i) & (N - 1)) * COLS, zero);
                }
                tmem_st_wait();
                const float2 s4 = fadd2(fadd2(sum[0], sum[1]), fadd2(sum[2], sum[3]));
                l_sum += s4.x + s4.y;
            };
            for (int t = first; t < tiles; t += step) {
                const uint32_t tile = tc + static_cast<uint32_t>(t), n = tile % ST_INFO;
                // (the mask was left before the copies of the tile began: the second wait only makes it visible here)
                ok = wait_warp(&sh->s_full[w], n_s & 1u) && wait_warp(&sh->info_full[n], (tile / ST_INFO) & 1u);
                if (!ok) break;
                ++n_s;
                tc_fence_after();
                bool rested = t == first;                                 // the group's P . V of the tile before is known to be done
                if (sh->partial[n] != 0u) {
                    // Rows of V that do not count: zeros, once they have landed.  The slot held V of SLOTS / 2 tiles before, the group's own tile before
                    // with four slots: its P . V is waited for first, as a barrier does not tell this V's phase from the one before that V's.  (More slots
                    // leave tiles between; of the fragment before this one the group has waited for everything.)
                    if (!rested) ok = wait_warp(&sh->pv_done[w], n_pv++ & 1u);
                    if (!ok) break;
                    rested = true;
                    const uint32_t un = 2 * tile + 1, slot = un % SLOTS;
                    ok = wait_warp(&sh->full[slot], (un / SLOTS) & 1u);
                    if (!ok) break;
                    if (r < KT && ((sh->mask[n][r >> 5] >> (r & 31)) & 1u) == 0u)
#pragma unroll
                        for (int c = 0; c < C::VA * 8; ++c) *reinterpret_cast<uint4*>(ring + slot * C::SLOT + (c >> 3) * KT * 128 + r * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                    fence_proxy_async();
                }
                if (busy) {
                    if (copies == 1) softmax(std::integral_constant<int, 1>{}, rested, n);
                    else softmax(std::integral_constant<int, C::COPIES>{}, rested, n);
                } else {
                    if (lane == 0) mbar_arrive(smem_u32(&sh->s_free[w]));
                    if (!rested) ok = wait_warp(&sh->pv_done[w], n_pv++ & 1u);
                }
                if (!ok) break;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh->p_full[w]));
            }
            if (!ok) break;
            // ---- what this fragment leaves
            const bool some = first < tiles;
            if (some) {
                ok = wait_warp(&sh->pv_done[w], n_pv++ & 1u);
                if (!ok) break;
                tc_fence_after();
            }
            // (of a prefix fragment both groups have 128 rows: their own, or outputs of the same rows; of an own one each has chunk_rows)
            const int pitch = f.prefix ? ST_ROWS : p.chunk_rows;
            const int64_t place = f.place * 2 + w;
            float4* dst = reinterpret_cast<float4*>(f.prefix ? p.pre_o : p.own_o) + place * (DV / 4) * pitch;
            float2* dst_ml = (f.prefix ? p.pre_ml : p.own_ml) + place * pitch;
            if (!some) {
                if (r < rows) dst_ml[r] = make_float2(neg_inf, 0.f);
            } else if (copies == 1) {
                if (busy)
#pragma unroll 1
                    for (int c = 0; c < DV / 32; ++c) {
                        uint32_t o[32];
                        tmem_ld32_wait(o_col + 32 * c, o);
                        if (r < rows)
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                dst[(8 * c + j) * pitch + r] = make_float4(__uint_as_float(o[4 * j]), __uint_as_float(o[4 * j + 1]), __uint_as_float(o[4 * j + 2]), __uint_as_float(o[4 * j + 3]));
                    }
                if (r < rows) dst_ml[r] = make_float2(m_ref, l_sum);
            } else {
                // The copies of a row become one, through shared memory, in a fixed order: up to eight rows 64 dims at a time, more rows fewer.
                const int lanes = copies * rows, dims = lanes <= 32 ? 64 : lanes <= 64 ? 32 : 16, gap = dims + 4;
                float* const join = sh->join[w];
                float* const mine = join + (copy * rows + row) * gap;
                sh->ml[w][r] = make_float2(m_ref, l_sum);
                auto leave = [&](const auto& o, int at) {
#pragma unroll
                    for (int j = 0; j < static_cast<int>(sizeof(o) / 16); ++j) *reinterpret_cast<uint4*>(mine + at + 4 * j) = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                };
#pragma unroll 1
                for (int d0 = 0; d0 < DV && ok; d0 += dims) {
                    if (d0 > 0) ok = meet();                               // what was there has been added up
                    if (!ok) break;
                    if (dims == 64) {
                        uint32_t o[2][32];
                        tmem_ld32_issue(o_col + d0, o[0]);
                        tmem_ld32_issue(o_col + d0 + 32, o[1]);
                        tmem_ld_wait(o[0]);
                        tmem_ld_wait(o[1]);
                        if (row < rows) { leave(o[0], 0); leave(o[1], 32); }
                    } else {
#pragma unroll 1
                        for (int k = 0; k < dims; k += 16) {
                            uint32_t o[16];
                            tmem_ld16_wait(o_col + d0 + k, o);
                            if (row < rows) leave(o, k);
                        }
                    }
                    ok = meet();
                    if (!ok) break;
                    for (int e = r; e < dims / 4 * rows; e += ST_ROWS) {   // (four dims, row)
                        const int rr = e >> (dims == 64 ? 4 : dims == 32 ? 3 : 2), c4 = e & (dims / 4 - 1);
                        float m = neg_inf, l = 0.f;
                        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (int i = 0; i < C::COPIES; ++i) m = fmaxf(m, sh->ml[w][i * (ST_ROWS / C::COPIES) + rr].x);
                        const float safe = m == neg_inf ? 0.f : m;
#pragma unroll
                        for (int i = 0; i < C::COPIES; ++i) {
                            const float2 v = sh->ml[w][i * (ST_ROWS / C::COPIES) + rr];
                            const float4 x = *reinterpret_cast<const float4*>(join + (i * rows + rr) * gap + 4 * c4);
                            const float g = st_exp2(v.x - safe);
                            l = fmaf(g, v.y, l);
                            sum.x = fmaf(g, x.x, sum.x); sum.y = fmaf(g, x.y, sum.y); sum.z = fmaf(g, x.z, sum.z); sum.w = fmaf(g, x.w, sum.w);
                        }
                        dst[(d0 / 4 + c4) * pitch + rr] = sum;
                        if (d0 == 0 && c4 == 0) dst_ml[rr] = make_float2(m, l);
                    }
                }
                ok = ok && meet();                                         // (before the next fragment's)
                if (!ok) break;
            }
            tc += static_cast<uint32_t>(tiles);
        }
    }
    if (!ok && lane == 0) report(p.dev_status, JANUS_DEV_WAIT_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == ST_QK_WARP) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// ---- merge: a block takes eight rows that lie one behind the other in the segments (128 bytes of every output at a time); its threads are
// (row, four dims, share of the row's outputs), HERE fours of dims.  A thread loads maxima, sums and outputs of AT_ONCE fragments together.
__device__ __forceinline__ SmPart sm_load(const SmPart* p) {
    SmPart s;
    const int64_t a = ld_input(reinterpret_cast<const int64_t*>(p)), b = ld_input(reinterpret_cast<const int64_t*>(p) + 1);
    s.n = static_cast<int>(a); s.row = static_cast<int>(a >> 32); s.step = static_cast<int>(b);
    s.place = ld_input(reinterpret_cast<const int64_t*>(p) + 2);
    return s;
}

// Infinite values.  A weight of 0 in fp32 makes NaN of one: that of a key of another copy, or of one far below the largest.  Every weight is positive by the
// definition, so a sum whose weights are numbers is infinite where its column holds infinite values of one sign, and NaN where it holds both or a NaN; where finite
// values have overflowed it stays as it is.  So for rows with such a NaN the block reads its dims of the session's values again, all threads together: bits of dim d0 + i
// in found[i]: 1 infinity, 2 minus infinity, 4 NaN.  (Here and not in the attention kernel, where other warps would wait for it.)
template <int DIMS>
__device__ __noinline__ void st_not_finite(const StParams& p, int b, int h, int d0, uint32_t* found) {
    constexpr int LANES = DIMS / 8, TOKENS = SM_THREADS / LANES, AT_ONCE = 4;
    bool bad;
    const int64_t len = st_length(p, b, bad);
    int64_t table = 0, entries = 0;
    if (len > p.prefix) {
        table = ld_input(p.table_offsets + b);
        entries = table < 0 ? 0 : ld_input(p.table_offsets + b + 1) - table;
    }
    const int part = threadIdx.x % LANES;
    const uint16_t* const values = p.v_pool + h * p.v_head_stride + d0 + 8 * part;
    uint32_t bits = 0u;      // three of each of eight dims
    for (int64_t s0 = threadIdx.x / LANES; s0 < len; s0 += TOKENS * AT_ONCE) {
        int32_t id[AT_ONCE];
        uint4 x[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int64_t s = s0 + k * TOKENS, e = s / p.page_size;
            id[k] = -1;
            if (s < p.prefix) id[k] = ld_input(p.prefix_table + e);
            else if (s < len && e < entries) id[k] = ld_input(p.page_tables + table + e);
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            x[k] = make_uint4(0u, 0u, 0u, 0u);
            if (id[k] >= 0 && id[k] < p.n_phys) x[k] = ld_input(reinterpret_cast<const uint4*>(values + id[k] * p.v_page_stride + (s0 + k * TOKENS) % p.page_size * p.v_tok_stride));
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t v = w[j >> 1] >> (16 * (j & 1));
                if ((v & 0x7f80u) == 0x7f80u) bits |= ((v & 0x7fu) != 0u ? 4u : (v & 0x8000u) != 0u ? 2u : 1u) << (3 * j);
            }
        }
    }
    for (int j = 0; j < 8 && bits != 0u; ++j, bits >>= 3)
        if ((bits & 7u) != 0u) atomicOr(found + 8 * part + j, bits & 7u);
}
// The sum in place of a NaN.
__device__ __forceinline__ float st_not_finite_sum(float sum, uint32_t found) {
    return sum == sum || found == 0u || found > 2u ? sum : __int_as_float(found == 1u ? 0x7f800000 : 0xff800000);
}

template <int DV, int HERE, int SHARES, int AT_ONCE>
__global__ void __launch_bounds__(SM_THREADS) attn_shared_merge_kernel(const __grid_constant__ StParams p) {
    static_assert(SM_ROWS * HERE * SHARES == SM_THREADS, "a thread for every row, four dims, share");
    constexpr int CHUNKS = DV / 4;
    __shared__ uint32_t found[HERE * 4];
    grid_launch_next();
    __shared__ float2 ml_s[SHARES][SM_ROWS];
    __shared__ float4 acc_s[SHARES > 1 ? SHARES - 1 : 1][HERE][SM_ROWS];
    const int tid = threadIdx.x;
    const float neg_inf = __int_as_float(0xff800000);
    const float inv_group = __frcp_rn(static_cast<float>(p.group));
    const int x_rows = p.B * p.group, blocks = (x_rows + SM_ROWS - 1) / SM_ROWS, h = blockIdx.x / blocks, x0 = (blockIdx.x - h * blocks) * SM_ROWS;
    grid_wait();
    const int row = tid % SM_ROWS, here = tid / SM_ROWS % HERE, chunk = blockIdx.y * HERE + here, share = tid / (SM_ROWS * HERE);
    const SmPart pre = sm_load(p.places + (static_cast<int64_t>(blockIdx.x) * SM_ROWS + row) * 2), own = sm_load(p.places + (static_cast<int64_t>(blockIdx.x) * SM_ROWS + row) * 2 + 1);
    const int n = pre.n + own.n;
    const float2* const pre_ml = p.pre_ml + pre.place * ST_ROWS + pre.row;
    const float2* const own_ml = p.own_ml + own.place * p.chunk_rows + own.row;
    const float4* const pre_o = reinterpret_cast<const float4*>(p.pre_o) + (pre.place * CHUNKS + chunk) * ST_ROWS + pre.row;
    const float4* const own_o = reinterpret_cast<const float4*>(p.own_o) + (own.place * CHUNKS + chunk) * p.chunk_rows + own.row;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = neg_inf, l = 0.f;
    for (int i0 = share; i0 < n; i0 += SHARES * AT_ONCE) {
        float2 v[AT_ONCE];
        float4 o[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int i = i0 + k * SHARES, j = i - pre.n;
            v[k] = make_float2(neg_inf, 0.f);
            if (i < n) {
                const int64_t step = i < pre.n ? static_cast<int64_t>(pre.step) * i * ST_ROWS : static_cast<int64_t>(j) * p.chunk_rows;
                v[k] = __ldcg((i < pre.n ? pre_ml : own_ml) + step);
                o[k] = __ldcg((i < pre.n ? pre_o : own_o) + step * CHUNKS);      // (whatever it is where the fragment has left nothing)
            }
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) top = fmaxf(top, v[k].x);
        const float safe = top == neg_inf ? 0.f : top, old = st_exp2(m - safe);
        l *= old; acc.x *= old; acc.y *= old; acc.z *= old; acc.w *= old;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (v[k].x == neg_inf && v[k].y == 0.f) continue;      // (a sum that is not a number counts)
            const float f = st_exp2(v[k].x - safe);
            l = fmaf(f, v[k].y, l);
            acc.x = fmaf(f, o[k].x, acc.x); acc.y = fmaf(f, o[k].y, acc.y); acc.z = fmaf(f, o[k].z, acc.z); acc.w = fmaf(f, o[k].w, acc.w);
        }
        m = top;
    }
    if constexpr (SHARES > 1) {
        if (here == 0) ml_s[share][row] = make_float2(m, l);
        if (share > 0) acc_s[share - 1][here][row] = acc;
        __syncthreads();
        if (share == 0) {
            float top = m;
#pragma unroll
            for (int i = 1; i < SHARES; ++i) top = fmaxf(top, ml_s[i][row].x);
            const float safe = top == neg_inf ? 0.f : top, old = st_exp2(m - safe);
            l *= old; acc.x *= old; acc.y *= old; acc.z *= old; acc.w *= old;
#pragma unroll
            for (int i = 1; i < SHARES; ++i) {
                const float2 w = ml_s[i][row];
                const float4 x = acc_s[i - 1][here][row];
                const float f = st_exp2(w.x - safe);
                l = fmaf(f, w.y, l);
                acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
            }
            m = top;
        }
    }
    const int x = x0 + row, b = st_divide(x, p.group, inv_group);
    const bool mine = share == 0 && x < x_rows;
    const float inv = l != 0.f ? 1.f / l : 0.f;        // (a NaN is a sum)
    acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
    if (l == 0.f) acc = make_float4(0.f, 0.f, 0.f, 0.f);      // (whatever the values of keys are that have no weight)
    const bool open = mine && l == l && (acc.x != acc.x || acc.y != acc.y || acc.z != acc.z || acc.w != acc.w);
    if (__syncthreads_or(open))
        for (int i = 0; i < SM_ROWS && x0 + i < x_rows; ++i) {
            const int session = st_divide(x0 + i, p.group, inv_group);
            if (i > 0 && session == st_divide(x0 + i - 1, p.group, inv_group)) continue;
            if (!__syncthreads_or(open && b == session)) continue;
            if (tid < HERE * 4) found[tid] = 0u;
            __syncthreads();
            st_not_finite<HERE * 4>(p, session, h, static_cast<int>(blockIdx.y) * HERE * 4, found);
            __syncthreads();
            if (open && b == session) {
                acc.x = st_not_finite_sum(acc.x, found[4 * here]); acc.y = st_not_finite_sum(acc.y, found[4 * here + 1]);
                acc.z = st_not_finite_sum(acc.z, found[4 * here + 2]); acc.w = st_not_finite_sum(acc.w, found[4 * here + 3]);
            }
        }
    if (mine) {
        const int64_t out = static_cast<int64_t>(b) * p.H_q + h * p.group + (x - b * p.group);
        *reinterpret_cast<uint2*>(p.out + out * DV + 4 * chunk) = make_uint2(st_pack_bf16x2(acc.x, acc.y), st_pack_bf16x2(acc.z, acc.w));
        if (p.lse != nullptr && chunk == 0) p.lse[out] = l != 0.f ? ((m == neg_inf ? 0.f : m) + log2f(l)) * 0.6931471805599453f : neg_inf;
    }
}

// ---- host
bool attn_shared_tc_supported(int d_qk, int d_v) { return (d_qk == 64 || d_qk == 128 || d_qk == 192) && (d_v == 64 || d_v == 128); }

// Chunks of rows, places of the fragments, and what they take of the workspace.
struct StLayout {
    int chunk_rows, parts, per_tile;
    int64_t chunks, row_tiles, prefix_segments, pre_places, own_places;
    size_t merge_parts, pre_ml, own_ml, pre_o, own_o, bytes;   // byte offsets
};

static StLayout st_layout(int B, int H_q, int n_kv, int d_v, int64_t prefix, int64_t max_len) {
    StLayout l;
    const int group = H_q / n_kv;
    l.chunk_rows = group < ST_ROWS ? group : ST_ROWS;
    l.parts = (group + ST_ROWS - 1) / ST_ROWS;
    l.per_tile = ST_ROWS / l.chunk_rows;
    l.chunks = static_cast<int64_t>(B) * l.parts;
    l.row_tiles = (l.chunks + 2 * l.per_tile - 1) / (2 * l.per_tile);
    l.prefix_segments = prefix > 0 ? l.row_tiles * n_kv : 0;
    l.pre_places = prefix > 0 ? l.prefix_segments + ST_MAX_CTAS : 0;
    l.own_places = max_len > prefix ? l.chunks * n_kv + ST_MAX_CTAS : 0;
    size_t at = 0;
    auto take = [&](size_t n) { const size_t x = at; at += (n + 127) & ~static_cast<size_t>(127); return x; };
    l.merge_parts = take(2 * sizeof(SmPart) * n_kv * ((static_cast<size_t>(B) * group + SM_ROWS - 1) / SM_ROWS * SM_ROWS));
    l.pre_ml = take(sizeof(float2) * l.pre_places * 2 * ST_ROWS);
    l.own_ml = take(sizeof(float2) * l.own_places * 2 * l.chunk_rows);
    l.pre_o = take(sizeof(float) * l.pre_places * 2 * ST_ROWS * d_v);
    l.own_o = take(sizeof(float) * l.own_places * 2 * l.chunk_rows * d_v);
    l.bytes = at;
    return l;
}

size_t attn_shared_tc_workspace(int B, int H_q, int n_kv, int d_v, int64_t prefix, int64_t max_len) {
    return st_layout(B < ST_MAX_SESSIONS ? B : ST_MAX_SESSIONS, H_q, n_kv, d_v, prefix, max_len).bytes;
}

static bool st_encode(CUtensorMap* map, const void* base, int axes, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    PFN_encodeTiled enc = get_encode_tiled();
    if (enc == nullptr) return false;
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    if (current_context_id() == 0) {      // the encoder is a driver call and wants a context on this thread
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || cudaSetDevice(dev) != cudaSuccess) return false;
    }
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, axes, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Pool [pages, page_size, heads, d] as a 4-D tensor (d, token, head, page); boxes of 64 dims x `box` tokens.
static bool st_tmap(CUtensorMap* map, const void* base, int d, int page_size, int heads, int64_t pages, int64_t page_stride, int64_t tok_stride, int64_t head_stride, int box) {
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(page_size), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(pages > 0 ? pages : 1)};
    // (the stride of an axis of one does not matter, but is looked at)
    const cuuint64_t strides[3] = {static_cast<cuuint64_t>(page_size > 1 ? tok_stride * 2 : 16), static_cast<cuuint64_t>(heads > 1 ? head_stride * 2 : 16),
                                   static_cast<cuuint64_t>(pages > 1 ? page_stride * 2 : 16)};
    const cuuint32_t boxes[4] = {64, static_cast<cuuint32_t>(box), 1, 1};
    return st_encode(map, base, 4, dims, strides, boxes);
}

// Queries [sessions, heads, d]; boxes of 64 dims x a chunk x so many sessions.
static bool st_tmap_q(CUtensorMap* map, const void* base, int d, int heads, int sessions, int chunk_rows, int box_sessions) {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(sessions)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(d) * 2, static_cast<cuuint64_t>(d) * 2 * heads};
    const cuuint32_t boxes[3] = {64, static_cast<cuuint32_t>(chunk_rows), static_cast<cuuint32_t>(box_sessions)};
    return st_encode(map, base, 3, dims, strides, boxes);
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
    const int64_t prefix_tiles = (p.prefix + C::KT - 1) / C::KT, own_most = p.max_len > p.prefix ? (p.max_len - p.own_start + C::KT - 1) / C::KT : 0;
    const int ctas = sms < ST_MAX_CTAS ? sms : ST_MAX_CTAS;
    // so many sessions at a time that units count in 31 bits, however long the sessions turn out to be
    constexpr int64_t MOST_UNITS = 1 << 30;
    const StLayout most_l = st_layout(a.B < ST_MAX_SESSIONS ? a.B : ST_MAX_SESSIONS, p.H_q, p.n_kv, DV, p.prefix, p.max_len);
    const int64_t own_units = own_most > 0 ? (own_most * ST_LIGHT + ST_SEGMENT) * p.n_kv * most_l.parts : 0;
    const int64_t prefix_units = (prefix_tiles * ST_HEAVY + ST_SEGMENT) * most_l.prefix_segments;
    if (own_units > MOST_UNITS || prefix_units > MOST_UNITS) return JANUS_ERR_UNSUPPORTED;
    int at_once = ST_MAX_SESSIONS;
    if (own_units > 0 && MOST_UNITS / own_units < at_once) at_once = static_cast<int>(MOST_UNITS / own_units);
    for (int b = 0; b < a.B; b += at_once) {
        p.B = a.B - b < at_once ? a.B - b : at_once;
        const StLayout l = st_layout(p.B, p.H_q, p.n_kv, DV, p.prefix, p.max_len);
        unsigned char* ws = static_cast<unsigned char*>(a.ws);
        p.places = reinterpret_cast<SmPart*>(ws + l.merge_parts);
        p.pre_ml = reinterpret_cast<float2*>(ws + l.pre_ml);
        p.own_ml = reinterpret_cast<float2*>(ws + l.own_ml);
        p.pre_o = reinterpret_cast<float*>(ws + l.pre_o);
        p.own_o = reinterpret_cast<float*>(ws + l.own_o);
        p.chunk_rows = l.chunk_rows; p.parts = l.parts; p.per_tile = l.per_tile; p.chunks = static_cast<int>(l.chunks);
        const int64_t last = l.chunks - (l.row_tiles - 1) * 2 * l.per_tile;
        p.heavy_segments = p.prefix > 0 ? static_cast<int>((l.row_tiles - (last > l.per_tile ? 0 : 1)) * p.n_kv) : 0;
        p.prefix_tiles = static_cast<int>(prefix_tiles);
        p.prefix_units = static_cast<int>(p.heavy_segments * (prefix_tiles * ST_HEAVY + ST_SEGMENT) + (l.prefix_segments - p.heavy_segments) * (prefix_tiles * ST_LIGHT + ST_SEGMENT));
        const int64_t most = p.prefix_units + own_units * p.B;
        p.n_ctas = static_cast<int>(most < 1 ? 1 : most < ctas ? most : ctas);
        p.q = static_cast<const uint16_t*>(a.q) + static_cast<int64_t>(b) * p.H_q * DQK;
        p.out = static_cast<uint16_t*>(a.out) + static_cast<int64_t>(b) * p.H_q * DV;
        p.lse = a.lse != nullptr ? a.lse + static_cast<int64_t>(b) * p.H_q : nullptr;
        p.kv_lens = a.kv_lens + b;
        p.table_offsets = a.table_offsets != nullptr ? a.table_offsets + b : nullptr;
        CUtensorMap map_q, map_q_own;
        if (!st_tmap_q(&map_q, p.q, DQK, p.H_q, p.B, l.chunk_rows, l.per_tile) || !st_tmap_q(&map_q_own, p.q, DQK, p.H_q, p.B, l.chunk_rows, 1)) return JANUS_ERR_CUDA;
        JANUS_CUDA_CHECK(launch_kernel(attn_shared_kernel<DQK, DV>, dim3(p.n_ctas), ST_THREADS, C::SMEM, stream, 1, map_k, map_v, map_q, map_q_own, p));
        // Few rows have many outputs each: eight shares of them, and the dims in several blocks, as long as those are resident at once.  Many rows fill the
        // SMs with a block for eight rows.
        const int64_t blocks = (static_cast<int64_t>(p.B) * p.group + SM_ROWS - 1) / SM_ROWS * p.n_kv;
        if (blocks * (DV / 16) <= 4 * ST_MAX_CTAS) JANUS_CUDA_CHECK(launch_kernel(attn_shared_merge_kernel<DV, 4, 8, 4>, dim3(static_cast<unsigned>(blocks), DV / 16), SM_THREADS, 0, stream, 1, p));
        else JANUS_CUDA_CHECK(launch_kernel(attn_shared_merge_kernel<DV, DV / 4, 128 / DV, 8>, dim3(static_cast<unsigned>(blocks)), SM_THREADS, 0, stream, 1, p));
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
    p.v_pool = static_cast<const uint16_t*>(a.v_pool);
    p.v_page_stride = a.v_page_stride; p.v_tok_stride = a.v_tok_stride; p.v_head_stride = a.v_head_stride;
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
