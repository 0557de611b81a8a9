// Plan of a serving step: from the lengths of a batch of sessions to the page tables, rows, positions and cache places that the calls of the
// step take.  With c cached and n new tokens of session b, page size p, t = c + n:
//
//     pages of b = ceil(t / p), the first ceil(c / p) from its block table, the others from the free list, in order of b;
//     offsets    = exclusive sums of n and of the pages;      slot of position x = page[x / p] * p + x % p.
//
// What bounds it: latency.  A full server (1024 sessions of up to 131072 tokens, pages of 64) moves 5 MB; a batch of twelve a few KB.  So there is
// one launch and no step in it waits for another CTA: every CTA adds up the lengths of all sessions by itself (8 bytes a session and array, from
// L2) and keeps the three exclusive sums in shared memory, then all threads of the grid go over the table entries and over the rows, each
// finding its session by bisection of the sums (sessions differ in length by orders of magnitude; a warp per session would leave the longest
// to one warp).  A page that is taken from the free list is known from the sums alone, so a row never reads what another thread writes.
#include "batch_plan_rows.h"
#include "janus_common.cuh"

namespace janus {

constexpr int BP_THREADS = 512;
constexpr int BP_MAX_SESSIONS = 8192;       // three sums of 4 bytes each in shared memory

struct BpParams {
    const int64_t* cached;
    const int64_t* fresh;
    int B, page_size, page_shift;
    int32_t* block_tables;
    int64_t block_ld;
    int32_t width;
    const int32_t* free_pages;
    int64_t n_free, n_phys;
    const int64_t* key_offsets;
    int64_t *row_offsets, *kv_lens, *table_offsets;
    int32_t* page_tables;
    int64_t table_capacity;
    int32_t* row_sessions;
    int64_t *positions, *slots, *key_rows;
    int64_t max_rows;
    int64_t* counts;
    int32_t* dev_status;
};

struct BpSession {
    int64_t cached, rows, total;    // tokens in the cache, new ones, both as far as the block table's width holds them
    int32_t held, pages;            // pages that hold the cached tokens, all pages
    bool bad, over;                 // a negative length; more tokens than a row of the block table has room for
};

__device__ __forceinline__ int64_t bp_pages(const BpParams& p, int64_t tokens) {
    return p.page_shift >= 0 ? (tokens + p.page_size - 1) >> p.page_shift : (tokens + p.page_size - 1) / p.page_size;
}

__device__ __forceinline__ BpSession bp_session(const BpParams& p, int b) {
    BpSession s;
    int64_t c = ld_input(p.cached + b), n = ld_input(p.fresh + b);
    s.bad = c < 0 || n < 0;
    if (c < 0) c = 0;
    if (n < 0) n = 0;
    const int64_t room = static_cast<int64_t>(p.width) * p.page_size;
    s.over = c > room || n > room - (c < room ? c : room);
    s.cached = c < room ? c : room;
    s.rows = n < INT32_MAX ? n : INT32_MAX;      // (2^31 rows are more than any max_rows)
    s.total = s.over ? room : c + n;
    s.held = static_cast<int32_t>(bp_pages(p, s.cached));
    s.pages = static_cast<int32_t>(bp_pages(p, s.total));
    return s;
}

// Largest b with sums[b] <= x, for sums[0] = 0 <= x < sums[B] (of sessions that add nothing, the last before one that does).
__device__ __forceinline__ int bp_find(const int32_t* sums, int B, int64_t x) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(BP_THREADS) batch_plan_kernel(const BpParams p) {
    grid_launch_next();
    extern __shared__ __align__(16) int32_t bp_smem[];
    int32_t *row_sum = bp_smem, *page_sum = bp_smem + p.B + 1, *free_sum = bp_smem + 2 * (p.B + 1);
    __shared__ int64_t warp_sums[3][BP_THREADS / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    grid_wait();

    // ---- exclusive sums: every thread adds up its own consecutive sessions, then the threads' sums are scanned
    const int per = (p.B + BP_THREADS - 1) / BP_THREADS;
    const int b0 = min(tid * per, p.B), b1 = min(b0 + per, p.B);
    int64_t v[3] = {0, 0, 0};
    bool bad = false, over = false;
    for (int b = b0; b < b1; ++b) {
        const BpSession s = bp_session(p, b);
        v[0] += s.rows;
        v[1] += s.pages;
        v[2] += s.pages - s.held;
        bad |= s.bad;
        over |= s.over;
    }
    int64_t before[3], total[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        int64_t incl = v[i];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += y;
        }
        if (lane == 31) warp_sums[i][warp] = incl;
        before[i] = incl - v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        total[i] = 0;
        for (int w = 0; w < BP_THREADS / 32; ++w) {
            if (w < warp) before[i] += warp_sums[i][w];
            total[i] += warp_sums[i][w];
        }
    }
    // (the sums of pages are below 2^31: the host has checked the whole block table; those of rows count up to max_rows)
    const bool first = blockIdx.x == 0;
    for (int b = b0; b < b1; ++b) {
        const BpSession s = bp_session(p, b);
        const int64_t row = min(before[0], p.max_rows);
        row_sum[b] = static_cast<int32_t>(row);
        page_sum[b] = static_cast<int32_t>(before[1]);
        free_sum[b] = static_cast<int32_t>(before[2]);
        if (first) {
            p.row_offsets[b] = row;
            p.table_offsets[b] = min(before[1], p.table_capacity);
            p.kv_lens[b] = s.total;
        }
        before[0] += s.rows;
        before[1] += s.pages;
        before[2] += s.pages - s.held;
    }
    if (tid == 0) {
        row_sum[p.B] = static_cast<int32_t>(min(total[0], p.max_rows));
        page_sum[p.B] = static_cast<int32_t>(total[1]);
        free_sum[p.B] = static_cast<int32_t>(total[2]);
        if (first) {
            p.row_offsets[p.B] = min(total[0], p.max_rows);
            p.table_offsets[p.B] = min(total[1], p.table_capacity);
            p.counts[0] = total[2];
            p.counts[1] = total[1];
            p.counts[2] = total[0];
            if (total[2] > p.n_free || total[1] > p.table_capacity || total[0] > p.max_rows) over = true;
        }
    }
    if (first && bad) report(p.dev_status, JANUS_DEV_INDEX_OUT_OF_RANGE);
    if (first && over) report(p.dev_status, JANUS_DEV_CAPACITY_EXCEEDED);
    __syncthreads();

    // page j of session b as it stands in the block table or the free list; INT32_MIN where the free list has ended
    auto load_page = [&](int b, int32_t j, bool& fresh) -> int32_t {
        const int32_t held = page_sum[b + 1] - page_sum[b] - (free_sum[b + 1] - free_sum[b]);
        fresh = j >= held;
        const int64_t rank = static_cast<int64_t>(free_sum[b]) + (j - held);
        if (fresh && rank >= p.n_free) return INT32_MIN;      // (reported with the counts)
        return max(fresh ? ld_input(p.free_pages + rank) : ld_input(p.block_tables + b * p.block_ld + j), -1);
    };
    // ... and as it goes out: -1 where there is none
    auto checked = [&](int32_t id) -> int32_t {
        if (id >= 0 && id < p.n_phys) return id;
        if (id != INT32_MIN) report(p.dev_status, JANUS_DEV_INDEX_OUT_OF_RANGE);
        return -1;
    };

    const int64_t stride = static_cast<int64_t>(gridDim.x) * BP_THREADS;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * BP_THREADS + tid;
    for (int64_t r = at; r < p.max_rows; r += stride) {
        int32_t session = -1;
        int64_t pos = -1, slot = -1, key_row = -1;
        if (r < row_sum[p.B]) {
            const int b = bp_find(row_sum, p.B, r);
            session = b;
            pos = bp_position(ld_input(p.cached + b), r - row_sum[b]);
            const int32_t j = bp_page_of(pos, p.page_size, p.page_shift, page_sum[b + 1] - page_sum[b]);
            bool fresh;
            const int32_t id = j >= 0 ? checked(load_page(b, j, fresh)) : -1;
            if (id >= 0) {
                slot = static_cast<int64_t>(id) * p.page_size + (pos - static_cast<int64_t>(j) * p.page_size);
                if (p.key_rows != nullptr) key_row = ld_input(p.key_offsets + b) + pos;
            }
        }
        p.row_sessions[r] = session;
        p.positions[r] = pos;
        p.slots[r] = slot;
        if (p.key_rows != nullptr) p.key_rows[r] = key_row;
    }
    // Where the threads would go round several times, four consecutive entries at a time: one search, and their loads go together (1024 sessions
    // of up to 131072 tokens, one run: one at a time 11.9 us, four 9.2, eight 10.2; the four took 10.3 to 11.0 in later runs.  Twelve sessions 4.7, with four
    // entries a thread 5.4).
    constexpr int AT_ONCE = 4;
    const int64_t entries = page_sum[p.B];
    const int per_turn = entries > stride ? AT_ONCE : 1;
    for (int64_t e = at * per_turn; e < entries; e += stride * per_turn) {
        int b = bp_find(page_sum, p.B, e);
        int32_t id[AT_ONCE], j[AT_ONCE];
        int session[AT_ONCE];
        bool fresh[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            fresh[k] = false;
            if (k >= per_turn || e + k >= entries) continue;
            while (e + k >= page_sum[b + 1]) ++b;
            session[k] = b;
            j[k] = static_cast<int32_t>(e + k - page_sum[b]);
            id[k] = load_page(b, j[k], fresh[k]);
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (k >= per_turn || e + k >= entries) continue;
            id[k] = checked(id[k]);
            if (fresh[k]) p.block_tables[session[k] * p.block_ld + j[k]] = id[k];
            if (e + k < p.table_capacity) p.page_tables[e + k] = id[k];
        }
    }
}

}  // namespace janus

extern "C" int janus_batch_plan(const int64_t* cached_lens, const int64_t* new_lens, int B, int page_size, int32_t* block_tables, int64_t block_ld,
                                int64_t width, const int32_t* free_pages, int64_t n_free, int64_t n_phys_pages, const int64_t* key_offsets,
                                int64_t* row_offsets, int64_t* kv_lens, int64_t* table_offsets, int32_t* page_tables, int64_t table_capacity,
                                int32_t* row_sessions, int64_t* positions, int64_t* slots, int64_t* key_rows, int64_t max_rows, int64_t* counts,
                                int32_t* dev_status, void* stream) {
    using namespace janus;
    if (B < 0 || page_size <= 0 || width < 0 || n_free < 0 || n_phys_pages < 0 || table_capacity < 0 || max_rows < 0) return JANUS_ERR_INVALID_ARG;
    if (n_phys_pages > INT32_MAX || max_rows > INT32_MAX || table_capacity > INT32_MAX || width > INT32_MAX) return JANUS_ERR_INVALID_ARG;
    if (B > BP_MAX_SESSIONS) return JANUS_ERR_UNSUPPORTED;
    if (B > 0 && width > INT32_MAX / B) return JANUS_ERR_UNSUPPORTED;
    if (B > 1 && block_ld < width) return JANUS_ERR_INVALID_ARG;                     // rows that share memory
    if (!row_offsets || !table_offsets || !counts) return JANUS_ERR_INVALID_ARG;
    if (B > 0 && (!cached_lens || !new_lens || !kv_lens)) return JANUS_ERR_INVALID_ARG;
    if (B > 0 && width > 0 && !block_tables) return JANUS_ERR_INVALID_ARG;
    if ((n_free > 0 && !free_pages) || (table_capacity > 0 && !page_tables)) return JANUS_ERR_INVALID_ARG;
    if (max_rows > 0 && (!row_sessions || !positions || !slots)) return JANUS_ERR_INVALID_ARG;
    if ((key_rows != nullptr) != (key_offsets != nullptr) && max_rows > 0) return JANUS_ERR_INVALID_ARG;
    // What is written shares no memory with anything else: every CTA reads all lengths by itself, at no set time.
    const int64_t table_bytes = B > 0 ? ((B - 1) * block_ld + width) * 4 : 0, n8 = 8 * static_cast<int64_t>(B);
    const struct { const void* at; int64_t bytes; bool written; } memory[] = {
        {row_offsets, n8 + 8, true}, {table_offsets, n8 + 8, true}, {counts, 24, true}, {kv_lens, n8, true}, {page_tables, 4 * table_capacity, true},
        {row_sessions, 4 * max_rows, true}, {positions, 8 * max_rows, true}, {slots, 8 * max_rows, true}, {key_rows, 8 * max_rows, true}, {block_tables, table_bytes, true},
        {cached_lens, n8, false}, {new_lens, n8, false}, {key_offsets, n8, false}, {free_pages, 4 * n_free, false}};
    for (const auto& x : memory)
        for (const auto& y : memory) {
            if (&x == &y || !x.written || x.at == nullptr || y.at == nullptr || x.bytes <= 0 || y.bytes <= 0) continue;
            const uintptr_t a = reinterpret_cast<uintptr_t>(x.at), b = reinterpret_cast<uintptr_t>(y.at);
            if (a < b + static_cast<uint64_t>(y.bytes) && b < a + static_cast<uint64_t>(x.bytes)) return JANUS_ERR_INVALID_ARG;
        }
    BpParams p;
    p.cached = cached_lens; p.fresh = new_lens;
    p.B = B; p.page_size = page_size;
    p.page_shift = -1;
    if ((page_size & (page_size - 1)) == 0) {
        p.page_shift = 0;
        while ((1 << p.page_shift) < page_size) ++p.page_shift;
    }
    p.block_tables = block_tables; p.block_ld = block_ld; p.width = static_cast<int32_t>(width);
    p.free_pages = free_pages; p.n_free = n_free; p.n_phys = n_phys_pages;
    p.key_offsets = key_offsets;
    p.row_offsets = row_offsets; p.kv_lens = kv_lens; p.table_offsets = table_offsets;
    p.page_tables = page_tables; p.table_capacity = table_capacity;
    p.row_sessions = row_sessions; p.positions = positions; p.slots = slots; p.key_rows = key_rows;
    p.max_rows = max_rows; p.counts = counts; p.dev_status = dev_status;
    const size_t smem = 3 * sizeof(int32_t) * (static_cast<size_t>(B) + 1);
    if (smem > 40 * 1024) {
        static once_per_context larger;
        JANUS_CUDA_CHECK(larger.run([] {
            return cudaFuncSetAttribute(batch_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(3 * sizeof(int32_t) * (BP_MAX_SESSIONS + 1)));
        }));
    }
    // a CTA for every 1024 rows or table entries there can be, at most one for each SM
    const int64_t most = B * width > max_rows ? B * width : max_rows;
    const int64_t ctas = (most + 2 * BP_THREADS - 1) / (2 * BP_THREADS);
    const unsigned grid = static_cast<unsigned>(ctas < 1 ? 1 : ctas < 148 ? ctas : 148);
    JANUS_CUDA_CHECK(launch_kernel(batch_plan_kernel, dim3(grid), BP_THREADS, smem, static_cast<cudaStream_t>(stream), 1, p));
    return JANUS_OK;
}
