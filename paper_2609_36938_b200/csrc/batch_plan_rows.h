// Positions and places of a step's new tokens.  Plain C++, so that it can be tested without a device.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define JANUS_PLAN_FN __host__ __device__ inline
#else
#define JANUS_PLAN_FN inline
#endif

namespace janus {

// Position of new token i (not negative) of a session with `cached` tokens in the cache, as the caller says: a negative number counts as none, and what does
// not fit in 63 bits is 2^63 - 1 (a sum that wrapped would be a position, and with it a page, that nobody asked for).
JANUS_PLAN_FN int64_t bp_position(int64_t cached, int64_t i) {
    const int64_t c = cached > 0 ? cached : 0;
    return i <= INT64_MAX - c ? c + i : INT64_MAX;
}

// Place of a position's page in its session's table of `pages` entries, or -1 behind its end.  page_shift: log2 of the page size, or -1.
JANUS_PLAN_FN int32_t bp_page_of(int64_t position, int page_size, int page_shift, int32_t pages) {
    const int64_t j = page_shift >= 0 ? position >> page_shift : position / page_size;
    return j >= 0 && j < pages ? static_cast<int32_t>(j) : -1;
}

}  // namespace janus
