// Whether two strided tensors can share memory.  Plain C++, so that it can be tested without a device.
#pragma once

#include <algorithm>
#include <cstdint>

namespace janus {

constexpr int MO_AXES = 3;

// Pieces of `bytes` at `at` plus any sum of index * stride (bytes, not negative) over the axes.
struct MoTensor {
    uintptr_t at;
    int64_t bytes;
    int64_t n[MO_AXES], stride[MO_AXES];
};

using mo_int = __int128;

struct MoAxis {
    mo_int stride;
    int64_t na, nb;
};

// Whether delta + sum d_i * stride_i, -na_i < d_i < nb_i, lies in (-b_bytes, a_bytes) for some d.  Strides descending; every d whose term the shorter strides can
// still make up for is tried: two at most where strides are nested.  `steps`: tries left; true when they run out.
inline bool mo_meet(const MoAxis* axes, int n, mo_int delta, mo_int a_bytes, mo_int b_bytes, int& steps) {
    if (n == 0) return -b_bytes < delta && delta < a_bytes;
    mo_int a_inner = a_bytes, b_inner = b_bytes;                 // what one index of the first axis spans
    for (int i = 1; i < n; ++i) {
        a_inner += axes[i].stride * (axes[i].na - 1);
        b_inner += axes[i].stride * (axes[i].nb - 1);
    }
    auto floor_div = [](mo_int x, mo_int d) { return x / d - (x % d < 0 ? 1 : 0); };
    const mo_int s = axes->stride;
    mo_int first = floor_div(-b_inner - delta, s) + 1, last = floor_div(a_inner - 1 - delta, s);
    if (first < 1 - axes->na) first = 1 - axes->na;
    if (last > axes->nb - 1) last = axes->nb - 1;
    for (mo_int d = first; d <= last; ++d)
        if (--steps < 0 || mo_meet(axes + 1, n - 1, delta + d * s, a_bytes, b_bytes, steps)) return true;
    return false;
}

// False where the tensors share no byte.  (True where they do, and where strides that are not nested at all leave too many combinations to try.)
inline bool mo_may_share(const MoTensor& a, const MoTensor& b) {
    MoAxis axes[2 * MO_AXES];
    int n = 0;
    if (a.bytes <= 0 || b.bytes <= 0) return false;
    for (int i = 0; i < MO_AXES; ++i) {
        if (a.n[i] <= 0 || b.n[i] <= 0) return false;
        if (a.n[i] > 1 && a.stride[i] != 0) axes[n++] = {a.stride[i], a.n[i], 1};
    }
    for (int i = 0; i < MO_AXES; ++i) {
        if (b.n[i] <= 1 || b.stride[i] == 0) continue;
        int at = 0;
        while (at < n && !(axes[at].stride == b.stride[i] && axes[at].nb == 1)) ++at;
        if (at == n) axes[n++] = {b.stride[i], 1, b.n[i]};
        else axes[at].nb = b.n[i];
    }
    std::sort(axes, axes + n, [](const MoAxis& x, const MoAxis& y) { return x.stride > y.stride; });
    int steps = 1 << 16;
    return mo_meet(axes, n, static_cast<mo_int>(b.at) - static_cast<mo_int>(a.at), a.bytes, b.bytes, steps);
}

// Whether every element has a place of its own: strides that are nested.
inline bool mo_apart(const MoTensor& a) {
    mo_int stride[MO_AXES];
    int64_t count[MO_AXES];
    int n = 0;
    for (int i = 0; i < MO_AXES; ++i) {
        if (a.n[i] <= 1) continue;
        int at = n++;
        for (; at > 0 && stride[at - 1] > a.stride[i]; --at) { stride[at] = stride[at - 1]; count[at] = count[at - 1]; }
        stride[at] = a.stride[i];
        count[at] = a.n[i];
    }
    mo_int inner = a.bytes;
    for (int i = 0; i < n; ++i) {
        if (stride[i] < inner) return false;
        inner += stride[i] * (count[i] - 1);
    }
    return true;
}

}  // namespace janus
