// paged_step.h -- what the kernels of the decode step over paged caches share.
#pragma once

#include "decode_rows.h"
#include "e4m3.h"
#include "paged.h"
#include "pi_common.h"

namespace pi_attn {

constexpr float kTau = 8.0f;   // a running maximum is raised in steps above this, log2 units

template <typename ST>
inline constexpr bool kQuantised = false;
template <>
inline constexpr bool kQuantised<e4m3> = true;

// The page that a table entry names, -1 if none.
__device__ inline int page_named(const Pages &g, int entry) { return entry >= 0 && entry < g.n_pages ? entry : -1; }

// The page of a sequence's position, -1 where it has none.
__device__ inline int page_of(const Pages &g, int64_t s, uint32_t slot) {
    return page_named(g, g.table[s * g.max_pages + slot]);
}

// Whether sequence s can take a row at t.
__device__ inline bool has_place(const Pages &g, int64_t s, int t) {
    return t >= 0 && t < (int64_t)g.page * g.max_pages && page_of(g, s, g.by_page.div(t)) >= 0;
}

// Ranges that a window of n rows has.
__device__ inline int ranges_of(int n, int range) { return max(1, (n + range - 1) / range); }

// A step of which pages in bf16 or e4m3 are multiplied on the matrix cores.
hipError_t launch_decode_paged_tiles(const PagedStepParams &p, bool bf16, hipStream_t stream);

}  // namespace pi_attn
