// paged_step.h -- what the kernels of the decode step over paged caches share.
#pragma once

#include <algorithm>

#include "decode_rows.h"
#include "e4m3.h"
#include "paged.h"
#include "pi_common.h"

namespace pi_attn {

constexpr float kTau = 8.0f;   // a running maximum is raised in steps above this, log2 units

// A row's weight 2^(d - m), d its logit as the maximum m has seen it.  Were the product that
// d comes from left unrounded here, the largest row's weight would be 2^r, r the rounding
// of m: 256 and more from logits of 2^32 on, which overflows or leaves no row a weight.
__device__ inline float weight(float d, float m) {
#pragma clang fp contract(off)
    return __builtin_amdgcn_exp2f(d - m);
}

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

// Rows of the longest window that the cache can hold, the new row apart.
inline int64_t longest_window(const PagedStepParams &p) {
    return std::min<int64_t>(p.k, (int64_t)p.pages.page * p.pages.max_pages - 1);
}

// Whether a step's window rows are not worth keeping in the caches: they are read once
// (one work-group has all of a key head's queries), and would push out what is there.
inline bool read_once(const PagedStepParams &p, int q_groups, int element_bytes) {
    constexpr int64_t kKeepBytes = 12 << 20;
    return q_groups == 1 && 2 * (int64_t)p.S * p.Hk * longest_window(p) * p.D * element_bytes > kKeepBytes;
}

// Rows of a range, and ranges, of a window of n rows in a split step: for three
// work-groups a CU (of each group of query heads) if all windows are alike, from 128 rows (a tile for each wavefront) to
// 1024, more where that would be more than p.parts ranges; whole steps of 128 rows.
__device__ inline int range_len(const PagedStepParams &p, int n) {
    const int64_t fill = (int64_t)n * (p.S * p.Hk) / 768, even = ((int64_t)n + p.parts - 1) / p.parts;
    return (int)((max(min(fill, (int64_t)1024), max(even, (int64_t)128)) + 127) & ~(int64_t)127);
}
__device__ inline int ranges_of(const PagedStepParams &p, int n) {
    const int len = range_len(p, n);
    return max(1, (int)(((int64_t)n + len - 1) / len));
}

// The step but for the join of its parts: pages in bf16 or e4m3, on the matrix cores; in
// float32.
hipError_t launch_decode_paged_tiles(const PagedStepParams &p, bool bf16, hipStream_t stream);
hipError_t launch_decode_paged_f32(const PagedStepParams &p, hipStream_t stream);

}  // namespace pi_attn
