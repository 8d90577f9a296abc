// paged.h -- parameters and launches of the rotary positions, of the paged
// caches' rows and of the decode step over them.
#pragma once

#include <algorithm>

#include "cached.h"
#include "kernels.h"
#include "rotary.h"

namespace pi_attn {

// The wavefronts of a launch over tiles of rows and groups of heads: the groups of a
// tile next to each other, or the tiles of a group.
struct WaveOrder {
    bool heads_first;
    uint32_t tiles, groups;
    uint32_t first;                 // wavefront, of several launches
    Divisor by_inner;
    WaveOrder() = default;
    WaveOrder(bool hf, uint32_t t, uint32_t g) : heads_first(hf), tiles(t), groups(g), first(0), by_inner(hf ? g : t) {}
    // Tile and group of a launch's wavefront; tile is past the last one for those without work.
    __device__ void place(uint32_t wave, uint32_t &tile, uint32_t &group) const {
        wave += first;
        const uint32_t outer = by_inner.div(wave), inner = wave - outer * (heads_first ? groups : tiles);
        tile = heads_first || outer >= groups ? (heads_first ? outer : tiles) : inner;
        group = heads_first ? inner : outer;
    }
};

// Launches `kernel` on work-groups of WAVES wavefronts, as often as it takes: a launch has fewer
// than 2^32 threads.
template <int WAVES, typename P>
hipError_t launch_in_order(void (*kernel)(P), P &p, hipStream_t stream) {
    constexpr int64_t kMost = (int64_t)1 << 23;
    const int64_t blocks = ((int64_t)p.order.tiles * p.order.groups + WAVES - 1) / WAVES;
    hipError_t e = hipSuccess;
    for (int64_t b = 0; e == hipSuccess && b < blocks; b += kMost) {
        p.order.first = (uint32_t)(b * WAVES);
        e = launch_kernel(kernel, dim3((unsigned)std::min(blocks - b, kMost)), dim3(64 * WAVES), stream, p);
    }
    return e;
}

// Rows of q [B][H][N][D] and k [B][Hk][N][D] turned, forward or back.
struct RotateParams {
    int B, H, Hk, N, D;
    const void *q, *k;
    void *q_out, *k_out;
    int64_t qsb, qsh, qsn, ksb, ksh, ksn;          // element strides of q and k,
    int64_t oqsb, oqsh, oqsn, oksb, oksh, oksn;    // of their results
    Rotary r;
    bool back;                      // the transpose: by the angle's negative
    uint32_t rows;                  // B * N, at least 1
    Divisor by_n;
    WaveOrder order;                // set by the launch
};

// A paged cache: position j of sequence s is row j mod page of page
// table[s][j / page]; an entry that names no page has no rows.
struct Pages {
    int n_pages, page, max_pages;   // pages in all, rows of one, entries of a sequence
    Divisor by_page;
    const int32_t *table;           // [S][max_pages]
    void *k, *v;                    // [n_pages][Hk][page][D], rows or codes
    uint8_t *k_exp, *v_exp;         // [n_pages][Hk][page]; nullptr: not quantised
};

// Rows of k and v [S][Hk][n][D] into or out of a paged cache.
struct PagedRowsParams {
    int S, Hk, n, D;
    void *k, *v;                    // read by a store, written by a load
    int64_t sb, sh, sn;
    const int32_t *start, *count;   // [S], or nullptr: 0, n
    Pages pages;
    Rotary r;                       // of the keys stored
    uint32_t rows;                  // S * n, at least 1
    Divisor by_n;
    WaveOrder order;                // set by the launch
};

// A decode step over a paged cache: H query heads, H / Hk to a key head.
struct PagedStepParams {
    int S, H, Hk, D, k, pi;
    const int32_t *len_in;
    int32_t *len_out;               // nullptr: not written
    const void *q_new, *k_new, *v_new;   // [S][H][D], [S][Hk][D]
    Pages pages;
    Rotary r;                       // of q_new and k_new
    const float *gate;
    int64_t gss, gsh;
    float scale, clamp;
    void *out;                      // [S][H][D]
    float *lse;                     // [S][H] or nullptr
    // Parts from ranges of the windows, at most `parts` of one (0: not split): for part x
    // at[x][s * H + h] the weighted values [D], then (max, sum) in log2 units.
    float *part_o, *part_ml;
    int parts;
};

hipError_t launch_rotate(const RotateParams &p, bool bf16_in, bool bf16_out, hipStream_t stream);
hipError_t launch_paged_rows(const PagedRowsParams &p, bool store, bool bf16, hipStream_t stream);

// The sizes of the parts, by the problem's sizes alone; then the step.
void plan_decode_paged(PagedStepParams &p);
hipError_t launch_decode_paged(const PagedStepParams &p, bool bf16, hipStream_t stream);

}  // namespace pi_attn
