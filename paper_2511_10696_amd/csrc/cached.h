// cached.h -- parameters and launches of the quantised caches and of the decode
// steps over them and behind a shared prefix.
#pragma once

#include "kernels.h"

namespace pi_attn {

// Division of x < 2^31 by a divisor d >= 1 that the host knows: with l =
// ceil(log2 d), m = floor(2^(31 + l) / d) + 1 < 2^32 has m d = 2^(31 + l) + e
// with 0 < e <= 2^l, so x m >> (31 + l) is floor(x / d).
struct Divisor {
    uint32_t m, shift;
    Divisor() = default;
    explicit Divisor(uint32_t d) {
        uint32_t l = 0;
        while (((uint64_t)1 << l) < d) ++l;
        shift = 31 + l;
        m = (uint32_t)(((uint64_t)1 << shift) / d + 1);
    }
    __host__ __device__ uint32_t div(uint32_t x) const { return (uint32_t)(((uint64_t)x * m) >> shift); }
};

// Rows of a quantised cache: stored from or loaded to k and v [S][H][n][D].
struct CacheRowsParams {
    int S, H, n, D, cap;
    uint32_t rows;                  // S * H * n, at least 1
    Divisor by_n, by_h;
    uint32_t runs;                  // of a head, and
    bool heads_first;               // their order; set by the launch, as is
    uint32_t first_group;           // the first work-group, of several launches
    void *k, *v;                    // read by a store, written by a load
    int64_t sb, sh, sn;             // element strides shared by k and v
    const int32_t *start, *count;   // [S], or nullptr: 0, n
    uint8_t *k_cache, *v_cache;     // codes [S][H][cap][D]
    uint8_t *k_exp, *v_exp;         // scale bytes [S][H][cap]
};

// A decode step over quantised caches, or behind a shared prefix, or both: the
// position of the new row is t = plen + len_in[s].
struct CachedParams {
    DecodeParams d;                 // caches of own rows: d.dtype's type, or e4m3 codes
    uint8_t *k_exp, *v_exp;         // scale bytes [S][H][cap]; nullptr: not quantised
    int plen;                       // shared rows, positions [0, plen)
    int64_t pcap;                   // rows from one head's prefix to the next's
    const void *k_prefix, *v_prefix;             // [H][pcap][D], the caches' type
    const uint8_t *k_prefix_exp, *v_prefix_exp;  // [H][pcap]
    // Parts of the softmax, from the chunks of the prefix rows that a window
    // meets and from `own_parts` ranges of own rows (0: not split): for part x,
    // at[x][s * H + h] the weighted values [D], then (max, sum) in log2 units.
    float *part_o, *part_ml;
    int near;                       // prefix rows from which on windows reach: [plen - near, plen)
    int tile, chunks;               // their tiles' rows; chunk x takes tiles x, x + chunks, ...
    int own_parts;
    bool direct;                    // prefix rows are read with the own ones, no chunks
};

// Behind the last row of a chunk: it is of no use to windows that begin there or later.
__host__ __device__ inline int chunk_end(const CachedParams &p, int x) {
    const int tiles = (p.near + p.tile - 1) / p.tile, last = x + (tiles - 1 - x) / p.chunks * p.chunks;
    return last + 1 == tiles ? p.plen : p.plen - p.near + (last + 1) * p.tile;
}

// Decode step of CachedParams: the parts' sizes, then the step.
void plan_decode_cached(CachedParams &p, bool bf16);
hipError_t launch_decode_cached(const CachedParams &p, bool bf16, hipStream_t stream);

// Its shared prefix: the parts of the chunks.
struct PrefixShape {
    int queries;                    // of a work-group
    int tile;                       // rows that it takes at a time, at least 64
    int per_cu;                     // work-groups that share a CU
};
PrefixShape prefix_shape(const CachedParams &p, bool bf16);
hipError_t launch_prefix(const CachedParams &p, bool bf16, hipStream_t stream);

// Rows into (store) or out of a quantised cache.
hipError_t launch_cache_rows(const CacheRowsParams &p, bool store, bool bf16, hipStream_t stream);

}  // namespace pi_attn
