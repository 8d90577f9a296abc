// kernels.h -- launch parameters and host launchers of the HIP kernels.
// The C ABI (api.hip) validates arguments and calls these; they only launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace pi_attn {

// Launch through hipLaunchKernel so the launch status is returned directly
// (no reliance on the per-thread last-error state).  Arguments convert to the
// kernel's parameter types.
template <typename... KArgs>
inline hipError_t launch_kernel(void (*kernel)(KArgs...), dim3 grid, dim3 block, hipStream_t stream,
                                typename std::common_type<KArgs>::type... args) {
    void *argv[] = {static_cast<void *>(&args)...};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, argv, 0, stream);
}

struct FwdParams {
    int B, H, N, D, k, pi;
    int causal;                     // 1: causal window and t - pi; 0: bidirectional, t -/+ pi
    const void *q, *k_ptr, *v;
    int64_t sb, sh, sn;             // element strides shared by q, k, v
    const float *gate;
    int64_t gsb, gsh, gsn;          // element strides of the gate logits
    float scale, clamp;             // clamp <= 0: off
    void *out;
    int64_t osb, osh, osn;
    float *lse;                     // [B][H][N] or nullptr
    // Sequence shard (the banded bf16 forward only): q/out/lse/gate row i is
    // absolute position qpos0 + i, k/v row i is kvpos0 + i, k/v rows end at
    // kvend, the sequence has nseq positions.  A whole sequence: 0, 0, N, N.
    int qpos0, kvpos0, kvend, nseq;
    int qend;                       // backward key pass: query rows held end at qend (a whole sequence: N)
    int64_t ksb, ksh, ksn;          // element strides of k and v (a whole sequence: sb, sh, sn)
};

struct DecodeParams {
    int S, H, D, cap, k, pi;
    const int32_t *len_in;
    int32_t *len_out;               // nullptr: not written
    const void *q_new, *k_new, *v_new;   // [S][H][D]
    void *k_cache, *v_cache;        // [S][H][cap][D]
    const float *gate;
    int64_t gss, gsh;
    float scale, clamp;
    void *out;                      // [S][H][D]
    float *lse;                     // [S][H] or nullptr
};

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
    bool heads_first;               // their order; set by the launch
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

struct BwdParams {
    FwdParams f;                    // inputs as for the forward (out/lse unused)
    int dtype;                      // 0 = float32, 1 = bf16 (q, k, v, dout)
    const float *lse;               // [B][H][N]
    const void *out, *dout;         // forward output and dL/dy
    int64_t osb, osh, osn;          // element strides of out and dout
    float *dq, *dk, *dv;            // [B][H][N][D] contiguous
    float *dgate, *rowterm;         // [B][H][N] contiguous
};

hipError_t launch_index_set(int n, int k, int pi, bool causal, int32_t *idx, hipStream_t stream);

// float32 forward (D = 64 or 128): MFMA tiles of 16 queries, or one wavefront
// per query where one_per_row().
bool one_per_row(const FwdParams &p);
hipError_t launch_forward_f32(const FwdParams &p, hipStream_t stream);
hipError_t launch_forward_rows_f32(const FwdParams &p, hipStream_t stream);

// bf16 banded MFMA forward (D = 64 or 128).
hipError_t launch_forward_bf16(const FwdParams &p, hipStream_t stream);

// Decode step, working set split across wavefronts (D = 64 or 128).
hipError_t launch_decode(const DecodeParams &p, bool bf16, hipStream_t stream);

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

// Backward: a query pass (dq, dgate, row terms <dL/dy_t, y_t>) and a key pass
// (dk, dv); picks the kernels by dtype and window.
hipError_t launch_backward(const BwdParams &p, hipStream_t stream);

// out[h] = sum over b and t of dgate[b][h][t] (fixed order, fp64 sums).
hipError_t launch_gate_grad_per_head(int B, int H, int N, const float *dgate, float *out, hipStream_t stream);

// Both passes for float32 data, the same two ways.
hipError_t launch_backward_f32(const BwdParams &p, hipStream_t stream);
hipError_t launch_backward_rows_f32(const BwdParams &p, hipStream_t stream);

// MFMA query pass (dq, dgate, row terms) for bf16 inputs.
hipError_t launch_backward_q_bf16(const BwdParams &p, hipStream_t stream);

// MFMA key pass (dk, dv) for bf16 inputs; needs the row terms.
hipError_t launch_backward_kv_bf16(const BwdParams &p, hipStream_t stream);

// The same at D = 64, one wavefront per 32 keys; rows of dL/dy within 32-bit
// byte offsets of a band's first row.
hipError_t launch_backward_kv64_bf16(const BwdParams &p, hipStream_t stream);

}  // namespace pi_attn
