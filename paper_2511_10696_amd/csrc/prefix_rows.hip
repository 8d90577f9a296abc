// prefix_rows.hip -- the rows of a shared prefix for all sequences of a decode
// step at once: partial softmaxes of chunks of prefix rows, on the matrix
// cores (bf16: v_mfma_f32_32x32x16_bf16, float32: v_mfma_f32_16x16x4f32).
//
// Of head h, sequence s at position t = plen + len_in[s] attends the prefix
// rows max(0, t - k)..plen - 1: an end of the prefix, the same rows for every
// sequence but for where they begin.  A work-group takes one chunk of the rows
// of one head and a tile of sequences, and leaves for each of them the largest
// logit m of the chunk (log2 units), l = sum 2^(x - m) and the values weighted
// alike, o; decode_cached.hip joins the chunks with the sequence's own rows.
//
// Tiles of rows go through LDS in the working type: the loads of the next tile
// (16 bytes a thread, whole lines) are issued before the present one is worked
// on and written behind it, e4m3 codes converted on the way, with the row's
// scale, which is exact.  The four wavefronts of a work-group are G groups of
// queries by RS shares of a tile's row blocks; with few sequences all four
// share one group of queries, and their states are joined at the end.
//
// As in forward_bf16.hip the scores are computed transposed, S^T = K Q^T, so
// that a lane holds scores of one query and the probabilities are the B operand
// of O^T = V^T P^T as they lie, the row order permuted alike in the V^T operand
// (bf16: LDS transpose reads).  The running maximum is raised with every block
// that has a larger logit, so a dominating row has weight 1 before it is
// rounded to bf16; the sums are of the unrounded weights.
//
// Rows that begin before a sequence's window are masked in the blocks that
// hold such rows.  A masked weight is 0, but 0 times an infinity or NaN is not:
// tiles with masked rows are searched for values that are not finite, and one
// that has some is added entry by entry.
#include <algorithm>

#include "bf16_rows.h"
#include "e4m3.h"
#include "kernels.h"
#include "pi_common.h"

namespace pi_attn {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int WAVES = 4;
constexpr int NT = 64 * WAVES;

// ---- one block of rows with one group of queries ------------------------------
// Lane (c, g) belongs to query c of the group.  QB queries and KB rows a block;
// NS score slots, slot i being row slot_row(i, g); the output's groups of four
// dims, group x being dims ODIM * x + 4 g + [0, 4).
template <typename T, int D>
struct Mma;

template <int D>
struct Mma<__bf16, D> {
    static constexpr int QB = 32, KB = 32, NS = 16, NO = D / 8, ODIM = 8;
    static constexpr int KROW = 2 * D + 16, VROW = 2 * D + 64;   // bytes of a row in LDS: no bank met twice
    bf16x8 qf[D / 16];
    f32x16 o[D / 32];

    static __device__ int slot_row(int i, int g) { return 8 * (i >> 2) + 4 * g + (i & 3); }
    __device__ void query(const __bf16 *q, int g) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qf[s] = *reinterpret_cast<const bf16x8 *>(q + 16 * s + 8 * g);
    }
    __device__ void clear() {
#pragma unroll
        for (int b = 0; b < D / 32; ++b) o[b] = f32x16{};
    }
    __device__ void clear_query() {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qf[s] = bf16x8{};
    }
    __device__ void scale(float a) {
#pragma unroll
        for (int b = 0; b < D / 32; ++b) o[b] *= a;
    }
    __device__ float &at(int x, int e) { return reinterpret_cast<float *>(&o[x >> 2])[4 * (x & 3) + e]; }
    __device__ void scores(const unsigned char *kt, int c, int g, float (&s)[NS]) const {
        bf16x8 kf[D / 16];
#pragma unroll
        for (int u = 0; u < D / 16; ++u) kf[u] = *reinterpret_cast<const bf16x8 *>(kt + c * KROW + (2 * u + g) * 16);
        f32x16 sc = {};
#pragma unroll
        for (int u = 0; u < D / 16; ++u) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[u], qf[u], sc, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < NS; ++i) s[i] = sc[i];
    }
    __device__ void values(const unsigned char *vt, int lane, const float (&p)[NS]) {
        const int g = lane >> 5, G = lane >> 4, r = (lane >> 2) & 3, qd = lane & 3;
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) {
            bf16x8 pb;
#pragma unroll
            for (int e = 0; e < 8; ++e) pb[e] = (__bf16)p[8 * cc + e];
#pragma unroll
            for (int b = 0; b < D / 32; ++b) {
                bf16x8 vf;
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const int row = 16 * cc + 8 * hh + 4 * g + r, chunk = 4 * b + 2 * (G & 1) + (qd >> 1);
                    const bf16x4 y = __builtin_bit_cast(
                        bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                    (lds_s16x4 *)(vt + row * VROW + chunk * 16 + (qd & 1) * 8)));
#pragma unroll
                    for (int e = 0; e < 4; ++e) vf[4 * hh + e] = y[e];
                }
                o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb, o[b], 0, 0, 0);
            }
        }
    }
    static __device__ float round(float p) { return (float)(__bf16)p; }
};

template <int D>
struct Mma<float, D> {
    static constexpr int QB = 16, KB = 16, NS = 4, NO = D / 16, ODIM = 16;
    static constexpr int KROW = 4 * D + 16, VROW = 4 * D + 16;
    f32x4 qf[D / 16];
    f32x4 o[D / 16];

    static __device__ int slot_row(int i, int g) { return 4 * g + i; }
    __device__ void query(const float *q, int g) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qf[s] = *reinterpret_cast<const f32x4 *>(q + 16 * s + 4 * g);
    }
    __device__ void clear() {
#pragma unroll
        for (int b = 0; b < D / 16; ++b) o[b] = f32x4{};
    }
    __device__ void clear_query() {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qf[s] = f32x4{};
    }
    __device__ void scale(float a) {
#pragma unroll
        for (int b = 0; b < D / 16; ++b) o[b] *= a;
    }
    __device__ float &at(int x, int e) { return reinterpret_cast<float *>(&o[x])[e]; }
    // Product step (u, e) contracts dims 16 u + 4 g + e, in four chains.
    __device__ void scores(const unsigned char *kt, int c, int g, float (&s)[NS]) const {
        f32x4 sc[4] = {};
#pragma unroll
        for (int u = 0; u < D / 16; ++u) {
            const f32x4 kf = *reinterpret_cast<const f32x4 *>(kt + c * KROW + (4 * u + g) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[u][e], sc[e], 0, 0, 0);
        }
        const f32x4 sum = (sc[0] + sc[1]) + (sc[2] + sc[3]);
#pragma unroll
        for (int i = 0; i < NS; ++i) s[i] = sum[i];
    }
    // Step i contracts rows 4 g + i, whose weights are the score slots i.
    __device__ void values(const unsigned char *vt, int lane, const float (&p)[NS]) {
        const int c = lane & 15, g = lane >> 4;
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int b = 0; b < D / 16; ++b) {
                const float v = *reinterpret_cast<const float *>(vt + (4 * g + i) * VROW + (16 * b + c) * 4);
                o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[i], o[b], 0, 0, 0);
            }
    }
    static __device__ float round(float p) { return p; }
};

// Maximum and sum over the lanes of a query.
template <int QB>
__device__ inline float query_max(float x) {
    if constexpr (QB == 16) x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}

template <int QB>
__device__ inline float query_sum(float x) {
    if constexpr (QB == 16) x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// ---- tiles ---------------------------------------------------------------------
template <typename T, typename ST, int D, int TR>
struct Stage {
    using M = Mma<T, D>;
    static constexpr bool Q = sizeof(ST) == 1;
    static constexpr int CPR = D * (int)sizeof(ST) / 16;   // 16-byte pieces of a row as it is stored
    static constexpr int U = TR * CPR / NT;                // of each thread, of keys and of values
    static_assert(TR * CPR % NT == 0, "whole pieces for every thread");
    uint4 k[U], v[U];
    unsigned kb[Q ? U : 1], vb[Q ? U : 1];

    // Tile rows row0 + [0, TR) of the head's rows; from `end` on row end - 1
    // again, written as zeros by put().
    __device__ void fetch(const CachedParams &p, int h, int row0, int end, int tid) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = u * NT + tid;
            const int64_t row = h * p.pcap + min(row0 + x / CPR, end - 1);
            const int64_t at = row * (D * (int)sizeof(ST)) + (x % CPR) * 16;
            k[u] = *reinterpret_cast<const uint4 *>((const uint8_t *)p.k_prefix + at);
            v[u] = *reinterpret_cast<const uint4 *>((const uint8_t *)p.v_prefix + at);
            if constexpr (Q) {
                kb[u] = p.k_prefix_exp[row];
                vb[u] = p.v_prefix_exp[row];
            }
        }
    }

    // A piece into LDS, and whether one of its values is not finite.
    static __device__ bool put_piece(uint4 raw, unsigned byte, unsigned char *to) {
        unsigned bad = 0;
        if constexpr (Q) {
            const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
            const float scale = e4m3_scale(byte);
            if constexpr (sizeof(T) == 2) {
                bf16x8 y[2];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false);
                    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true);
                    y[i >> 1][4 * (i & 1)] = a[0];
                    y[i >> 1][4 * (i & 1) + 1] = a[1];
                    y[i >> 1][4 * (i & 1) + 2] = b[0];
                    y[i >> 1][4 * (i & 1) + 3] = b[1];
                }
                reinterpret_cast<bf16x8 *>(to)[0] = y[0];
                reinterpret_cast<bf16x8 *>(to)[1] = y[1];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4 y;
                    float x[4];
                    e4m3_unpack4(w[i], x);
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = x[e] * scale;
                    reinterpret_cast<f32x4 *>(to)[i] = y;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) bad |= ((w[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;   // 0x7f, 0xff
            bad |= byte >= 247;   // 256 * 2^120 is past the largest float
        } else {
            *reinterpret_cast<uint4 *>(to) = raw;
            const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2) {   // exponents of all ones
                    bad |= ((w[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                } else {
                    bad |= ((w[i] & 0x7f800000u) + 0x00800000u) & 0x80000000u;
                }
            }
        }
        return bad != 0;
    }

    // The fetched tile into LDS; whether a value is not finite.
    __device__ bool put(unsigned char *kt, unsigned char *vt, int row0, int end, int tid) {
        bool bad = false;
        constexpr int WIDE = 16 * (int)(sizeof(T) / sizeof(ST));   // bytes of a piece in LDS
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = u * NT + tid, r = x / CPR, pc = x % CPR;
            if (row0 + r >= end) k[u] = v[u] = make_uint4(0, 0, 0, 0);
            put_piece(k[u], Q ? kb[u] : 0, kt + r * M::KROW + pc * WIDE);
            bad |= put_piece(v[u], Q ? vb[u] : 0, vt + r * M::VROW + pc * WIDE);
        }
        return bad;
    }
};

// G groups of queries, RS = 4 / G shares of the blocks of a tile of TR rows.
template <typename T, typename ST, int D, int G, int TR>
__global__ __launch_bounds__(NT, TR * D > 64 * 128 ? 1 : 2) void prefix_kernel(CachedParams p, int n_qt, uint32_t n_logical) {
    using M = Mma<T, D>;
    constexpr int RS = WAVES / G, QB = M::QB, KB = M::KB, QT = QB * G;
    constexpr int TILE_BYTES = TR * (M::KROW + M::VROW);
    constexpr int STATE = 64 * 4 * (M::NO * 4 + 2);   // of a wavefront: o, m, l
    constexpr int LDS = TILE_BYTES > (RS - 1) * G * STATE ? TILE_BYTES : (RS - 1) * G * STATE;
    __shared__ __align__(16) unsigned char lds[LDS];
    __shared__ int s_bad[2];
    unsigned char *const kt = lds, *const vt = lds + TR * M::KROW;

    const uint32_t logical = xcd_remap(blockIdx.x, n_logical);
    if (logical >= n_logical) return;
    const DecodeParams &d = p.d;
    const DivMod qt_of = divmod(logical, n_qt), chunk_of = divmod(qt_of.quot, p.chunks);
    const int qt = (int)qt_of.rem, x = (int)chunk_of.rem, h = (int)chunk_of.quot;
    const int row_begin = p.plen - p.near + x * p.chunk;
    const int end = min(row_begin + p.chunk, p.plen);

    const int tid = threadIdx.x, lane = __lane_id();
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int qg = w % G, rs = w / G;
    const int c = lane % QB, g = lane / QB;

    // Where the window of a sequence begins; INT32_MAX for none.
    auto low_of = [&](int s) {
        if (s >= d.S) return INT32_MAX;
        const int n = d.len_in[s];
        return n >= 0 && n < d.cap ? window_lo(p.plen + n, d.k) : INT32_MAX;
    };
    // Over the tile's sequences that meet the chunk: where the first window
    // begins, and the last.
    int lo_min = INT32_MAX, lo_max = 0;
#pragma unroll
    for (int i = 0; i < QT; i += 64) {
        const int a = i + lane < QT ? low_of(qt * QT + i + lane) : INT32_MAX;
        lo_min = min(lo_min, a);
        if (a < end) lo_max = max(lo_max, a);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        lo_min = min(lo_min, __shfl_xor(lo_min, o));
        lo_max = max(lo_max, __shfl_xor(lo_max, o));
    }
    lo_min = __builtin_amdgcn_readfirstlane(lo_min);
    lo_max = __builtin_amdgcn_readfirstlane(lo_max);
    if (lo_min >= end) return;

    const int s = qt * QT + qg * QB + c;
    const int lo = low_of(s);
    M mm;
    mm.clear();
    float bias = 0.0f;
    if (s < d.S) {
        mm.query((const T *)d.q_new + ((int64_t)s * d.H + h) * D, g);
        bias = fusion_bias(d.gate[s * d.gss + h * d.gsh], true).local;
    } else {
        mm.clear_query();
    }
    const float c2 = d.scale * kLog2e;
    const bool clamped = d.clamp > 0.0f;

    float m = -INFINITY, l = 0.0f;
    const int row0 = row_begin + max(lo_min - row_begin, 0) / TR * TR;
    if (tid < 2) s_bad[tid] = 0;
    Stage<T, ST, D, TR> stage;
    stage.fetch(p, h, row0, end, tid);
    __syncthreads();
    int turn = 0;
    for (int row = row0; row < end; row += TR, turn ^= 1) {
        const bool masked = row < lo_max;   // some sequence's window begins behind the tile's first row
        if (stage.put(kt, vt, row, end, tid) && masked) s_bad[turn] = 1;
        __syncthreads();
        if (row + TR < end) stage.fetch(p, h, row + TR, end, tid);
        const bool bad = masked && s_bad[turn];
        if (tid == 0) s_bad[turn ^ 1] = 0;
#pragma unroll
        for (int b = 0; b < TR / KB / RS; ++b) {
            const int blk = b * RS + rs, j0 = row + blk * KB;
            // rows of the block that the group's sequences meet
            if (j0 >= end || !__builtin_amdgcn_ballot_w64(lo < min(j0 + KB, end))) continue;
            const unsigned char *kb = kt + blk * KB * M::KROW, *vb = vt + blk * KB * M::VROW;
            float sc[M::NS];
            mm.scores(kb, c, g, sc);
            if (clamped) {
#pragma unroll
                for (int i = 0; i < M::NS; ++i)
                    sc[i] = fminf(fmaxf(sc[i] * d.scale + bias, -d.clamp), d.clamp) * kLog2e;
            } else {
#pragma unroll
                for (int i = 0; i < M::NS; ++i) sc[i] *= c2;
            }
            if (j0 < lo_max || j0 + KB > end) {
#pragma unroll
                for (int i = 0; i < M::NS; ++i) {
                    const int j = j0 + M::slot_row(i, g);
                    sc[i] = j >= lo && j < end ? sc[i] : -INFINITY;
                }
            }
            float mx = sc[0];
#pragma unroll
            for (int i = 1; i < M::NS; ++i) mx = fmaxf(mx, sc[i]);
            mx = query_max<QB>(mx);
            if (__builtin_amdgcn_ballot_w64(mx > m)) {
                const float m_new = fmaxf(m, mx);
                const float alpha = mx > m ? __builtin_amdgcn_exp2f(m - m_new) : 1.0f;
                m = m_new;
                l *= alpha;
                mm.scale(alpha);
            }
            const float m_use = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int i = 0; i < M::NS; ++i) {
                sc[i] = __builtin_amdgcn_exp2f(sc[i] - m_use);
                l += sc[i];
            }
            if (!bad) {
                mm.values(vb, lane, sc);
            } else {
                // Row by row, for the sequences whose window holds it.
#pragma unroll 1
                for (int r = 0; r < KB; ++r) {
                    // the lane and slot of the query that hold row r
                    const int gr = (r >> 2) % (64 / QB), ir = (r / (4 * (64 / QB))) * 4 + (r & 3);
                    float pr = 0.0f;
#pragma unroll
                    for (int i = 0; i < M::NS; ++i) {
                        const float y = __shfl(sc[i], c + QB * gr);
                        pr = i == ir ? y : pr;
                    }
                    pr = M::round(pr);
                    const int j = j0 + r;
                    const bool in = j >= lo && j < end;
#pragma unroll
                    for (int y = 0; y < M::NO; ++y) {
                        const T *vr = reinterpret_cast<const T *>(vb + r * M::VROW) + M::ODIM * y + 4 * g;
#pragma unroll
                        for (int e = 0; e < 4; ++e) mm.at(y, e) = in ? mm.at(y, e) + pr * (float)vr[e] : mm.at(y, e);
                    }
                }
            }
        }
        __syncthreads();
    }
    l = query_sum<QB>(l);

    // The states of the RS wavefronts of a group of queries, joined by the first.
    if constexpr (RS > 1) {
        float *mine = reinterpret_cast<float *>(lds) + ((rs - 1) * G + qg) * (STATE / 4) + lane;
        if (rs > 0) {
#pragma unroll
            for (int y = 0; y < M::NO; ++y)
#pragma unroll
                for (int e = 0; e < 4; ++e) mine[64 * (4 * y + e)] = mm.at(y, e);
            mine[64 * (4 * M::NO)] = m;
            mine[64 * (4 * M::NO + 1)] = l;
        }
        __syncthreads();
        if (rs > 0) return;
        float all = m;
        const float *theirs = reinterpret_cast<const float *>(lds) + qg * (STATE / 4) + lane;
#pragma unroll
        for (int r = 0; r < RS - 1; ++r) all = fmaxf(all, theirs[r * G * (STATE / 4) + 64 * (4 * M::NO)]);
        const float all_use = all == -INFINITY ? 0.0f : all;
        const float a = __builtin_amdgcn_exp2f(m - all_use);
        m = all;
        l *= a;
        mm.scale(a);
#pragma unroll
        for (int r = 0; r < RS - 1; ++r) {
            const float *from = theirs + r * G * (STATE / 4);
            const float f = __builtin_amdgcn_exp2f(from[64 * (4 * M::NO)] - all_use);
            l += f * from[64 * (4 * M::NO + 1)];
#pragma unroll
            for (int y = 0; y < M::NO; ++y)
#pragma unroll
                for (int e = 0; e < 4; ++e) mm.at(y, e) += f * from[64 * (4 * y + e)];
        }
    }
    if (lo >= end) return;   // no window here, or no sequence
    const int64_t at = (int64_t)x * d.S * d.H + (int64_t)s * d.H + h;
#pragma unroll
    for (int y = 0; y < M::NO; ++y) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = mm.at(y, e);
        *reinterpret_cast<f32x4 *>(p.part_o + at * D + M::ODIM * y + 4 * g) = v;
    }
    if (g == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(m, l);
}

template <typename T, typename ST, int D, int G, int TR>
hipError_t launch_g(const CachedParams &p, hipStream_t stream) {
    constexpr int QT = Mma<T, D>::QB * G;
    const int n_qt = (p.d.S + QT - 1) / QT;
    const int64_t n = (int64_t)p.d.H * p.chunks * n_qt;
    return launch_kernel(prefix_kernel<T, ST, D, G, TR>, dim3((unsigned)xcd_grid(n)), dim3(NT), stream, p, n_qt,
                         (uint32_t)n);
}

template <typename T, typename ST, int D>
hipError_t launch_d(const CachedParams &p, hipStream_t stream) {
    constexpr int QB = Mma<T, D>::QB;
    constexpr int FEW = sizeof(T) == 2 ? 128 : 64;   // rows of a tile that four wavefronts share
    if (p.d.S <= QB) return launch_g<T, ST, D, 1, FEW>(p, stream);
    if (p.d.S <= 2 * QB) return launch_g<T, ST, D, 2, 64>(p, stream);
    return launch_g<T, ST, D, 4, 64>(p, stream);
}

template <typename T, typename ST>
hipError_t launch_t(const CachedParams &p, hipStream_t stream) {
    return p.d.D == 64 ? launch_d<T, ST, 64>(p, stream) : launch_d<T, ST, 128>(p, stream);
}

}  // namespace

PrefixShape prefix_shape(int S, bool bf16) {
    const int QB = bf16 ? 32 : 16;
    return PrefixShape{S <= QB ? QB : S <= 2 * QB ? 2 * QB : 4 * QB, bf16 && S <= QB ? 128 : 64};
}

hipError_t launch_prefix(const CachedParams &p, bool bf16, hipStream_t stream) {
    if (p.k_prefix_exp) return bf16 ? launch_t<__bf16, e4m3>(p, stream) : launch_t<float, e4m3>(p, stream);
    return bf16 ? launch_t<__bf16, __bf16>(p, stream) : launch_t<float, float>(p, stream);
}

}  // namespace pi_attn
