// prefix_rows.hip -- the rows of a shared prefix for all sequences of a decode
// step at once: partial softmaxes of chunks of prefix rows, on the matrix
// cores (bf16: v_mfma_f32_32x32x16_bf16, float32: v_mfma_f32_16x16x4f32).
//
// Of head h, sequence s at position t = plen + len_in[s] attends the prefix
// rows max(0, t - k)..plen - 1: an end of the prefix, the same rows for every
// sequence but for where they begin.  A work-group takes one chunk of the rows
// of one head and a group of sequences, and leaves for each of them an m little
// above the largest logit of the chunk (log2 units), l = sum 2^(x - m) and the
// values weighted alike, o; decode_cached.hip joins the chunks with the
// sequence's own rows.  A chunk is every n-th tile of rows, so that whatever the
// windows leave is shared by all work-groups, and the last tile comes first,
// which every window that meets the prefix holds: the first loads wait for no
// length.
//
// Rows go from global memory straight into LDS as they are stored, through a
// ring of stages: while a stage is worked on, the next ones are on their way,
// and a wait counts the loads that may stay in flight.  The 16-byte pieces of a
// row are XOR-swizzled by the row, each lane fetching the piece that belongs at
// its place, so that no operand read below meets a bank twice.  e4m3 codes are
// converted as they become operands: a key row's scale with its codes (exact),
// a value row's in the weight (exact).  The wavefronts of a work-group are
// G groups of queries by RS shares of a stage's row blocks.  With one group
// every wavefront has a ring of its own, and they wait for nobody until their
// states are joined at the end.
//
// As in forward_bf16.hip the scores are computed transposed, S^T = K Q^T, so
// that a lane holds scores of one query and the probabilities are the B operand
// of O^T = V^T P^T as they lie, the row order permuted alike in the V^T operand
// (LDS transpose reads).  In bf16 a weight is the sum of two bf16 terms, two
// products with each value operand, so that outputs are as near the definition
// as with float32 weights, which a step has that reads its rows with vector
// instructions.  One term, off by 2^-8, took 76 us where two take 82 (64
// sequences of 32 heads behind 32768 e4m3 rows, D = 128), 121 and 137 (128
// behind as many of bf16), 93 and 93 (24 of 16 behind 65536).
//
// Rows that begin before a sequence's window are masked in the blocks that
// hold such rows.  A masked weight is 0, but 0 times an infinity or NaN is not:
// blocks with masked rows are searched for values that are not finite; these
// become 0 in LDS, and where there were any, they are added at the end, row by
// row, for the sequences that do attend them.  (Added in their block, by
// instructions other than the product's, they cost the product's loop 80
// registers.)
//
// What bounds it, whole steps: HBM in bf16 (24 sequences of 16 heads behind 65536
// rows, D = 128: 537 MB in 93 us, 5.8 TB/s; 64 of 32 behind 32768: 98 us) and in
// e4m3 up to 32 sequences (32 of 32 heads behind 32768 rows: 271 MB in 59 us); with
// 64 of e4m3 softmax, products and conversions, which overlap the loads only in
// part (82 us, with the rows in the caches 75); from 128 the matrix and the softmax
// instructions (bf16 137 us, e4m3 132); in float32 the products (64 of 32 behind
// 8192: 96 us, 89 TFLOP/s; over e4m3 104).  Short of that the two launches, a
// round trip each, and the parts, 17 MB written and read again at 64 of 32 heads.
#include "bf16_rows.h"
#include "cached.h"
#include "e4m3.h"
#include "pi_common.h"

namespace pi_attn {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// ---- rows as they lie in LDS -----------------------------------------------------
// Row r of a block: piece pc (16 bytes) at place pc ^ key(r) of the keys' and pc ^
// value(r) of the values'.
template <typename ST, int D>
struct Rows {
    static constexpr int RB = D * (int)sizeof(ST);   // bytes
    static constexpr int CPR = RB / 16;              // pieces
    // The keys' reads: 16 lanes, 16 rows, one piece each.
    static __device__ int key(int r) { return (RB >= 256 ? r : r / (256 / RB)) & (CPR < 16 ? CPR - 1 : 15); }
    // The values': 4 rows of 64 bytes (bf16), 8 rows of 32 bytes (e4m3, rows r..r+3 and r+8..r+11), rows r, r + 4, r + 8,
    // r + 12 of 64 bytes (float32).
    static __device__ int value(int r) {
        if constexpr (sizeof(ST) == 4) return 4 * ((r >> 2) & 3);
        if constexpr (sizeof(ST) == 2) return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1);
        return D == 128 ? 2 * ((r >> 1) & 1) + 4 * ((r >> 3) & 1) : 2 * ((r >> 3) & 1);
    }
    // The bits of a word's elements that are not finite: all ones for each of them.
    static __device__ unsigned not_finite(unsigned w) {
        if constexpr (sizeof(ST) == 4) return (w & 0x7f800000u) == 0x7f800000u ? ~0u : 0u;
        unsigned high;   // the top bit of each such element
        if constexpr (sizeof(ST) == 2) high = ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
        if constexpr (sizeof(ST) == 1) high = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;   // codes 0x7f, 0xff
        constexpr int N = sizeof(ST) == 2 ? 16 : 8;
        return (high >> (N - 1)) * (unsigned)((1ull << N) - 1);
    }
};

__device__ inline float element(float x) { return x; }
__device__ inline float element(__bf16 x) { return (float)x; }
__device__ inline float element(e4m3 x) { return __builtin_amdgcn_cvt_f32_fp8((int)x.code, 0); }

__device__ inline uint4 lds16(const unsigned char *p) { return *reinterpret_cast<const uint4 *>(p); }

// Eight bf16 values of eight codes, times scale.
__device__ inline bf16x8 widen8(unsigned lo, unsigned hi, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight weights p as sums of two bf16 terms: hi, p without its low 16 bits, and lo, the rest, which is below 2^-7 p and is
// rounded by at most 2^-8 of itself: 2^-15 p.  The rest of p (1 + 2^-23) is taken, which is not 0 where p is not, so that
// an infinite value has two products of one sign and stays infinite.
__device__ inline void split8(const float *p, bf16x8 &hi, bf16x8 &lo) {
    unsigned h[4];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const unsigned a = __float_as_uint(p[e]), b = __float_as_uint(p[e + 1]);
        h[e / 2] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        lo[e] = (__bf16)__builtin_fmaf(p[e], 1.0f + 0x1p-23f, -__uint_as_float(a & 0xffff0000u));
        lo[e + 1] = (__bf16)__builtin_fmaf(p[e + 1], 1.0f + 0x1p-23f, -__uint_as_float(b & 0xffff0000u));
    }
    hi = __builtin_bit_cast(bf16x8, make_uint4(h[0], h[1], h[2], h[3]));
}

// ---- one block of rows with a wavefront's queries -------------------------------
// NG groups of QB queries, which share the operands made of the rows; lane (c, g)
// belongs to query c of each.  KB rows a block; NS score slots, slot i being row
// slot_row(i, g) (four slots in a row are four rows in a row); the output's NO
// groups of four dims, group x being dims ODIM * x + 4 g + [0, 4).
template <typename T, typename ST, int D, int NG>
struct Mma;

template <typename ST, int D, int NG>
struct Mma<__bf16, ST, D, NG> {
    using R = Rows<ST, D>;
    static constexpr bool Q = sizeof(ST) == 1;
    static constexpr int QB = 32, KB = 32, NS = 16, NO = D / 8, ODIM = 8;
    bf16x8 qf[NG][D / 16];
    f32x16 o[NG][D / 32];

    static __device__ int slot_row(int i, int g) { return 8 * (i >> 2) + 4 * g + (i & 3); }
    // Product step s contracts dims dim0(s, g) + [0, 8).
    static __device__ int dim0(int s, int g) { return Q ? 32 * (s >> 1) + 16 * g + 8 * (s & 1) : 16 * s + 8 * g; }
    __device__ void query(int n, const __bf16 *q, int g, bool there) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
            qf[n][s] = there ? *reinterpret_cast<const bf16x8 *>(q + dim0(s, g)) : bf16x8{};
#pragma unroll
        for (int b = 0; b < D / 32; ++b) o[n][b] = f32x16{};
    }
    __device__ void query_landed() {
#pragma unroll
        for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                u32x4 u = __builtin_bit_cast(u32x4, qf[n][s]);
                asm volatile("" : "+v"(u));
                qf[n][s] = __builtin_bit_cast(bf16x8, u);
            }
    }
    __device__ void scale(int n, float a) {
#pragma unroll
        for (int b = 0; b < D / 32; ++b) o[n][b] *= a;
    }
    __device__ float &at(int n, int x, int e) { return reinterpret_cast<float *>(&o[n][x >> 2])[4 * (x & 3) + e]; }
    // A block's operands as they lie in LDS.
    uint4 kr[R::CPR / 2];
    uint2 vr[2][D / 32][Q ? 1 : 2];
    __device__ void read_keys(const unsigned char *kt, int c, int g) {
        const unsigned char *row = kt + c * R::RB;
        const int sw = R::key(c);
#pragma unroll
        for (int u = 0; u < R::CPR / 2; ++u) kr[u] = lds16(row + ((2 * u + g) ^ sw) * 16);
    }
    __device__ void read_values(const unsigned char *vt, int lane) {
        const int g = lane >> 5, half = (lane >> 4) & 1;
        if constexpr (Q) {
            // the 16 lanes of a half: eight rows (two lanes each) by 16 dims
            const int i = lane & 15, pr = i >> 1, row = 8 * (pr >> 2) + 4 * g + (pr & 3);
            const unsigned char *at = vt + row * R::RB + (i & 1) * 8;
            const int sw = R::value(row);
#pragma unroll
            for (int cc = 0; cc < 2; ++cc)
#pragma unroll
                for (int b = 0; b < D / 32; ++b)
                    vr[cc][b][0] = __builtin_bit_cast(
                        uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                                   (lds_i32x2 *)(at + 16 * cc * R::RB + ((2 * b + half) ^ sw) * 16)));
        } else {
            const int r = (lane >> 2) & 3, qd = lane & 3;
            const unsigned char *at = vt + (4 * g + r) * R::RB + (qd & 1) * 8;
            const int sw = R::value(r);
#pragma unroll
            for (int cc = 0; cc < 2; ++cc)
#pragma unroll
                for (int b = 0; b < D / 32; ++b)
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh)
                        vr[cc][b][hh] = __builtin_bit_cast(
                            uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (lds_s16x4 *)(at + (16 * cc + 8 * hh) * R::RB +
                                                     ((4 * b + 2 * half + (qd >> 1)) ^ sw) * 16)));
        }
    }
    __device__ void scores(float kscale, float (&s)[NG][NS]) const {
        f32x16 sc[NG] = {};
#pragma unroll
        for (int u = 0; u < D / 16; ++u) {
            bf16x8 kf;
            if constexpr (Q) {
                const uint4 k = kr[u >> 1];
                kf = u & 1 ? widen8(k.z, k.w, kscale) : widen8(k.x, k.y, kscale);
            } else {
                kf = __builtin_bit_cast(bf16x8, kr[u]);
            }
#pragma unroll
            for (int n = 0; n < NG; ++n) sc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[n][u], sc[n], 0, 0, 0);
        }
#pragma unroll
        for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int i = 0; i < NS; ++i) s[n][i] = sc[n][i];
    }
    __device__ void values(const float (&p)[NG][NS]) {
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) {
            bf16x8 hi[NG], lo[NG];
#pragma unroll
            for (int n = 0; n < NG; ++n) split8(&p[n][8 * cc], hi[n], lo[n]);
#pragma unroll
            for (int b = 0; b < D / 32; ++b) {
                bf16x8 vf;
                if constexpr (Q) {
                    vf = widen8(vr[cc][b][0].x, vr[cc][b][0].y, 1.0f);
                } else {
                    const uint2 r0 = vr[cc][b][0], r8 = vr[cc][b][1];   // rows from 0 and 8 on
                    vf = __builtin_bit_cast(bf16x8, make_uint4(r0.x, r0.y, r8.x, r8.y));
                }
#pragma unroll
                for (int n = 0; n < NG; ++n) {
                    o[n][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, hi[n], o[n][b], 0, 0, 0);
                    o[n][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, lo[n], o[n][b], 0, 0, 0);
                }
            }
        }
    }
    // This lane's part of its query's product with a row (without a scale).
    __device__ float dot(int n, const ST *k, int g) const {
        float x = 0.0f;
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) x = __builtin_fmaf((float)qf[n][s][e], element(k[dim0(s, g) + e]), x);
        return x;
    }
};

template <typename ST, int D, int NG>
struct Mma<float, ST, D, NG> {
    using R = Rows<ST, D>;
    static constexpr bool Q = sizeof(ST) == 1;
    static constexpr int QB = 16, KB = 16, NS = 4, NO = D / 16, ODIM = 16;
    f32x4 qf[NG][D / 16];
    f32x4 o[NG][D / 16];

    static __device__ int slot_row(int i, int g) { return 4 * g + i; }
    // Product steps (s, e) contract dims dim0(s, g) + e.
    static __device__ int dim0(int s, int g) { return Q ? 64 * (s >> 2) + 16 * g + 4 * (s & 3) : 16 * s + 4 * g; }
    __device__ void query(int n, const float *q, int g, bool there) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qf[n][s] = there ? *reinterpret_cast<const f32x4 *>(q + dim0(s, g)) : f32x4{};
#pragma unroll
        for (int b = 0; b < D / 16; ++b) o[n][b] = f32x4{};
    }
    __device__ void query_landed() {
#pragma unroll
        for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int s = 0; s < D / 16; ++s) asm volatile("" : "+v"(qf[n][s]));
    }
    __device__ void scale(int n, float a) {
#pragma unroll
        for (int b = 0; b < D / 16; ++b) o[n][b] *= a;
    }
    __device__ float &at(int n, int x, int e) { return reinterpret_cast<float *>(&o[n][x])[e]; }
    // A block's operands as they lie in LDS.
    uint4 kr[R::CPR / 4];
    unsigned vr[D / 16][Q ? 1 : NS];   // e4m3: four rows of dim 16 b + c
    __device__ void read_keys(const unsigned char *kt, int c, int g) {
        const unsigned char *row = kt + c * R::RB;
        const int sw = R::key(c);
#pragma unroll
        for (int u = 0; u < R::CPR / 4; ++u) kr[u] = lds16(row + ((4 * u + g) ^ sw) * 16);
    }
    __device__ void read_values(const unsigned char *vt, int lane) {
        const int c = lane & 15, g = lane >> 4;
        if constexpr (Q) {
            // four rows (two lanes each) of 16 dims, then the same rows of the next 16
            const int pr = c >> 1, row = 4 * g + (pr & 3);
            const unsigned char *at = vt + row * R::RB + (c & 1) * 8;
            const int sw = R::value(row);
#pragma unroll
            for (int b = 0; b < D / 16; b += 2) {
                const i32x2 y =
                    __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(at + ((b + (pr >> 2)) ^ sw) * 16));
                vr[b][0] = (unsigned)y.x;
                vr[b + 1][0] = (unsigned)y.y;
            }
        } else {
#pragma unroll
            for (int b = 0; b < D / 16; ++b)
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    const int row = 4 * g + i;
                    vr[b][i] = *reinterpret_cast<const unsigned *>(
                        vt + row * R::RB + ((4 * b + (c >> 2)) ^ R::value(row)) * 16 + (c & 3) * 4);
                }
        }
    }
    // In four chains.
    __device__ void scores(float kscale, float (&s)[NG][NS]) const {
        f32x4 sc[NG][4] = {};
#pragma unroll
        for (int u = 0; u < D / 16; ++u) {
            float kf[4];
            if constexpr (Q) {
                const uint4 k = kr[u >> 2];
                const unsigned w[4] = {k.x, k.y, k.z, k.w};
                e4m3_unpack4(w[u & 3], kf);
#pragma unroll
                for (int e = 0; e < 4; ++e) kf[e] *= kscale;
            } else {
                const f32x4 k = __builtin_bit_cast(f32x4, kr[u]);
#pragma unroll
                for (int e = 0; e < 4; ++e) kf[e] = k[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int n = 0; n < NG; ++n)
                    sc[n][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[n][u][e], sc[n][e], 0, 0, 0);
        }
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            const f32x4 sum = (sc[n][0] + sc[n][1]) + (sc[n][2] + sc[n][3]);
#pragma unroll
            for (int i = 0; i < NS; ++i) s[n][i] = sum[i];
        }
    }
    // Step i contracts rows 4 g + i, whose weights are the score slots i.
    __device__ void values(const float (&p)[NG][NS]) {
#pragma unroll
        for (int b = 0; b < D / 16; ++b) {
            float vf[NS];
            if constexpr (Q) {
                e4m3_unpack4(vr[b][0], vf);
            } else {
#pragma unroll
                for (int i = 0; i < NS; ++i) vf[i] = __uint_as_float(vr[b][i]);
            }
#pragma unroll
            for (int i = 0; i < NS; ++i)
#pragma unroll
                for (int n = 0; n < NG; ++n)
                    o[n][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i], p[n][i], o[n][b], 0, 0, 0);
        }
    }
    __device__ float dot(int n, const ST *k, int g) const {
        float x = 0.0f;
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) x = __builtin_fmaf(qf[n][s][e], element(k[dim0(s, g) + e]), x);
        return x;
    }
};

// A weight 2^(s c - m) of a score s, m at least the largest of the rounded s c.  The product is rounded with the
// difference, which costs nothing and keeps its last bits; but then all weights are off by 2^r, r the rounding of m.  WIDE,
// once some |m| has passed 2^22 (r up to 1/4; at 2^32 it would be 256): the product is rounded first, as m is.
constexpr float kWide = 0x1p22f;

// m is set above the largest score so far, so that few later blocks raise it and rescale the state; weights are at most 1
// either way.  64 sequences of 32 heads behind 32768 e4m3 rows, D = 128, 85 -> 81 us, 128 behind bf16 146 -> 138.
constexpr float kHeadroom = 4.0f;

template <bool WIDE>
__device__ inline float weight(float s, float c, float m) {
    if constexpr (WIDE) {
#pragma clang fp contract(off)
        const float x = s * c;
        return __builtin_amdgcn_exp2f(x - m);
    }
    return __builtin_amdgcn_exp2f(__builtin_fmaf(s, c, -m));
}

// Maximum and sum over the lanes of a query.
__device__ inline float other_row(float x) {   // of the neighbouring 16 lanes
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(__lane_id() & 16 ? p[0] : p[1]);
}

// Smallest and largest of the wavefront's whole numbers: round the 16 lanes of a
// row, then across rows.
template <bool MAX>
__device__ inline int wave_extreme(int x) {
    auto join = [](int a, int b) { return MAX ? max(a, b) : min(a, b); };
    x = join(x, __builtin_amdgcn_mov_dpp(x, 0x128, 0xF, 0xF, false));
    x = join(x, __builtin_amdgcn_mov_dpp(x, 0x124, 0xF, 0xF, false));
    x = join(x, __builtin_amdgcn_mov_dpp(x, 0x122, 0xF, 0xF, false));
    x = join(x, __builtin_amdgcn_mov_dpp(x, 0x121, 0xF, 0xF, false));
    x = join(x, __float_as_int(other_row(__int_as_float(x))));
    x = join(x, __float_as_int(other_half(__int_as_float(x))));
    return __builtin_amdgcn_readfirstlane(x);
}

template <int QB>
__device__ inline float query_max(float x) {
    if constexpr (QB == 16) x = fmaxf(x, other_row(x));
    return fmaxf(x, other_half(x));
}

template <int QB>
__device__ inline float query_sum(float x) {
    if constexpr (QB == 16) x += other_row(x);
    return x + other_half(x);
}

// ---- the ring ----------------------------------------------------------------------
// G wavefronts side by side over the queries (NG groups each), RS shares of a
// stage's blocks.  OWN: a ring for each wavefront, whose stages are one block;
// else one for all, of SR rows a stage.
//
// Two work-groups of four wavefronts share a CU where two stages of each fit.
// float32 work-groups of one ring have eight and a CU each.
template <typename T, typename ST, int D, int G, int NG>
struct Shape {
    using Type = T;
    using M = Mma<T, ST, D, NG>;
    using R = Rows<ST, D>;
    using Stored = ST;
    static constexpr int DIM = D;
    static constexpr bool Q = sizeof(ST) == 1;
    static constexpr bool OWN = G == 1;
    static constexpr int WAVES = OWN || sizeof(T) == 2 ? 4 : 8, NT = 64 * WAVES;
    static constexpr int RS = WAVES / G;
    static constexpr int SIDE = G, GROUPS = NG;
    static constexpr int QT = M::QB * NG * G;                                     // queries of a work-group
    static constexpr bool SMALL = M::KB * RS <= 64 && R::CPR >= WAVES;            // whole loads of 64 rows
    static constexpr int SR = OWN ? M::KB : SMALL ? 64 : 128;                     // rows of a stage
    static constexpr int TR = OWN ? WAVES * M::KB : SR;                           // rows that a work-group takes at a time
    static constexpr int BL = OWN ? 1 : SR / M::KB / RS;                          // blocks of a wavefront among them
    static constexpr int TABLE = SR * R::RB;                                      // bytes of the stage's keys
    static constexpr int STAGE = 2 * TABLE + (Q ? 8 * SR : 0);                    // and values, scale bytes (a word each)
    static constexpr int RINGS = OWN ? WAVES : 1;
    static constexpr bool TWO = WAVES == 4 && 2 * RINGS * STAGE <= 80 << 10 && !(D == 128 && NG == 2);
    // as many stages as fit, two at least and four at most
    static constexpr int FIT = (TWO ? 80 << 10 : 156 << 10) / (RINGS * STAGE);
    static constexpr int NST = FIT > 4 ? 4 : FIT;
    static constexpr int KI = SR * R::CPR / 64 / (OWN ? 1 : WAVES);   // a wavefront's loads of a stage's keys
    static constexpr int LOADS = 2 * KI + (Q ? (OWN ? 2 : 1) : 0);    // and of everything
    static constexpr int PITCH = D + 4;                               // floats from one query's o to the next
    static constexpr int RING_BYTES = RINGS * NST * STAGE;
    static constexpr int JOIN_BYTES = WAVES * M::QB * (PITCH * 4 + 16);   // the wavefronts' states of a group
    static constexpr int LDS = RING_BYTES > JOIN_BYTES ? RING_BYTES : JOIN_BYTES;
    static_assert(SR * R::CPR % (64 * (OWN ? 1 : WAVES)) == 0 && BL >= 1 && NST >= 2, "whole loads, whole blocks");
};

// lds_fetch16 to a 32-bit LDS address (a pointer's arithmetic is in 64 bits).
// ONCE: of rows that are not to be kept in the caches.
template <bool ONCE>
__device__ inline void fetch16(u32x4 rsrc, int voff, unsigned lds_at) {
    const unsigned m0 = __builtin_amdgcn_readfirstlane(lds_at);
    if constexpr (ONCE) {
        asm volatile("buffer_load_dwordx4 %0, %1, 0 offen nt lds" ::"v"(voff), "s"(rsrc), "{m0}"(m0));
    } else {
        asm volatile("buffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "{m0}"(m0));
    }
}

// One byte a lane into the words at lds_at + 4 * lane.
__device__ inline void fetch1(u32x4 rsrc, int voff, unsigned lds_at) {
    const unsigned m0 = __builtin_amdgcn_readfirstlane(lds_at);
    asm volatile("buffer_load_ubyte %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "{m0}"(m0));
}

// Waits until at most N of this wavefront's loads are on their way.
template <int N>
__device__ inline void wait_loads() {
    static_assert(N < 64, "a six-bit counter");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}

// ONCE: the prefix's rows are not kept in the caches.
template <typename S, bool ONCE>
__global__ __launch_bounds__(S::NT, (S::TWO || S::WAVES == 8 ? 2 : 1)) void prefix_kernel(CachedParams p, int n_qt,
                                                                                  uint32_t n_logical) {
    using T = typename S::Type;
    using ST = typename S::Stored;
    using M = typename S::M;
    using R = typename S::R;
    constexpr bool Q = S::Q;
    constexpr int D = S::DIM, G = S::SIDE, NG = S::GROUPS, WAVES = S::WAVES, NT = S::NT;
    constexpr int RS = S::RS, QB = M::QB, KB = M::KB, QT = S::QT, NST = S::NST;
    __shared__ __align__(16) unsigned char lds[S::LDS];
    __shared__ int s_cleaned;   // !OWN: some wavefront has

    const uint32_t logical = xcd_remap(blockIdx.x, n_logical);
    if (logical >= n_logical) return;
    const DecodeParams &d = p.d;
    const DivMod qt_of = divmod(logical, n_qt), chunk_of = divmod(qt_of.quot, p.chunks);
    const int qt = (int)qt_of.rem, x = (int)chunk_of.rem, h = (int)chunk_of.quot;
    // The chunk's tiles x, x + chunks, ..., the last one first: every window that
    // meets the prefix ends with it, so the first loads wait for no length.
    const int plen = p.plen, reach = chunk_end(p, x), step = p.chunks * S::TR;
    const int all = (p.near - 1) / S::TR + 1;   // of all chunks
    const int last = x + (all - 1 - x) / p.chunks * p.chunks, mine = last / p.chunks + 1;   // and of this one
    const int row_last = plen - p.near + last * S::TR;

    const int tid = threadIdx.x, lane = __lane_id();
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int qg = w % G, rs = w / G;
    const int c = lane % QB, g = lane / QB;

    // This lane's pieces of a stage: byte offsets from the stage's first row.
    unsigned char *const ring = lds + (S::OWN ? w * NST * S::STAGE : 0);
    int koff[S::KI], voff[S::KI];
#pragma unroll
    for (int u = 0; u < S::KI; ++u) {
        const int y = 64 * (S::OWN ? u : u * WAVES + w) + lane, r = y / R::CPR, pc = y % R::CPR;
        koff[u] = r * R::RB + (pc ^ R::key(r)) * 16;
        voff[u] = r * R::RB + (pc ^ R::value(r)) * 16;
    }
    // First row of this wavefront's stage of tile m.
    auto stage_row = [&](int m) { return row_last - m * step + (S::OWN ? w * KB : 0); };
    // The stage that is fetched next: its first row's address in each table, how
    // many rows the prefix has from there on, and its place.
    const int64_t row_first = h * p.pcap + stage_row(0);
    const uint8_t *kat = (const uint8_t *)p.k_prefix + row_first * R::RB;
    const uint8_t *vat = (const uint8_t *)p.v_prefix + row_first * R::RB;
    const uint8_t *kbat = p.k_prefix_exp + row_first, *vbat = p.v_prefix_exp + row_first;
    // The bytes of a stage for all: 64 rows a wavefront, the keys' by one half of
    // them, the values' by the other (some of them the same ones).
    const int byte_row = 64 * (w % (WAVES / 2) % (S::SR < 64 ? 1 : S::SR / 64)) + lane;
    if (Q && !S::OWN) kbat = w >= WAVES / 2 ? vbat : kbat;
    int left = plen - stage_row(0);
    const unsigned ring_at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void *)ring;
    unsigned to = ring_at;
    // Fetches it; rows behind the prefix read as zeros.
    auto fetch = [&]() __attribute__((always_inline)) {
        const int rows = min(max(left, 0), S::SR);
        const u32x4 rk = raw_rsrc(kat, rows * R::RB), rv = raw_rsrc(vat, rows * R::RB);
#pragma unroll
        for (int u = 0; u < S::KI; ++u) fetch16<ONCE>(rk, koff[u], to + 1024 * (S::OWN ? u : u * WAVES + w));
#pragma unroll
        for (int u = 0; u < S::KI; ++u) fetch16<ONCE>(rv, voff[u], to + S::TABLE + 1024 * (S::OWN ? u : u * WAVES + w));
        if constexpr (Q) {
            const unsigned bytes = to + 2 * S::TABLE;
            if constexpr (S::OWN) {
                const u32x4 bk = raw_rsrc(kbat, rows), bv = raw_rsrc(vbat, rows);
                if (lane < S::SR) {
                    fetch1(bk, lane, bytes);
                    fetch1(bv, lane, bytes + 4 * S::SR);
                }
            } else {
                fetch1(raw_rsrc(kbat, rows), byte_row, bytes + 4 * (byte_row - lane + (w >= WAVES / 2 ? S::SR : 0)));
            }
            kbat -= step;
            vbat -= step;
        }
        kat -= (int64_t)step * R::RB;
        vat -= (int64_t)step * R::RB;
        left += step;
        to += S::STAGE;
        to = to == ring_at + NST * S::STAGE ? ring_at : to;
    };
#pragma unroll
    for (int m = 0; m < NST - 1; ++m)
        if (m < mine) fetch();
    if (!S::OWN && tid == 0) s_cleaned = 0;   // before the first stage's barrier

    // Where the window of a sequence begins; INT32_MAX for none.
    auto low_of = [&](int s) {
        if (s >= d.S) return INT32_MAX;
        const int n = d.len_in[s];
        return n >= 0 && n < d.cap ? window_lo(plen + n, d.k) : INT32_MAX;
    };
    // Over the tile's sequences that meet the chunk: where the first window
    // begins, and the last.
    int lo_min = INT32_MAX, lo_max = 0;
#pragma unroll
    for (int i = 0; i < QT; i += 64) {
        const int a = i + lane < QT ? low_of(qt * QT + i + lane) : INT32_MAX;
        lo_min = min(lo_min, a);
        if (a < reach) lo_max = max(lo_max, a);
    }
    lo_min = wave_extreme<false>(lo_min);
    lo_max = wave_extreme<true>(lo_max);
    if (lo_min >= reach) {   // nothing for anybody, once the loads have landed
        wait_loads<0>();
        return;
    }
    const int tiles = (row_last + S::TR - 1 - lo_min) / step + 1;   // that some window meets

    int lo[NG];
    float bias[NG], m[NG], l[NG];
    M mm;
    const int s0 = qt * QT + qg * NG * QB + c;   // this lane's queries: s0, s0 + QB
#pragma unroll
    for (int n = 0; n < NG; ++n) {
        const int s = s0 + n * QB;
        lo[n] = low_of(s);
        mm.query(n, (const T *)d.q_new + ((int64_t)s * d.H + h) * D, g, s < d.S);
        bias[n] = s < d.S ? fusion_bias(d.gate[s * d.gss + h * d.gsh], true).local : 0.0f;
        m[n] = -INFINITY;
        l[n] = 0.0f;
    }
    // The queries are waited for here: left to the compiler, the wait stands where
    // they are used first, in the loop, and there it is for the stages, too.
    mm.query_landed();
    int lo_first = lo[0];
#pragma unroll
    for (int n = 1; n < NG; ++n) lo_first = min(lo_first, lo[n]);
    const bool clamped = d.clamp > 0.0f;
    const float c2 = clamped ? 1.0f : d.scale * kLog2e;   // to log2 units

    // Zeros for the values of a block that are not finite.  Wavefronts that share
    // the block may all do so: each has written its zeros before it reads.
    bool cleaned = false;   // wave-uniform
    bool wide = false;      // and so
    auto clean = [&](unsigned char *vb, unsigned *vbytes) {
        cleaned = true;
        if (!S::OWN) s_cleaned = 1;
#pragma unroll 1
        for (int i = 0; i < KB * R::RB / 1024; ++i) {
            uint4 v = lds16(vb + 1024 * i + 16 * lane);
            v.x &= ~R::not_finite(v.x), v.y &= ~R::not_finite(v.y), v.z &= ~R::not_finite(v.z), v.w &= ~R::not_finite(v.w);
            *reinterpret_cast<uint4 *>(vb + 1024 * i + 16 * lane) = v;
        }
        if (Q && lane < KB && vbytes[lane] >= 247) vbytes[lane] = 0;
    };

    // One block: rows [j0, j0 + KB), rows [blk * KB, + KB) of the stage at kt.
    auto block = [&](unsigned char *stage, int blk, int j0) __attribute__((always_inline)) {
        unsigned char *kb = stage + blk * KB * R::RB, *vb = kb + S::TABLE;
        unsigned *kbytes = reinterpret_cast<unsigned *>(stage + 2 * S::TABLE) + blk * KB, *vbytes = kbytes + S::SR;
        const bool masked = j0 < lo_max;   // some sequence's window begins behind the block's first row
        if (masked) {
            unsigned bad = 0;
#pragma unroll
            for (int i = 0; i < KB * R::RB / 1024; ++i) {
                const uint4 v = lds16(vb + 1024 * i + 16 * lane);
                bad |= R::not_finite(v.x) | R::not_finite(v.y) | R::not_finite(v.z) | R::not_finite(v.w);
            }
            // a code's value past the largest float: 256 * 2^120
            const bool past = Q && lane < KB && vbytes[lane] >= 247;
            if (__builtin_amdgcn_ballot_w64(bad || past)) clean(vb, vbytes);
        }
        // Every operand is on its way from LDS before the first is used.
        const unsigned kbyte = Q ? kbytes[c] : 0;
        uint4 vbyte[Q ? M::NS / 4 : 1];
        mm.read_keys(kb, c, g);
        if constexpr (Q) {
#pragma unroll
            for (int i = 0; i < M::NS / 4; ++i)
                vbyte[i] = *reinterpret_cast<const uint4 *>(vbytes + M::slot_row(4 * i, g));
        }
        mm.read_values(vb, lane);
        __builtin_amdgcn_sched_barrier(0);
        float sc[NG][M::NS];
        mm.scores(e4m3_scale(kbyte), sc);
        if (clamped) {
#pragma unroll
            for (int n = 0; n < NG; ++n)
#pragma unroll
                for (int i = 0; i < M::NS; ++i)
                    sc[n][i] = clamped_logit(sc[n][i] * d.scale + bias[n], d.clamp) * kLog2e;
        }
        if (masked || j0 + KB > plen) {
#pragma unroll
            for (int n = 0; n < NG; ++n)
#pragma unroll
                for (int i = 0; i < M::NS; ++i) {
                    const int j = j0 + M::slot_row(i, g);
                    sc[n][i] = j >= lo[n] && j < plen ? sc[n][i] : -INFINITY;
                }
        }
        float mx[NG];
        bool raised = false;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            mx[n] = sc[n][0];
#pragma unroll
            for (int i = 1; i < M::NS; ++i) mx[n] = fmaxf(mx[n], sc[n][i]);
            mx[n] = query_max<QB>(mx[n]) * c2;
            raised |= mx[n] > m[n];
        }
        if (__builtin_amdgcn_ballot_w64(raised)) {
            bool large = false;
#pragma unroll
            for (int n = 0; n < NG; ++n) {
                large |= mx[n] > m[n] && fabsf(mx[n]) > kWide;
                const float m_new = mx[n] > m[n] ? mx[n] + kHeadroom : m[n];
                const float alpha = mx[n] > m[n] ? __builtin_amdgcn_exp2f(m[n] - m_new) : 1.0f;
                m[n] = m_new;
                l[n] *= alpha;
                mm.scale(n, alpha);
            }
            wide |= __builtin_amdgcn_ballot_w64(large) != 0;
        }
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            const float m_use = m[n] == -INFINITY ? 0.0f : m[n];
            if (wide) {
#pragma unroll
                for (int i = 0; i < M::NS; ++i) sc[n][i] = weight<true>(sc[n][i], c2, m_use);
            } else {
#pragma unroll
                for (int i = 0; i < M::NS; ++i) sc[n][i] = weight<false>(sc[n][i], c2, m_use);
            }
#pragma unroll
            for (int i = 0; i < M::NS; ++i) l[n] += sc[n][i];
        }
        if constexpr (Q) {
#pragma unroll
            for (int i = 0; i < M::NS; i += 4) {
                const uint4 b = vbyte[i / 4];
                const float f[4] = {e4m3_scale(b.x), e4m3_scale(b.y), e4m3_scale(b.z), e4m3_scale(b.w)};
#pragma unroll
                for (int n = 0; n < NG; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[n][i + e] *= f[e];
            }
        }
        mm.values(sc);
    };

    unsigned char *stage = ring;
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) {
        // Stage t has landed when at most the loads of the stages behind it are on
        // their way.
        if (t + NST - 1 <= tiles) {
            wait_loads<(NST - 2) * S::LOADS>();
        } else {
            wait_loads<0>();
        }
        // The stage that is fetched next is the one that was read last: by this
        // wavefront alone, or by all, who are past it at the barrier.
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        if constexpr (!S::OWN) __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        if (t + NST - 1 < tiles) fetch();
        const int first = stage_row(t);
#pragma unroll
        for (int b = 0; b < S::BL; ++b) {
            const int blk = S::OWN ? 0 : b * RS + rs, j0 = first + blk * KB;
            // rows that the group's sequences meet
            if (j0 < plen && __builtin_amdgcn_ballot_w64(lo_first < min(j0 + KB, plen))) block(stage, blk, j0);
        }
        stage += S::STAGE;
        stage = stage == ring + NST * S::STAGE ? ring : stage;
    }
#pragma unroll
    for (int n = 0; n < NG; ++n) l[n] = query_sum<QB>(l[n]);

    if constexpr (!S::OWN) {
        __syncthreads();
        cleaned = s_cleaned != 0;
    }
    if (cleaned) {
        // The rows of this wavefront's masked blocks that have values which are not
        // finite (or too large a scale).
        const int64_t head = h * p.pcap;
#pragma unroll 1
        for (int y = 0; y < tiles * S::BL; ++y) {
            const int j0 = stage_row(y / S::BL) + (S::OWN ? 0 : (y % S::BL * RS + rs) * KB);
            if (j0 >= lo_max) continue;
#pragma unroll 1
            for (int j = j0; j < min(j0 + KB, plen); ++j) {
                const ST *kr = (const ST *)p.k_prefix + (head + j) * D, *vr = (const ST *)p.v_prefix + (head + j) * D;
                const unsigned vbyte = Q ? p.v_prefix_exp[head + j] : 127;
                unsigned bad = 0;
#pragma unroll
                for (int i = 0; i < R::RB; i += 256)
                    bad |= R::not_finite(reinterpret_cast<const unsigned *>(vr)[(i / 4 + lane) % (R::RB / 4)]);
                const bool past = Q && vbyte >= 247;
                if (!past && !__builtin_amdgcn_ballot_w64(bad != 0)) continue;
#pragma unroll
                for (int n = 0; n < NG; ++n) {
                    float sc = query_sum<QB>(mm.dot(n, kr, g));
                    if constexpr (Q) sc *= e4m3_scale(p.k_prefix_exp[head + j]);
                    if (clamped) sc = clamped_logit(sc * d.scale + bias[n], d.clamp) * kLog2e;
                    const float pr = wide ? weight<true>(sc, c2, m[n]) : weight<false>(sc, c2, m[n]);
                    const bool in = j >= lo[n];
#pragma unroll
                    for (int z = 0; z < M::NO; ++z) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float v = element(vr[M::ODIM * z + 4 * g + e]);
                            const bool there = in && (past || !(fabsf(v) < INFINITY));
                            mm.at(n, z, e) += there ? pr * (Q ? e4m3_scale(vbyte) * v : v) : 0.0f;
                        }
                        __builtin_amdgcn_sched_barrier(0);   // few registers at a time
                    }
                }
            }
        }
    }

    // The states of the RS wavefronts of the same queries, joined on the way out:
    // through LDS, so that the parts are written in whole lines.
    wait_loads<0>();   // stages that nobody needed
    constexpr int QUADS = D / 4;
    float *const o_at = reinterpret_cast<float *>(lds);                             // [wavefront][query][PITCH]
    float4 *const ml_at = reinterpret_cast<float4 *>(o_at + WAVES * QB * S::PITCH);   // [wavefront][query]
#pragma unroll
    for (int n = 0; n < NG; ++n) {
        __syncthreads();
#pragma unroll
        for (int y = 0; y < M::NO; ++y) {
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = mm.at(n, y, e);
            *reinterpret_cast<f32x4 *>(o_at + (w * QB + c) * S::PITCH + M::ODIM * y + 4 * g) = v;
        }
        if (g == 0) ml_at[w * QB + c] = make_float4(m[n], l[n], __int_as_float(lo[n]), 0.0f);
        __syncthreads();
#pragma unroll 4
        for (int i = tid; i < G * QB * QUADS; i += NT) {
            const int q = i / QUADS, quad = i % QUADS;   // of wavefront r * G + q / QB
            if (__float_as_int(ml_at[q].z) >= reach) continue;   // no window here, or no sequence
            float top = -INFINITY;
#pragma unroll
            for (int r = 0; r < RS; ++r) top = fmaxf(top, ml_at[r * G * QB + q].x);
            const float use = top == -INFINITY ? 0.0f : top;
            f32x4 sum = {};
            float total = 0.0f;
#pragma unroll
            for (int r = 0; r < RS; ++r) {
                const float4 ml = ml_at[r * G * QB + q];
                const float f = __builtin_amdgcn_exp2f(ml.x - use);
                total += f * ml.y;
                sum += f * *reinterpret_cast<const f32x4 *>(o_at + (r * G * QB + q) * S::PITCH + 4 * quad);
            }
            const int s = qt * QT + (q / QB * NG + n) * QB + q % QB;
            const int64_t at = (int64_t)x * d.S * d.H + (int64_t)s * d.H + h;
            *reinterpret_cast<f32x4 *>(p.part_o + at * D + 4 * quad) = sum;
            if (quad == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(top, total);
        }
    }
}

// Calls f with the Shape for a problem: one work-group for all sequences as far
// as that goes.  Two groups of queries a wavefront share what the rows' operands
// cost, where their registers leave two wavefronts a SIMD (D = 128: bf16 needs
// more than 256 a lane, and one wavefront a SIMD is slower than two of one group;
// float32 in the larger work-groups, too).
template <typename T, typename ST, int D, typename F>
auto with_queries(int S, F f) {
    constexpr int QB = Mma<T, ST, D, 1>::QB;
    if (S <= QB) return f(Shape<T, ST, D, 1, 1>());
    if constexpr (D == 64) {
        if (S <= 2 * QB) return f(Shape<T, ST, D, 1, 2>());
        return S <= 4 * QB ? f(Shape<T, ST, D, 2, 2>()) : f(Shape<T, ST, D, 4, 2>());
    } else {
        if (S <= 2 * QB) {
            if constexpr (sizeof(T) == 4) return f(Shape<T, ST, D, 1, 2>());
            else return f(Shape<T, ST, D, 2, 1>());
        }
        if constexpr (sizeof(T) == 4) {
            if (S > 4 * QB) return f(Shape<T, ST, D, 8, 1>());
        }
        return f(Shape<T, ST, D, 4, 1>());
    }
}

template <typename T, typename ST, typename F>
auto with_dim(const CachedParams &p, F f) {
    return p.d.D == 64 ? with_queries<T, ST, 64>(p.d.S, f) : with_queries<T, ST, 128>(p.d.S, f);
}

template <typename F>
auto with_shape(const CachedParams &p, bool bf16, F f) {
    if (p.k_prefix_exp) return bf16 ? with_dim<__bf16, e4m3>(p, f) : with_dim<float, e4m3>(p, f);
    return bf16 ? with_dim<__bf16, __bf16>(p, f) : with_dim<float, float>(p, f);
}

}  // namespace

// ONCE, by the bytes of the prefix rows that windows reach: the step of one layer
// reads them once, and the other layers' come before the next.  With sixteen
// layers in turn (more than the last-level cache together), kept and not: 16 MB
// 17.5 and 16.2 us (bf16, D = 128, 16 sequences of 32 heads), 67 MB 29.4 and 26.4
// (e4m3, 32 of 32), 134 MB 34.2 and 30.5, 537 MB 106 and 94.  With three, which
// the cache holds up to 67 MB, the other way round there, 14.5 and 15.5, 24.5 and
// 26.1.  Where work-groups of several tiles of sequences read the same rows, they
// are kept.
constexpr int64_t kKeepPrefix = 12 << 20;

PrefixShape prefix_shape(const CachedParams &p, bool bf16) {
    return with_shape(p, bf16, [](auto s) {
        using S = decltype(s);
        return PrefixShape{S::QT, S::TR, S::TWO ? 2 : 1};
    });
}

hipError_t launch_prefix(const CachedParams &p, bool bf16, hipStream_t stream) {
    return with_shape(p, bf16, [&](auto s) {
        using S = decltype(s);
        const int n_qt = (p.d.S + S::QT - 1) / S::QT;
        const int64_t n = (int64_t)p.d.H * p.chunks * n_qt;
        const bool once = n_qt == 1 && 2 * (int64_t)p.d.H * p.near * S::R::RB > kKeepPrefix;
        return launch_kernel(once ? prefix_kernel<S, true> : prefix_kernel<S, false>, dim3((unsigned)xcd_grid(n)),
                             dim3(S::NT), stream, p, n_qt, (uint32_t)n);
    });
}

}  // namespace pi_attn
