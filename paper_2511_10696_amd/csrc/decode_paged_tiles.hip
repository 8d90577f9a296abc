// decode_paged_tiles.hip -- the decode step over a paged cache on the matrix
// cores: pages in bf16 or e4m3, up to 16 query heads of a key head at a time.
// (The new row and the partner are rows of the tiles, behind the window's last.)
//
// A work-group is a sequence, a key head, up to 16 of its query heads and a range
// of the window; its wavefronts take tiles of 32 rows in turn, each with a running
// maximum, sum and accumulator for every query, joined at the end.
//
// A tile's keys, then its values, go from registers (whole rows, 16 bytes a lane)
// into the wavefront's own 32 rows of LDS, as bf16; the registers are free for the
// next tile's loads at once, which stay under way meanwhile.  No wavefront waits for
// another before the end.  (Keys loaded in the layout of the scores' operand, 64
// bytes of each of 16 rows an instruction, need no LDS, but neighbouring lanes are
// then in different rows, which costs the vector memory path four times the cycles.)
//
// MFMA layout (v_mfma_f32_16x16x32_bf16; lane = (c, g) = (l % 16, l / 16)).  Scores
// S^T = K Q^T, 16 rows at a time: A = K, lane (c, g) holding elements 32x + 8g.. of
// row c, B = Q^T the same of query c; C holds rows 4g + i of query c.  Output O^T +=
// V^T P^T over 32 rows: B = P^T is the weights of two blocks where they are (rows 4g
// + i and 16 + 4g + i), A = V^T comes by LDS transpose reads of the same rows.
//
// Precision.  The products take bf16: cached rows are that, or e4m3, whose codes and
// scales together are bf16 numbers.  A query (turned, not rounded) and a weight are
// split into TERMS bf16 numbers, two (off by 2^-17) where the result is bf16, three
// (2^-24) where it is float32: the matrix cores have time to spare (8 KFLOP a row of 256
// bytes for 16 columns of two terms; busy 8% of the time).
//
// What bounds it: HBM with many long windows (64 sequences of 2000 to 8191 rows, 8 key
// heads of four queries, bf16, D = 128: 1.34 GB in 218 us, 6.1 TB/s, with the join 224;
// one wavefront after the other on rows by fused multiply-adds 414).  With few, the chain
// of one wavefront: length, page, rows (one microsecond each) and 1.3 us a tile (one user
// of 32 heads, 512 rows: 11.3 us).  Eight wavefronts of a work-group instead of four, where
// it has its CU to itself: 11.3 and 13.3 us there; 256 work-groups of 1024 rows 26.6 and
// 29.0.  Sixteen with tiles of 16 rows: 12.0 and 26.6.
#include <algorithm>

#include "bf16_rows.h"
#include "paged_step.h"

namespace pi_attn {

namespace {

constexpr int TILE = 32;   // rows, two blocks of 16
constexpr int NQ = 16;     // query columns

template <typename ST, int D>
struct Tiles {
    using R = Row<ST, D>;
    static constexpr int RB = D * (int)sizeof(ST);   // bytes of a cached row
    static constexpr int LOADS = TILE / R::RPI;      // load instructions of a tile's keys
    static constexpr int STEPS = D / 32;             // k-steps of the scores
    static constexpr int DB = D / 16;                // 16-dim output blocks
    // LDS rows, padded by 16 bytes: the reads of the scores take one 16-byte piece of 16
    // rows, the transpose reads 32 bytes of them, and both meet all banks equally.  Writes of
    // codes do not (a lane's two pieces lie 32 bytes from its neighbour's): of the LDS cycles
    // 42% are conflicts there, 20% with bf16 pages.
    static constexpr int PITCH = 2 * D + 16;
    static constexpr int BYTES = TILE * PITCH;
};

// Eight codes times a scale that is a power of two, in bf16 (exact).
__device__ inline bf16x8 codes_bf16(unsigned lo, unsigned hi, float scale) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// TERMS bf16 numbers that sum to x, but for what the last one cannot hold.
template <int TERMS>
__device__ inline void split(float x, __bf16 (&t)[TERMS]) {
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        t[i] = (__bf16)x;
        x -= (float)t[i];
    }
}

// The same of a query's element past bf16's largest number: no infinity for a finite one, and no
// second term beside an infinity or NaN (their difference is NaN, and a clamp makes an infinite
// logit finite).
constexpr float kLargestBf16 = 0x1.fep127f;

template <int TERMS>
__device__ inline void split_large(float x, __bf16 (&t)[TERMS]) {
    const bool finite = fabsf(x) < INFINITY;
    t[0] = (__bf16)(finite ? fminf(fmaxf(x, -kLargestBf16), kLargestBf16) : x);
    x = finite ? x - (float)t[0] : 0.0f;
#pragma unroll
    for (int i = 1; i < TERMS; ++i) {
        t[i] = (__bf16)x;
        x -= (float)t[i];
    }
}

// Orders a wavefront's own LDS accesses: its lanes read what others wrote.
__device__ inline void lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Largest and sum over the four lanes of a query.
__device__ inline float query_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float query_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// ONCE: the window's rows are not kept in the caches.
template <typename T, typename ST, int D, bool CLAMP, bool ONCE, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES == 4 ? 3 : 2) void decode_tiles_kernel(PagedStepParams p, int q_groups) {
    using L = Tiles<ST, D>;
    constexpr bool Q = kQuantised<ST>;
    constexpr int TERMS = sizeof(T) == 4 ? 3 : 2;
    static_assert(L::STEPS <= WAVES, "a k-step of the queries a wavefront");
    // a tile's rows for each wavefront; its accumulators at the end
    __shared__ alignas(16) unsigned char s_v[WAVES * L::BYTES];
    __shared__ float s_m[WAVES][NQ], s_l[WAVES][NQ];
    __shared__ float2 s_cs[D / 2];
    __shared__ uint4 s_new[2][L::R::LPR];         // the new row, as it is stored
    __shared__ unsigned s_new_bytes[2];           // and its scale bytes
    __shared__ bf16x8 s_q[TERMS][L::STEPS][64];   // the queries, as the scores take them

    const bool part = p.parts != 0;
    // The first range of every window, then the second: the shorter last ones come late.
    const DivMod range_of = divmod(blockIdx.x, part ? p.S * p.Hk * q_groups : gridDim.x);
    const int range = (int)range_of.quot;
    const DivMod group_of = divmod(range_of.rem, q_groups);
    const DivMod head_of = divmod(group_of.quot, p.Hk);
    const int s = (int)head_of.quot, hk = (int)head_of.rem;
    const int G = p.H / p.Hk, g0 = (int)group_of.rem * NQ, nq = min(NQ, G - g0);
    const int64_t first_head = (int64_t)s * p.H + hk * G + g0;   // of S * H
    const int tid = threadIdx.x, lane = __lane_id();
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const Pages &pages = p.pages;
    const int t = p.len_in[s];
    const int64_t reach = (int64_t)pages.page * pages.max_pages;
    const bool in_reach = t >= 0 && t < reach;
    const int lo = window_lo(max(t, 0), p.k);
    const int len = part ? range_len(p, t - lo) : t - lo;   // of a range
    if (in_reach && range > 0 && (int64_t)range * len >= t - lo) return;
    const int place = in_reach ? page_of(pages, s, pages.by_page.div(t)) : -1;   // page of the new row

    // What does not depend on the pages is asked for first: the queries (a k-step by
    // each wavefront; the other elements of their pairs too) and the gate.
    const bool rotary = p.r.freq != nullptr;
    const Angle angle = angle_of(p.r, min(tid, D / 2), s, 0, t);   // of pair tid
    // N elements of a new row in the working type.
    auto wide = [&](const T *from, auto &f) __attribute__((always_inline)) {
        constexpr int N = sizeof(f) / 4, E = 16 / (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < N / E; ++i) {
            float y[E];
            to_f32<T>(ld16(from + i * E), y);
#pragma unroll
            for (int e = 0; e < E; ++e) f[i * E + e] = y[e];
        }
    };
    // Wavefront 0 makes the new row: a lane the piece that it would load of any row.
    constexpr int EPL = L::R::EPL;
    const int sub = lane % L::R::LPR, rg = lane / L::R::LPR;
    float k_own[EPL], k_other[EPL], v_own[EPL];
    if (w == 0) {
        const int64_t at = ((int64_t)s * p.Hk + hk) * D;
        wide((const T *)p.k_new + at + sub * EPL, k_own);
        wide((const T *)p.k_new + at + (sub ^ (L::R::LPR / 2)) * EPL, k_other);
        wide((const T *)p.v_new + at + sub * EPL, v_own);
    }
    const T *const q_row = (const T *)p.q_new + (first_head + min(c, nq - 1)) * D;
    const int q_dim = 32 * min(w, L::STEPS - 1) + 8 * g;
    float q_own[8], q_other[8];
    wide(q_row + q_dim, q_own);
    wide(q_row + (q_dim ^ (D / 2)), q_other);
    const float gate = p.gate[s * p.gss + (hk * G + g0 + min(c, nq - 1)) * p.gsh];

    // This work-group's rows: the window's, first + [0, nwin), and behind those of the
    // last range the new one and the partner.
    const int first = lo + range * len;
    const int nwin = in_reach ? min(len, t - first) : 0;
    const bool last = in_reach && first + nwin == t;
    const int jp = partner_of(t, p.k, p.pi);
    const int nrows = nwin + (last ? jp >= 0 ? 2 : 1 : 0);
    const int ntiles = (nrows + TILE - 1) / TILE;

    // Rows of the pool (fewer than 2^31): lane l finds that of a tile's row l % TILE, -1
    // where none is there; its page is looked up a tile ahead.
    const int per_page = p.Hk * pages.page, kv = hk * pages.page;
    const int32_t *const table = pages.table + (int64_t)s * pages.max_pages;
    int entry = -1;
    auto position = [&](int tile) __attribute__((always_inline)) {
        const int i = min(tile * TILE + lane % TILE, nrows - 1);
        return (uint32_t)(i < nwin ? first + i : i == nwin ? t : jp);
    };
    auto look_up = [&](int tile) __attribute__((always_inline)) {
        if (tile < ntiles) entry = table[pages.by_page.div(position(tile))];   // not looked at here: no wait
    };
    auto find = [&](int tile) __attribute__((always_inline)) {
        const uint32_t at = position(tile);
        return page_named(pages, entry) >= 0 && tile * TILE + lane % TILE < nrows
                   ? entry * per_page + kv + (int)(at - pages.by_page.div(at) * pages.page)
                   : -1;
    };
    // The row that load instruction i covers in this lane.
    auto row_of = [&](int row, int i) __attribute__((always_inline)) {
        return __builtin_amdgcn_ds_bpermute(4 * (i * L::R::RPI + rg), row);
    };
    // Rows that are not there read row 0 of the pool.
    auto load = [&](const void *rows, int row, uint4 (&r)[L::LOADS]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < L::LOADS; ++i) {
            const uint8_t *const from = (const uint8_t *)rows + (int64_t)max(row_of(row, i), 0) * L::RB + 16 * sub;
            r[i] = ONCE ? ld16_once(from) : ld16(from);
        }
    };
    // Scale bytes: of the keys in the first TILE lanes, of the values in the next (of rows
    // that are not there whatever, and not looked at here: no wait).
    auto load_bytes = [&](int row) __attribute__((always_inline)) -> int {
        if constexpr (!Q) return 0;
        return (lane < TILE ? pages.k_exp : pages.v_exp)[max(row, 0)];
    };
    look_up(w);
    if (place < 0) {
        if (part) return;
        for (int i = tid; i < nq * D; i += 64 * WAVES) ((T *)p.out)[first_head * D + i] = (T)NAN;
        if (p.lse && tid < nq) p.lse[first_head + tid] = NAN;
        if (p.len_out && hk == 0 && g0 == 0 && tid == 0) p.len_out[s] = t;
        return;
    }
    uint4 kr[L::LOADS], vr[L::LOADS];
    int row = -1, bytes = 127;
    if (w < ntiles) {
        row = find(w);
        look_up(w + WAVES);
        bytes = load_bytes(row);
        load(pages.k, row, kr);
        load(pages.v, row, vr);
    }

    if (rotary && tid < D / 2) s_cs[tid] = cos_sin(angle.pos, angle.freq);
    // Elements from `dim` on turned, `o` the other elements of their pairs.
    auto turned = [&](auto &f, const auto &o, int dim) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < (int)sizeof(f) / 4; ++e) {
            const int pair = (dim & (D / 2 - 1)) + e;
            const float2 cs = s_cs[pair];
            const float x = f[e] * cs.x, y = o[e] * cs.y;
            if (pair < p.r.pairs) f[e] = dim < D / 2 ? x - y : x + y;
        }
    };
    if (rotary) __syncthreads();
    if (w == 0 && last) {
        if (rotary) turned(k_own, k_other, sub * EPL);
        // as stored: in the pages' type
        auto stored = [&](const float (&f)[EPL], uint4 &u) __attribute__((always_inline)) {
            if constexpr (Q) {
                unsigned a = 0;
#pragma unroll
                for (int e = 0; e < EPL; ++e) a = max(a, finite_bits(f[e]));
                const unsigned byte = e4m3_byte(row_max<L::R::LPR>(a));
                const float inv = e4m3_inverse(byte);
                u = make_uint4(e4m3_pack4(f, inv), e4m3_pack4(f + 4, inv), e4m3_pack4(f + 8, inv), e4m3_pack4(f + 12, inv));
                return byte;
            } else {
                bf16x8 y;
#pragma unroll
                for (int e = 0; e < EPL; ++e) y[e] = (__bf16)f[e];
                u = __builtin_bit_cast(uint4, y);
                return 127u;
            }
        };
        uint4 kx, vx;
        const unsigned kb = stored(k_own, kx), vb = stored(v_own, vx);
        if (rg == 0) {
            s_new[0][sub] = kx;
            s_new[1][sub] = vx;
            if (sub == 0) {
                s_new_bytes[0] = kb;
                s_new_bytes[1] = vb;
            }
            if (g0 == 0) {   // of row t nothing is used that is read here
                const int64_t mine = place * per_page + kv + (int)(t - pages.by_page.div(t) * pages.page);
                *reinterpret_cast<uint4 *>((uint8_t *)pages.k + mine * L::RB + 16 * sub) = kx;
                *reinterpret_cast<uint4 *>((uint8_t *)pages.v + mine * L::RB + 16 * sub) = vx;
                if (Q && sub == 0) {
                    pages.k_exp[mine] = (uint8_t)kb;
                    pages.v_exp[mine] = (uint8_t)vb;
                }
            }
        }
    }
    if (w < L::STEPS) {
        if (rotary) turned(q_own, q_other, q_dim);
        bf16x8 q[TERMS];
        auto split_row = [&](auto &&one) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                __bf16 terms[TERMS];
                one(c < nq ? q_own[e] : 0.0f, terms);
#pragma unroll
                for (int i = 0; i < TERMS; ++i) q[i][e] = terms[i];
            }
        };
        float most = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(q_own[e]));
        if (__builtin_amdgcn_ballot_w64(most > kLargestBf16)) {
            split_row([](float x, __bf16 (&t)[TERMS]) { split_large<TERMS>(x, t); });
        } else {
            split_row([](float x, __bf16 (&t)[TERMS]) { split<TERMS>(x, t); });
        }
#pragma unroll
        for (int i = 0; i < TERMS; ++i) s_q[i][w][lane] = q[i];
    }
    __syncthreads();
    const FusionBias fb = fusion_bias(gate, CLAMP);
    const float c2 = p.scale * kLog2e;

    f32x4 o[L::DB];
#pragma unroll
    for (int db = 0; db < L::DB; ++db) o[db] = f32x4{};
    float m = -INFINITY, l = 0.0f;   // of query c; l: this lane's rows

    unsigned char *const lds = s_v + w * L::BYTES;
    // A lane's 8 (bf16) or 16 (codes) elements of row r of the tile into LDS.
    auto put = [&](uint4 u, int r, float scale) __attribute__((always_inline)) {
        unsigned char *const to = lds + r * L::PITCH + 2 * L::R::EPL * sub;
        if constexpr (Q) {
            *reinterpret_cast<bf16x8 *>(to) = codes_bf16(u.x, u.y, scale);
            *reinterpret_cast<bf16x8 *>(to + 16) = codes_bf16(u.z, u.w, scale);
        } else {
            *reinterpret_cast<uint4 *>(to) = u;
        }
    };
    for (int tile = w; tile < ntiles; tile += WAVES) {
        const bool more = tile + WAVES < ntiles;
        int next = -1, next_bytes = 127;
        if (more) {
            next = find(tile + WAVES);
            look_up(tile + 2 * WAVES);
            next_bytes = load_bytes(next);
        }
        const uint32_t there = (uint32_t)__builtin_amdgcn_ballot_w64(row >= 0);   // bit r: row r
        const bool whole = there == ~0u;
        const int new_r = nwin - tile * TILE;   // the new row's, where last
        const bool special = last && new_r < TILE && new_r >= -1;   // it or the partner is in the tile
        auto scale_of = [&](int i, int table) __attribute__((always_inline)) {
            return Q ? e4m3_scale(__builtin_amdgcn_ds_bpermute(4 * (i * L::R::RPI + rg + TILE * table), bytes)) : 1.0f;
        };
        lds_order();   // the tile before has been read
#pragma unroll
        for (int i = 0; i < L::LOADS; ++i) put(kr[i], i * L::R::RPI + rg, scale_of(i, 0));
        if (special && new_r >= 0) {
            lds_order();   // over what its place held, by other lanes
            if (rg == 0) put(s_new[0][sub], new_r, e4m3_scale(s_new_bytes[0]));
        }
        if (more) load(pages.k, next, kr);
        lds_order();
        f32x4 sc[2] = {f32x4{}, f32x4{}};
#pragma unroll
        for (int x = 0; x < L::STEPS; ++x) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const bf16x8 a = *reinterpret_cast<const bf16x8 *>(lds + (16 * b + c) * L::PITCH + 64 * x + 16 * g);
#pragma unroll
                for (int i = TERMS - 1; i >= 0; --i)
                    sc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, s_q[i][x][lane], sc[b], 0, 0, 0);
            }
        }
        // A lane's scores are of rows 4g + i and 16 + 4g + i.
        float d[8];   // logits, log2 units
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = CLAMP ? sc[i >> 2][i & 3] : sc[i >> 2][i & 3] * c2;
        if (CLAMP || special) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool partner = special && 16 * (i >> 2) + 4 * g + (i & 3) == new_r + 1;
                d[i] = CLAMP ? clamped_logit(d[i] * p.scale + (partner ? fb.partner : fb.local), p.clamp) * kLog2e
                             : d[i] + (partner ? fb.partner * kLog2e : 0.0f);
            }
        }
        if (!whole) {
            const uint32_t mine = there >> 4 * g;
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = mine >> (16 * (i >> 2) + (i & 3)) & 1 ? d[i] : -INFINITY;
        }
        float top = d[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, d[i]);
        if (__builtin_amdgcn_ballot_w64(top > m + kTau)) {
            top = query_max(top);
            const float m_new = top > m + kTau ? top : m;
            const float a = m_new == m ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= a;
#pragma unroll
            for (int db = 0; db < L::DB; ++db) o[db] *= a;
        }
        const float mu = m == -INFINITY ? 0.0f : m;
        bf16x8 pb[TERMS];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float pr = weight(d[i], mu);
            l += pr;
            __bf16 terms[TERMS];
            split<TERMS>(pr, terms);
#pragma unroll
            for (int x = 0; x < TERMS; ++x) pb[x][i] = terms[x];
        }
        lds_order();   // the keys have been read
#pragma unroll
        for (int i = 0; i < L::LOADS; ++i) put(vr[i], i * L::R::RPI + rg, scale_of(i, 1));
        if (!whole) {   // rows that are not there may hold anything
            lds_order();   // over what other lanes wrote
            if (row < 0) {
                constexpr int LANES = 64 / TILE;   // of a row
                unsigned char *const to = lds + lane % TILE * L::PITCH + lane / TILE * (2 * D / LANES);
#pragma unroll
                for (int i = 0; i < 2 * D / LANES; i += 16) *reinterpret_cast<uint4 *>(to + i) = make_uint4(0, 0, 0, 0);
            }
        }
        if (special && new_r >= 0) {
            lds_order();
            if (rg == 0) put(s_new[1][sub], new_r, e4m3_scale(s_new_bytes[1]));
        }
        if (more) load(pages.v, next, vr);
        lds_order();
        const int vrow = 4 * g + ((lane >> 2) & 3), qd = lane & 3;
#pragma unroll
        for (int db = 0; db < L::DB; ++db) {
            bf16x8 a;
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const unsigned char *src = lds + (vrow + 16 * hh) * L::PITCH + 32 * db + 8 * qd;
                const bf16x4 y = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)src));
#pragma unroll
                for (int j = 0; j < 4; ++j) a[4 * hh + j] = y[j];
            }
#pragma unroll
            for (int x = TERMS - 1; x >= 0; --x) o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb[x], o[db], 0, 0, 0);
        }
        row = next;
        bytes = next_bytes;
    }

    // Join the wavefronts.
    l = query_sum(l);
    if (lane < NQ) {
        s_m[w][c] = m;
        s_l[w][c] = l;
    }
    __syncthreads();   // the tiles are done with
    float *const s_o = reinterpret_cast<float *>(s_v);   // [WAVES][nq][D]
    static_assert(NQ * D * 4 <= L::BYTES, "a wavefront's accumulators fit its tile");
    if (c < nq) {
#pragma unroll
        for (int db = 0; db < L::DB; ++db)
            *reinterpret_cast<f32x4 *>(s_o + ((int64_t)w * nq + c) * D + 16 * db + 4 * g) = o[db];
    }
    __syncthreads();
    for (int i = tid; i < nq * D; i += 64 * WAVES) {
        const int j = i / D, e = i % D;
        float M = -INFINITY;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) M = fmaxf(M, s_m[x][j]);
        float sum = 0.0f, out = 0.0f;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) {
            const float f = s_m[x][j] == M ? 1.0f : __builtin_amdgcn_exp2f(s_m[x][j] - M);
            sum += s_l[x][j] * f;
            out += s_o[(x * nq + j) * D + e] * f;
        }
        if (part) {
            const int64_t at = (int64_t)range * p.S * p.H + first_head + j;
            p.part_o[at * D + e] = out;
            if (e == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(M, sum);
        } else {
            ((T *)p.out)[first_head * D + i] = (T)(out / sum);
            if (e == 0 && p.lse) {
                const FusionBias b = fusion_bias(p.gate[s * p.gss + (hk * G + g0 + j) * p.gsh], CLAMP);
                p.lse[first_head + j] = (M + __log2f(sum)) * kLn2 + b.lse_shift;
            }
        }
    }
    if (!part && p.len_out && hk == 0 && g0 == 0 && tid == 0) p.len_out[s] = t + 1;
}

// Eight wavefronts where the work-groups have a CU each, four otherwise, which lets
// three of them share one (registers and LDS).
template <typename T, typename ST, int D, bool CLAMP, bool ONCE>
hipError_t launch_w(const PagedStepParams &p, int64_t groups, int q_groups, hipStream_t stream) {
    if (p.parts == 0 && groups <= 256)
        return launch_kernel(decode_tiles_kernel<T, ST, D, CLAMP, ONCE, 8>, dim3((unsigned)groups), dim3(512), stream, p, q_groups);
    return launch_kernel(decode_tiles_kernel<T, ST, D, CLAMP, ONCE, 4>, dim3((unsigned)(groups * std::max(p.parts, 1))),
                         dim3(256), stream, p, q_groups);
}

template <typename T, typename ST, int D, bool CLAMP>
hipError_t launch_d(const PagedStepParams &p, hipStream_t stream) {
    const int q_groups = (p.H / p.Hk + NQ - 1) / NQ;
    const int64_t groups = (int64_t)p.S * p.Hk * q_groups;
    return read_once(p, q_groups, sizeof(ST)) ? launch_w<T, ST, D, CLAMP, true>(p, groups, q_groups, stream)
                                              : launch_w<T, ST, D, CLAMP, false>(p, groups, q_groups, stream);
}

template <typename T, typename ST>
hipError_t launch_t(const PagedStepParams &p, hipStream_t stream) {
    const bool clamp = p.clamp > 0.0f;
    if (p.D == 64) return clamp ? launch_d<T, ST, 64, true>(p, stream) : launch_d<T, ST, 64, false>(p, stream);
    return clamp ? launch_d<T, ST, 128, true>(p, stream) : launch_d<T, ST, 128, false>(p, stream);
}

}  // namespace

hipError_t launch_decode_paged_tiles(const PagedStepParams &p, bool bf16, hipStream_t stream) {
    if (!p.pages.k_exp) return launch_t<__bf16, __bf16>(p, stream);
    return bf16 ? launch_t<__bf16, e4m3>(p, stream) : launch_t<float, e4m3>(p, stream);
}

}  // namespace pi_attn
