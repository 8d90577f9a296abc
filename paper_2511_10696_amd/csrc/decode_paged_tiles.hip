// decode_paged_tiles.hip -- the decode step over a paged cache on the matrix
// cores: pages in bf16 or e4m3, up to 16 query heads of a key head at a time.
//
// A work-group is a sequence, a key head, up to 16 of its query heads and a range
// of the window; its wavefronts take tiles of 32 rows in turn, each with a running
// maximum, sum and accumulator for every query, joined at the end.
//
// MFMA layout (v_mfma_f32_16x16x32_bf16; lane = (c, g) = (l % 16, l / 16)).  Scores
// S^T = K Q^T, 16 rows at a time: A = K, lane (c, g) holding of row c the elements
// that it loads from memory as they lie, 16 bytes of every 64; B = Q^T with the same
// elements; C holds rows 4g + i of query c.  Output O^T += V^T P^T over 32 rows: B =
// P^T is the weights of two blocks where they are (rows 4g + i and 16 + 4g + i), A =
// V^T comes from LDS by transpose reads of the same rows.  Only the values pass
// through LDS, a wavefront's own part of it: no wavefront waits for another before
// the end.
//
// Precision.  The products take bf16: cached rows are that, or e4m3, whose codes and
// scales together are bf16 numbers.  A query (turned, not rounded) and a weight are
// split into TERMS bf16 numbers, two (off by 2^-17) where the result is bf16, three
// (2^-24) where it is float32: the matrix cores have time to spare, a row of 256
// bytes costs 32 query columns 16 KFLOP.
#include <algorithm>

#include "bf16_rows.h"
#include "paged_step.h"

namespace pi_attn {

namespace {

constexpr int WAVES = 8;
constexpr int TILE = 32;   // rows
constexpr int NQ = 16;     // query columns

template <typename ST, int D>
struct Tiles {
    static constexpr int RB = D * (int)sizeof(ST);   // bytes of a cached row
    static constexpr int NP = RB / 64;               // 16-byte pieces of a lane's row
    static constexpr int STEPS = D / 32;             // k-steps of the scores
    static constexpr int DB = D / 16;                // 16-dim output blocks
    // LDS rows, padded by 32 bytes: a transpose read takes 32 bytes of 16 rows, 8 of
    // which then cover all banks
    static constexpr int PITCH = 2 * D + 32;
    static constexpr int BYTES = TILE * PITCH;
    // first element of a lane's part in k-step `step`
    static __device__ int dim(int step, int g) {
        return kQuantised<ST> ? 64 * (step >> 1) + 16 * g + 8 * (step & 1) : 32 * step + 8 * g;
    }
};

// The bf16 numbers of eight codes times a scale that is a power of two.
__device__ inline bf16x8 codes_bf16(unsigned lo, unsigned hi, float scale) {
    float f[8];
    e4m3_unpack4(lo, f);
    e4m3_unpack4(hi, f + 4);
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)(f[i] * scale);
    return r;
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

template <typename T, typename ST, int D, bool PART>
__global__ __launch_bounds__(64 * WAVES) void decode_tiles_kernel(PagedStepParams p, int q_groups) {
    using L = Tiles<ST, D>;
    constexpr bool Q = kQuantised<ST>;
    constexpr int TERMS = sizeof(T) == 4 ? 3 : 2;
    __shared__ alignas(16) unsigned char s_v[WAVES][L::BYTES];
    __shared__ float s_m[WAVES][NQ], s_l[WAVES][NQ];
    __shared__ float2 s_cs[WAVES][D / 2];

    const DivMod range_of = divmod(blockIdx.x, PART ? p.parts : 1);
    const int range = (int)range_of.rem;
    const DivMod group_of = divmod(range_of.quot, q_groups);
    const DivMod head_of = divmod(group_of.quot, p.Hk);
    const int s = (int)head_of.quot, hk = (int)head_of.rem;
    const int G = p.H / p.Hk, g0 = (int)group_of.rem * NQ, nq = min(NQ, G - g0);
    const int64_t first_head = (int64_t)s * p.H + hk * G + g0;   // of S * H
    const int tid = threadIdx.x, lane = __lane_id();
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const Pages &pages = p.pages;
    const int t = p.len_in[s];

    if (!has_place(pages, s, t)) {
        if (PART) return;
        for (int i = tid; i < nq * D; i += 64 * WAVES) ((T *)p.out)[first_head * D + i] = (T)NAN;
        if (p.lse && tid < nq) p.lse[first_head + tid] = NAN;
        if (p.len_out && hk == 0 && g0 == 0 && tid == 0) p.len_out[s] = t;
        return;
    }
    const int lo = window_lo(t, p.k);
    if (PART && range >= ranges_of(t - lo, p.range)) return;
    // this work-group's window rows: first + [0, nwin)
    const int first = PART ? lo + range * p.range : lo;
    const int nwin = PART ? min(p.range, t - first) : t - lo;
    const int ntiles = (nwin + TILE - 1) / TILE;

    const int64_t kv = (int64_t)hk * pages.page;                  // row 0 of this head in page 0
    const int64_t per_page = (int64_t)p.Hk * pages.page;
    const uint8_t *kc = (const uint8_t *)pages.k + 16 * g, *vc = (const uint8_t *)pages.v + 16 * g;
    // A lane's row of each block: page (looked up ahead), place, then its pieces.
    int entry[2];
    bool there[2];
    uint4 kr[2][L::NP], vr[2][L::NP];
    unsigned kb[2], vb[2];
    auto look_up = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const uint32_t at = (uint32_t)(first + min(tile * TILE + 16 * b + c, nwin - 1));
            entry[b] = page_of(pages, s, pages.by_page.div(at));
        }
    };
    auto load = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int i = tile * TILE + 16 * b + c;
            const uint32_t at = (uint32_t)(first + min(i, nwin - 1));
            there[b] = entry[b] >= 0 && i < nwin;
            const int64_t row = max(entry[b], 0) * per_page + kv + (at - pages.by_page.div(at) * pages.page);
#pragma unroll
            for (int x = 0; x < L::NP; ++x) {
                kr[b][x] = ld16(kc + row * L::RB + 64 * x);
                vr[b][x] = ld16(vc + row * L::RB + 64 * x);
            }
            if constexpr (Q) {
                kb[b] = pages.k_exp[row];
                vb[b] = pages.v_exp[row];
            }
        }
    };
    if (w < ntiles) {
        look_up(w);
        load(w);
        if (w + WAVES < ntiles) look_up(w + WAVES);
    }

    // Cosines and sines: one pair a lane, by every wavefront for itself.
    const bool rotary = p.r.freq != nullptr;
    if (rotary) {
        if (lane < D / 2) s_cs[w][lane] = cos_sin_of(p.r, lane, s, 0, t);
        lds_order();
    }
    // Eight elements of a new row from `dim` on, turned (the other elements of their
    // pairs are read too).
    auto load_new = [&](const T *row, int dim, bool turns, float (&f)[8]) __attribute__((always_inline)) {
        constexpr int N = 16 / (int)sizeof(T);
        auto eight = [&](int at, float (&x)[8]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8 / N; ++i) {
                float y[N];
                to_f32<T>(ld16(row + at + i * N), y);
#pragma unroll
                for (int e = 0; e < N; ++e) x[i * N + e] = y[e];
            }
        };
        eight(dim, f);
        if (!turns) return;
        float o[8];
        eight(dim ^ (D / 2), o);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int pair = (dim & (D / 2 - 1)) + e;
            const float2 cs = s_cs[w][pair];
            const float x = f[e] * cs.x, y = o[e] * cs.y;
            if (pair < p.r.pairs) f[e] = dim < D / 2 ? x - y : x + y;
        }
    };
    bf16x8 qf[TERMS][L::STEPS];
#pragma unroll
    for (int x = 0; x < L::STEPS; ++x) {
        float f[8];
        load_new((const T *)p.q_new + (first_head + min(c, nq - 1)) * D, L::dim(x, g), rotary, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            __bf16 terms[TERMS];
            split<TERMS>(c < nq ? f[e] : 0.0f, terms);
#pragma unroll
            for (int i = 0; i < TERMS; ++i) qf[i][x][e] = terms[i];
        }
    }
    const bool clamped = p.clamp > 0.0f;
    const FusionBias fb = fusion_bias(p.gate[s * p.gss + (hk * G + g0 + min(c, nq - 1)) * p.gsh], clamped);
    const float c2 = p.scale * kLog2e;

    f32x4 o[L::DB];
#pragma unroll
    for (int db = 0; db < L::DB; ++db) o[db] = f32x4{};
    float m = -INFINITY, l = 0.0f;   // of query c; l: this lane's rows

    unsigned char *const tile_v = s_v[w];
    // The tile in kr, vr: rows 4g + i and 16 + 4g + i are in use where bit i and 4 + i of
    // `mask` are set; row 1 of the extra tile is the partner.  `next` runs once the
    // registers are free.
    auto attend = [&](bool extra, auto next) __attribute__((always_inline)) {
        // scores
        f32x4 sc[2] = {f32x4{}, f32x4{}};
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (extra && b == 1) break;
            const float ks = Q ? e4m3_scale(kb[b]) : 1.0f;
#pragma unroll
            for (int x = 0; x < L::STEPS; ++x) {
                bf16x8 a;
                if constexpr (Q) {
                    const uint4 u = kr[b][x >> 1];
                    a = x & 1 ? codes_bf16(u.z, u.w, ks) : codes_bf16(u.x, u.y, ks);
                } else {
                    a = __builtin_bit_cast(bf16x8, kr[b][x]);
                }
#pragma unroll
                for (int i = TERMS - 1; i >= 0; --i)
                    sc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[i][x], sc[b], 0, 0, 0);
            }
        }
        // values, zero where no row is there
        uint64_t rows[2];
        lds_order();   // the tile before has been read
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            rows[b] = __builtin_amdgcn_ballot_w64(there[b]);
            unsigned char *to = tile_v + (16 * b + c) * L::PITCH;
            const float vs = Q && there[b] ? e4m3_scale(vb[b]) : 1.0f;
#pragma unroll
            for (int x = 0; x < L::NP; ++x) {
                const uint4 u = there[b] ? vr[b][x] : make_uint4(0, 0, 0, 0);
                if constexpr (Q) {
                    *reinterpret_cast<bf16x8 *>(to + 128 * x + 32 * g) = codes_bf16(u.x, u.y, vs);
                    *reinterpret_cast<bf16x8 *>(to + 128 * x + 32 * g + 16) = codes_bf16(u.z, u.w, vs);
                } else {
                    *reinterpret_cast<uint4 *>(to + 64 * x + 16 * g) = u;
                }
            }
        }
        next();
        float d[8], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int b = i >> 2, row = 4 * g + (i & 3);
            float x = sc[b][i & 3];
            const bool partner = extra && row == 1;
            x = clamped ? clamped_logit(x * p.scale + (partner ? fb.partner : fb.local), p.clamp) * kLog2e
                        : x * c2 + (partner ? fb.partner * kLog2e : 0.0f);
            d[i] = rows[b] >> row & 1 ? x : -INFINITY;
            top = fmaxf(top, d[i]);
        }
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
            const float pr = __builtin_amdgcn_exp2f(d[i] - mu);
            l += pr;
            __bf16 terms[TERMS];
            split<TERMS>(pr, terms);
#pragma unroll
            for (int x = 0; x < TERMS; ++x) pb[x][i] = terms[x];
        }
        lds_order();
        const int r = (lane >> 2) & 3, qd = lane & 3;
#pragma unroll
        for (int db = 0; db < L::DB; ++db) {
            bf16x8 a;
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const unsigned char *src = tile_v + (4 * g + r + 16 * hh) * L::PITCH + 32 * db + 8 * qd;
                const bf16x4 y = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)src));
#pragma unroll
                for (int j = 0; j < 4; ++j) a[4 * hh + j] = y[j];
            }
#pragma unroll
            for (int x = TERMS - 1; x >= 0; --x) o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb[x], o[db], 0, 0, 0);
        }
    };

    for (int tile = w; tile < ntiles; tile += WAVES) {
        attend(false, [&]() __attribute__((always_inline)) {
            if (tile + WAVES < ntiles) {
                load(tile + WAVES);
                if (tile + 2 * WAVES < ntiles) look_up(tile + 2 * WAVES);
            }
        });
    }

    // The new row (row 0 of a tile) and the partner (row 1), by the wavefront whose
    // turn comes after the last tile.
    if (range == 0 && w == ntiles % WAVES) {
        const int jp = partner_of(t, p.k, p.pi);
        const int pe = jp >= 0 ? page_of(pages, s, pages.by_page.div(jp)) : -1;
        there[0] = c == 0 || (c == 1 && pe >= 0);
        there[1] = false;
        kb[0] = vb[0] = kb[1] = vb[1] = 127;
#pragma unroll
        for (int x = 0; x < L::NP; ++x) kr[0][x] = vr[0][x] = vr[1][x] = make_uint4(0, 0, 0, 0);
        if (c == 1 && pe >= 0) {
            const int64_t row = pe * per_page + kv + (jp - pages.by_page.div(jp) * pages.page);
#pragma unroll
            for (int x = 0; x < L::NP; ++x) {
                kr[0][x] = ld16(kc + row * L::RB + 64 * x);
                vr[0][x] = ld16(vc + row * L::RB + 64 * x);
            }
            if constexpr (Q) {
                kb[0] = pages.k_exp[row];
                vb[0] = pages.v_exp[row];
            }
        }
        const int64_t at = ((int64_t)s * p.Hk + hk) * D;
        // as stored
        auto stored = [&](const T *row, bool turns, uint4 (&r)[L::NP], unsigned &byte) __attribute__((always_inline)) {
            float f[L::STEPS][8];
#pragma unroll
            for (int x = 0; x < L::STEPS; ++x) load_new(row, L::dim(x, g), turns, f[x]);
            if constexpr (Q) {
                unsigned a = 0;
#pragma unroll
                for (int x = 0; x < L::STEPS; ++x)
#pragma unroll
                    for (int e = 0; e < 8; ++e) a = max(a, finite_bits(f[x][e]));
                a = max(a, (unsigned)__shfl_xor((int)a, 16));
                a = max(a, (unsigned)__shfl_xor((int)a, 32));
                const unsigned by = e4m3_byte(a);
                const float inv = e4m3_inverse(by);
                if (c == 0) {
                    byte = by;
#pragma unroll
                    for (int x = 0; x < L::NP; ++x)
                        r[x] = make_uint4(e4m3_pack4(f[2 * x], inv), e4m3_pack4(f[2 * x] + 4, inv),
                                          e4m3_pack4(f[2 * x + 1], inv), e4m3_pack4(f[2 * x + 1] + 4, inv));
                }
            } else {
                if (c != 0) return;
#pragma unroll
                for (int x = 0; x < L::NP; ++x) {
                    if (turns) {
                        bf16x8 y;
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = (__bf16)f[x][e];
                        r[x] = __builtin_bit_cast(uint4, y);
                    } else {
                        r[x] = ld16(row + L::dim(x, g));
                    }
                }
            }
        };
        stored((const T *)p.k_new + at, rotary, kr[0], kb[0]);
        stored((const T *)p.v_new + at, false, vr[0], vb[0]);
        if (c == 0 && g0 == 0) {   // no row read here is row t
            const uint32_t slot = pages.by_page.div(t);
            const int64_t row = page_of(pages, s, slot) * per_page + kv + (t - slot * pages.page);
#pragma unroll
            for (int x = 0; x < L::NP; ++x) {
                *reinterpret_cast<uint4 *>((uint8_t *)pages.k + 16 * g + row * L::RB + 64 * x) = kr[0][x];
                *reinterpret_cast<uint4 *>((uint8_t *)pages.v + 16 * g + row * L::RB + 64 * x) = vr[0][x];
            }
            if (Q && g == 0) {
                pages.k_exp[row] = (uint8_t)kb[0];
                pages.v_exp[row] = (uint8_t)vb[0];
            }
        }
        attend(true, []() {});
    }

    // Join the wavefronts.
    l = query_sum(l);
    if (lane < NQ) {
        s_m[w][c] = m;
        s_l[w][c] = l;
    }
    __syncthreads();   // the tiles are done with
    float *const s_o = reinterpret_cast<float *>(s_v[0]);   // [WAVES][nq][D]
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
        if (PART) {
            const int64_t at = (int64_t)range * p.S * p.H + first_head + j;
            p.part_o[at * D + e] = out;
            if (e == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(M, sum);
        } else {
            ((T *)p.out)[first_head * D + i] = (T)(out / sum);
            if (e == 0 && p.lse) {
                const FusionBias b = fusion_bias(p.gate[s * p.gss + (hk * G + g0 + j) * p.gsh], clamped);
                p.lse[first_head + j] = (M + __log2f(sum)) * kLn2 + b.lse_shift;
            }
        }
    }
    if (!PART && p.len_out && hk == 0 && g0 == 0 && tid == 0) p.len_out[s] = t + 1;
}

template <typename T, typename ST, int D>
hipError_t launch_d(const PagedStepParams &p, hipStream_t stream) {
    const int q_groups = (p.H / p.Hk + NQ - 1) / NQ;
    const int64_t groups = (int64_t)p.S * p.Hk * q_groups;
    if (p.parts)
        return launch_kernel(decode_tiles_kernel<T, ST, D, true>, dim3((unsigned)(groups * p.parts)), dim3(64 * WAVES), stream, p,
                             q_groups);
    return launch_kernel(decode_tiles_kernel<T, ST, D, false>, dim3((unsigned)groups), dim3(64 * WAVES), stream, p, q_groups);
}

template <typename T, typename ST>
hipError_t launch_t(const PagedStepParams &p, hipStream_t stream) {
    return p.D == 64 ? launch_d<T, ST, 64>(p, stream) : launch_d<T, ST, 128>(p, stream);
}

}  // namespace

hipError_t launch_decode_paged_tiles(const PagedStepParams &p, bool bf16, hipStream_t stream) {
    if (!p.pages.k_exp) return launch_t<__bf16, __bf16>(p, stream);
    return bf16 ? launch_t<__bf16, e4m3>(p, stream) : launch_t<float, e4m3>(p, stream);
}

}  // namespace pi_attn
