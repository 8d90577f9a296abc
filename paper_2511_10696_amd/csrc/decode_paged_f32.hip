// decode_paged_f32.hip -- the decode step over a paged cache in float32, fp32
// arithmetic, D = 64 or 128.
//
// One work-group per sequence, key head, up to QN of its query heads and range of the
// window.  A row is covered by lanes with 16-byte loads, CH load instructions of keys
// and of values a chunk; the next chunk's are under way while one is worked on.  Every
// row read serves QN queries.  Each group of lanes that covers a row keeps a softmax of
// its own (nothing is exchanged from row to row); they are merged at the end.
//
// What bounds it: HBM where a key head has one query (64 sequences of 16 heads, 250 to 400
// rows, D = 128: 314 MB in 52 us, 6.0 TB/s); the multiply-adds and the sums across lanes
// where it has more (16 sequences of 1000 to 1990 rows, 8 key heads of four: 197 MB in 48
// us, 4.1 TB/s).  Rows a chunk ahead: 34 -> 22 us (16 sequences of 16 heads, 800 to 990
// rows, D = 64).
#include <algorithm>

#include "paged_step.h"

namespace pi_attn {

namespace {

constexpr int CH = 4;

__device__ inline void load4(const float *from, float (&f)[4]) { to_f32<float>(ld16(from), f); }

// Sum over the LPR lanes of a row, left in each of them.
template <int LPR>
__device__ inline float row_total(float x) {
    x = row_sum<16>(x);
    if constexpr (LPR == 32) {   // rows of 16 lanes 0 and 1, 2 and 3
        const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
    return x;
}

template <int D, int QN, bool CLAMP, bool ONCE, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void decode_paged_f32_kernel(PagedStepParams p, int q_groups) {
    using R = Row<float, D>;
    constexpr int LPR = R::LPR, RPI = R::RPI;
    constexpr int RPC = RPI * CH;   // rows per chunk

    __shared__ float s_m[WAVES][QN], s_l[WAVES][QN];
    __shared__ float s_acc[WAVES][QN][D];
    __shared__ float2 s_cs[D / 2];

    const bool part = p.parts != 0;
    // The first range of every window, then the second: the shorter last ones come late.
    const DivMod range_of = divmod(blockIdx.x, part ? p.S * p.Hk * q_groups : gridDim.x);
    const int range = (int)range_of.quot;
    const DivMod group_of = divmod(range_of.rem, q_groups);
    const DivMod head_of = divmod(group_of.quot, p.Hk);
    const int s = (int)head_of.quot, hk = (int)head_of.rem;
    const int G = p.H / p.Hk, g0 = (int)group_of.rem * QN, nq = min(QN, G - g0);
    const int64_t first_head = (int64_t)s * p.H + hk * G + g0;   // of S * H
    const int tid = threadIdx.x, lane = __lane_id();
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int sub = lane % LPR, rg = lane / LPR;
    const Pages &pages = p.pages;
    const int t = p.len_in[s];
    const bool in_reach = t >= 0 && t < (int64_t)pages.page * pages.max_pages;
    const int lo = window_lo(max(t, 0), p.k);
    const int len = part ? range_len(p, t - lo) : t - lo;   // of a range
    if (in_reach && range > 0 && (int64_t)range * len >= t - lo) return;
    const int place = in_reach ? page_of(pages, s, pages.by_page.div(t)) : -1;   // page of the new row

    // This work-group's window rows: first + [0, nwin); the new row and the partner go
    // with the first range.
    const int first = lo + range * len;
    const int nwin = in_reach ? min(len, t - first) : 0;
    const int nchunks = (nwin + RPC - 1) / RPC;

    // Rows of the pool (fewer than 2^31); the pages are looked up a chunk ahead.
    const int per_page = p.Hk * pages.page, kv = hk * pages.page;
    const int32_t *const table = pages.table + (int64_t)s * pages.max_pages;
    const float *const kc = (const float *)pages.k + 4 * sub, *const vc = (const float *)pages.v + 4 * sub;
    auto position = [&](int ch, int c) __attribute__((always_inline)) {
        return (uint32_t)(first + min(ch * RPC + c * RPI + rg, nwin - 1));
    };
    int entry[CH];
    auto look_up = [&](int ch) __attribute__((always_inline)) {
        if (ch >= nchunks) return;
#pragma unroll
        for (int c = 0; c < CH; ++c) entry[c] = table[pages.by_page.div(position(ch, c))];   // not looked at here: no wait
    };
    struct Rows {
        uint4 k[CH], v[CH];
        bool there[CH];
    };
    auto load = [&](int ch, Rows &r) __attribute__((always_inline)) {
        if (ch >= nchunks) return;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = position(ch, c);
            const int e = page_named(pages, entry[c]);
            r.there[c] = e >= 0 && ch * RPC + c * RPI + rg < nwin;
            const int64_t row = (int64_t)(max(e, 0) * per_page + kv + (int)(at - pages.by_page.div(at) * pages.page)) * D;
            r.k[c] = ONCE ? ld16_once(kc + row) : ld16(kc + row);
            r.v[c] = ONCE ? ld16_once(vc + row) : ld16(vc + row);
        }
    };
    // What does not depend on the pages is asked for first.
    const float *const kn = (const float *)p.k_new + ((int64_t)s * p.Hk + hk) * D;
    const float *const vn = (const float *)p.v_new + ((int64_t)s * p.Hk + hk) * D;
    const bool rotary = p.r.freq != nullptr;
    const Angle angle = angle_of(p.r, min(tid, D / 2), s, 0, t);   // of pair tid
    float q[QN][4], gate[QN];
#pragma unroll
    for (int j = 0; j < QN; ++j) {
        const int jj = min(j, nq - 1);
        load4((const float *)p.q_new + (first_head + jj) * D + 4 * sub, q[j]);
        gate[j] = p.gate[s * p.gss + (hk * G + g0 + jj) * p.gsh];
    }
    look_up(w);
    if (place < 0) {
        if (part) return;
        for (int i = tid; i < nq * D; i += 64 * WAVES) ((float *)p.out)[first_head * D + i] = NAN;
        if (p.lse && tid < nq) p.lse[first_head + tid] = NAN;
        if (p.len_out && hk == 0 && g0 == 0 && tid == 0) p.len_out[s] = t;
        return;
    }
    // The new row (row group 0) and the partner (row group 1), by the wavefront whose
    // turn comes after the last chunk.
    const bool extra = range == 0 && w == nchunks % WAVES;   // wave-uniform
    const int jp = partner_of(t, p.k, p.pi);
    uint4 kx = make_uint4(0, 0, 0, 0), vx = kx;
    bool entered = rg == 0;
    if (extra) {
        const int pe = jp >= 0 ? page_of(pages, s, pages.by_page.div(jp)) : -1;
        if (rg == 1 && pe >= 0) {
            const int64_t row = (int64_t)(pe * per_page + kv + (int)(jp - pages.by_page.div(jp) * pages.page)) * D;
            kx = ld16(kc + row);
            vx = ld16(vc + row);
            entered = true;
        } else if (rg == 0) {
            kx = ld16(kn + 4 * sub);
            vx = ld16(vn + 4 * sub);
        }
    }
    Rows ra, rb;
    load(w, ra);
    look_up(w + WAVES);

    if (rotary && tid < D / 2) s_cs[tid] = cos_sin(angle.pos, angle.freq);
    // Four elements of a row from 4 * sub on turned; `row`: where the others of their
    // pairs are.
    auto turned = [&](const float *row, float (&f)[4]) __attribute__((always_inline)) {
        float o[4];
        load4(row + 4 * (sub ^ (LPR / 2)), o);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int pair = sub % (LPR / 2) * 4 + e;
            const float2 cs = s_cs[pair];
            const float x = f[e] * cs.x, y = o[e] * cs.y;
            if (pair < p.r.pairs) f[e] = sub < LPR / 2 ? x - y : x + y;
        }
    };
    if (rotary) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < QN; ++j) turned((const float *)p.q_new + (first_head + min(j, nq - 1)) * D, q[j]);
    }
    float bias[QN], shift[QN];   // the partner's (and, clamped, the window's) prior
#pragma unroll
    for (int j = 0; j < QN; ++j) {
        const FusionBias fb = fusion_bias(gate[j], CLAMP);
        bias[j] = fb.partner;
        shift[j] = fb.local;
    }
    const float c2 = p.scale * kLog2e;

    float m[QN], l[QN], acc[QN][4];
#pragma unroll
    for (int j = 0; j < QN; ++j) {
        m[j] = -INFINITY;
        l[j] = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = 0.0f;
    }
    // logits (log2 units) of a row from this lane's part of it
    auto logits = [&](uint4 k, bool partner, float (&d)[QN]) __attribute__((always_inline)) {
        float kf[4];
        to_f32<float>(k, kf);
#pragma unroll
        for (int j = 0; j < QN; ++j) {
            float x = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) x += q[j][e] * kf[e];
            x = row_total<LPR>(x);
            d[j] = CLAMP ? clamped_logit(x * p.scale + (partner ? bias[j] : shift[j]), p.clamp) * kLog2e
                         : x * c2 + (partner ? bias[j] * kLog2e : 0.0f);
        }
    };

    if (extra) {
        if (rotary && rg == 0) {
            float f[4];
            to_f32<float>(kx, f);
            turned(kn, f);
            kx = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        }
        float d[QN], vf[4];
        logits(kx, rg == 1, d);
        to_f32<float>(vx, vf);
#pragma unroll
        for (int j = 0; j < QN; ++j) {
            if (!entered) continue;
            m[j] = d[j];
            l[j] = weight(d[j], d[j] == -INFINITY ? 0.0f : d[j]);   // 1, 0 or NaN
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] = l[j] * vf[e];
        }
        if (rg == 0 && g0 == 0) {   // no row read here is row t
            const int64_t row = (int64_t)(place * per_page + kv + (int)(t - pages.by_page.div(t) * pages.page)) * D + 4 * sub;
            *reinterpret_cast<uint4 *>((float *)pages.k + row) = kx;
            *reinterpret_cast<uint4 *>((float *)pages.v + row) = vx;
        }
    }

    auto attend = [&](Rows &r) __attribute__((always_inline)) {
        float sc[CH][QN], top[QN];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            logits(r.k[c], false, sc[c]);
#pragma unroll
            for (int j = 0; j < QN; ++j) {
                sc[c][j] = r.there[c] ? sc[c][j] : -INFINITY;
                top[j] = c == 0 ? sc[c][j] : fmaxf(top[j], sc[c][j]);
            }
        }
        bool need = false;
#pragma unroll
        for (int j = 0; j < QN; ++j) need = need || top[j] > m[j] + kTau;
        if (__builtin_amdgcn_ballot_w64(need)) {
#pragma unroll
            for (int j = 0; j < QN; ++j) {
                const float m_new = top[j] > m[j] + kTau ? top[j] : m[j];
                const float a = m_new == m[j] ? 1.0f : __builtin_amdgcn_exp2f(m[j] - m_new);
                m[j] = m_new;
                l[j] *= a;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][e] *= a;
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            // rows that are not there may hold anything
            if (!r.there[c]) r.v[c] = make_uint4(0, 0, 0, 0);
            float vf[4];
            to_f32<float>(r.v[c], vf);
#pragma unroll
            for (int j = 0; j < QN; ++j) {
                const float pr = weight(sc[c][j], m[j] == -INFINITY ? 0.0f : m[j]);
                l[j] += pr;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][e] += pr * vf[e];
            }
        }
    };
    for (int ch = w; ch < nchunks; ch += 2 * WAVES) {
        load(ch + WAVES, rb);
        look_up(ch + 2 * WAVES);
        attend(ra);
        if (ch + WAVES >= nchunks) break;
        load(ch + 2 * WAVES, ra);
        look_up(ch + 3 * WAVES);
        attend(rb);
    }

    // Merge the row groups of the wavefront (lanes with the same sub).
#pragma unroll
    for (int j = 0; j < QN; ++j) {
        float M = m[j];
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
        const float f = m[j] == M ? 1.0f : __builtin_amdgcn_exp2f(m[j] - M);
        m[j] = M;
        l[j] *= f;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] *= f;
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1) {
            l[j] += __shfl_xor(l[j], o);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] += __shfl_xor(acc[j][e], o);
        }
        if (rg == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s_acc[w][j][4 * sub + e] = acc[j][e];
            if (sub == 0) {
                s_m[w][j] = m[j];
                s_l[w][j] = l[j];
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < nq * D; i += 64 * WAVES) {
        const int j = i / D, e = i % D;
        float M = -INFINITY;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) M = fmaxf(M, s_m[x][j]);
        float L = 0.0f, o = 0.0f;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) {
            const float f = s_m[x][j] == M ? 1.0f : __builtin_amdgcn_exp2f(s_m[x][j] - M);
            L += s_l[x][j] * f;
            o += s_acc[x][j][e] * f;
        }
        if (part) {
            const int64_t at = (int64_t)range * p.S * p.H + first_head + j;
            p.part_o[at * D + e] = o;
            if (e == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(M, L);
        } else {
            ((float *)p.out)[first_head * D + i] = o / L;
            if (e == 0 && p.lse) {
                const FusionBias fb = fusion_bias(p.gate[s * p.gss + (hk * G + g0 + j) * p.gsh], CLAMP);
                p.lse[first_head + j] = (M + __log2f(L)) * kLn2 + fb.lse_shift;
            }
        }
    }
    if (!part && p.len_out && hk == 0 && g0 == 0 && tid == 0) p.len_out[s] = t + 1;
}

template <int D, int QN, bool CLAMP, bool ONCE>
hipError_t launch_w(const PagedStepParams &p, int64_t groups, int q_groups, hipStream_t stream) {
    if (p.parts == 0 && groups <= 256)
        return launch_kernel(decode_paged_f32_kernel<D, QN, CLAMP, ONCE, 8>, dim3((unsigned)groups), dim3(512), stream, p, q_groups);
    return launch_kernel(decode_paged_f32_kernel<D, QN, CLAMP, ONCE, 4>, dim3((unsigned)(groups * std::max(p.parts, 1))), dim3(256), stream,
                         p, q_groups);
}

template <int D, int QN, bool CLAMP>
hipError_t launch_q(const PagedStepParams &p, hipStream_t stream) {
    const int q_groups = (p.H / p.Hk + QN - 1) / QN;
    const int64_t groups = (int64_t)p.S * p.Hk * q_groups;
    return read_once(p, q_groups, 4) ? launch_w<D, QN, CLAMP, true>(p, groups, q_groups, stream)
                                     : launch_w<D, QN, CLAMP, false>(p, groups, q_groups, stream);
}

template <int D, bool CLAMP>
hipError_t launch_d(const PagedStepParams &p, hipStream_t stream) {
    const int G = p.H / p.Hk;
    if (G == 1) return launch_q<D, 1, CLAMP>(p, stream);
    if (G == 2) return launch_q<D, 2, CLAMP>(p, stream);
    return G <= 4 ? launch_q<D, 4, CLAMP>(p, stream) : launch_q<D, 8, CLAMP>(p, stream);
}

}  // namespace

hipError_t launch_decode_paged_f32(const PagedStepParams &p, hipStream_t stream) {
    const bool clamp = p.clamp > 0.0f;
    if (p.D == 64) return clamp ? launch_d<64, true>(p, stream) : launch_d<64, false>(p, stream);
    return clamp ? launch_d<128, true>(p, stream) : launch_d<128, false>(p, stream);
}

}  // namespace pi_attn
