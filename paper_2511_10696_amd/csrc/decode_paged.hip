// decode_paged.hip -- the decode step over a paged cache: causal pi-Attention of
// one new row a sequence, H query heads over Hk key heads, pages in the working
// type (float32 or bf16) or e4m3 (e4m3.h), fp32 arithmetic, D = 64 or 128.
//
// With t = len_in[s], the working set W_t (Sec. 3.5, eq. online_ws) is the
// window's rows max(0, t - k)..t - 1, the partner t - pi and the new row, which is
// turned by its position (rotary.h), written to its page as row t and attended as
// stored.  Rows whose page is not there (given back) are not in W_t.
//
// One work-group per sequence, key head, up to QN of its query heads and, where
// few of these have long windows, range of the window; ranges leave parts (max,
// sum, weighted values) that a second launch joins in a fixed order.  A row is
// covered by lanes with 16-byte loads; every row read serves QN queries.  Each
// group of lanes that covers a row keeps a softmax of its own (nothing is
// exchanged from row to row); they are merged at the end.
//
// What bounds it: HBM.
#include <algorithm>
#include <stdlib.h>

#include "half_rows.h"
#include "paged_step.h"

namespace pi_attn {

namespace {

// What a lane holds of a cached row.
template <typename ST, int EPL>
__device__ inline void unpack(uint4 u, float (&f)[EPL]) {
    if constexpr (kQuantised<ST>) {
        e4m3_unpack4(u.x, f);
        e4m3_unpack4(u.y, f + 4);
        e4m3_unpack4(u.z, f + 8);
        e4m3_unpack4(u.w, f + 12);
    } else {
        to_f32<ST>(u, f);
    }
}

// EPL consecutive elements in the working type.
template <typename T, int EPL>
__device__ inline void load_wide(const T *from, float (&f)[EPL]) {
    constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < EPL / N; ++i) {
        float x[N];
        to_f32<T>(ld16(from + i * N), x);
#pragma unroll
        for (int e = 0; e < N; ++e) f[i * N + e] = x[e];
    }
}

template <typename T, typename ST, int D, int QN, bool PART, int WAVES, int CH>
__global__ __launch_bounds__(64 * WAVES) void decode_paged_kernel(PagedStepParams p, int q_groups) {
    using R = Row<ST, D>;
    constexpr bool Q = kQuantised<ST>;
    constexpr int LPR = R::LPR, RPI = R::RPI, EPL = R::EPL;
    constexpr int RPC = RPI * CH;   // rows per chunk
    constexpr int64_t RB = D * sizeof(ST);

    __shared__ float s_m[WAVES][QN], s_l[WAVES][QN];
    __shared__ float s_acc[WAVES][QN][D];
    __shared__ float2 s_cs[WAVES][D / 2];

    // The first range of every window, then the second: the shorter last ones come late.
    const DivMod range_of = divmod(blockIdx.x, PART ? p.S * p.Hk * q_groups : gridDim.x);
    const int range = (int)range_of.quot;
    const DivMod group_of = divmod(range_of.rem, q_groups);
    const DivMod head_of = divmod(group_of.quot, p.Hk);
    const int s = (int)head_of.quot, hk = (int)head_of.rem;
    const int G = p.H / p.Hk, g0 = (int)group_of.rem * QN, nq = min(QN, G - g0);
    const int64_t first_head = (int64_t)s * p.H + hk * G + g0;   // of S * H
    const int tid = threadIdx.x, lane = __lane_id();
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int sub = lane % LPR, rg = lane / LPR;
    const Pages &g = p.pages;
    const int t = p.len_in[s];

    if (!has_place(g, s, t)) {
        if (PART) return;
        for (int i = tid; i < nq * D; i += 64 * WAVES) ((T *)p.out)[first_head * D + i] = (T)NAN;
        if (p.lse && tid < nq) p.lse[first_head + tid] = NAN;
        if (p.len_out && hk == 0 && g0 == 0 && tid == 0) p.len_out[s] = t;
        return;
    }
    const int lo = window_lo(t, p.k);
    const int len = PART ? range_len(p, t - lo) : t - lo;   // of a range
    if (range > 0 && (int64_t)range * len >= t - lo) return;
    // this work-group's window rows: first + [0, nwin)
    const int first = lo + range * len, nwin = min(len, t - first);
    const int nchunks = (nwin + RPC - 1) / RPC;

    const int64_t kv = (int64_t)hk * g.page;                  // row 0 of this head in page 0
    const int64_t per_page = (int64_t)p.Hk * g.page;
    const uint8_t *kc = (const uint8_t *)g.k + sub * 16, *vc = (const uint8_t *)g.v + sub * 16;
    uint4 kr[CH], vr[CH];
    unsigned kb[CH], vb[CH];
    int entry[CH];
    // The chunk's pages, looked up ahead of its rows.  Slots past the window read
    // its last row again.
    auto position = [&](int ch, int c) __attribute__((always_inline)) {
        return (uint32_t)(first + min(ch * RPC + c * RPI + rg, nwin - 1));
    };
    auto look_up = [&](int ch) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < CH; ++c) entry[c] = page_of(g, s, g.by_page.div(position(ch, c)));
    };
    auto load = [&](int ch, bool (&there)[CH]) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const uint32_t at = position(ch, c);
            there[c] = entry[c] >= 0 && ch * RPC + c * RPI + rg < nwin;
            const int64_t row = max(entry[c], 0) * per_page + kv + (at - g.by_page.div(at) * g.page);
            kr[c] = ld16(kc + row * RB);
            vr[c] = ld16(vc + row * RB);
            if constexpr (Q) {
                kb[c] = g.k_exp[row];
                vb[c] = g.v_exp[row];
            }
        }
    };
    bool there[CH];
    if (w < nchunks) {
        look_up(w);
        load(w, there);
        if (w + WAVES < nchunks) look_up(w + WAVES);
    }

    // Cosines and sines: one pair a lane, by every wavefront for itself.
    const bool rotary = p.r.freq != nullptr;
    if (rotary) {
        if (lane < D / 2) s_cs[w][lane] = cos_sin_of(p.r, lane, s, 0, t);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    // This lane's elements of a new row, turned; the other half of its pairs is read too.
    auto load_new = [&](const T *row, bool turns, float (&f)[EPL]) __attribute__((always_inline)) {
        load_wide<T, EPL>(row + sub * EPL, f);
        if (!turns) return;
        float o[EPL];
        load_wide<T, EPL>(row + (sub ^ (LPR / 2)) * EPL, o);
        const int pair = sub % (LPR / 2) * EPL;
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
            const float2 cs = s_cs[w][pair + e];
            const float x = f[e] * cs.x, y = o[e] * cs.y;
            if (pair + e < p.r.pairs) f[e] = sub < LPR / 2 ? x - y : x + y;
        }
    };
    float qf[QN][EPL];
    float bias[QN], shift[QN];   // the partner's (and, clamped, the window's) prior
    const bool clamped = p.clamp > 0.0f;
#pragma unroll
    for (int j = 0; j < QN; ++j) {
        const int jj = min(j, nq - 1);
        load_new((const T *)p.q_new + (first_head + jj) * D, rotary, qf[j]);
        const FusionBias fb = fusion_bias(p.gate[s * p.gss + (hk * G + g0 + jj) * p.gsh], clamped);
        bias[j] = fb.partner;
        shift[j] = clamped ? fb.local : fb.lse_shift;
    }
    const float c2 = p.scale * kLog2e;

    float m[QN], l[QN], acc[QN][EPL];
#pragma unroll
    for (int j = 0; j < QN; ++j) {
        m[j] = -INFINITY;
        l[j] = 0.0f;
#pragma unroll
        for (int e = 0; e < EPL; ++e) acc[j][e] = 0.0f;
    }
    // logits (log2 units) of a row from this lane's part of it
    auto logits = [&](uint4 k, unsigned byte, bool partner, float (&d)[QN]) __attribute__((always_inline)) {
        float kf[EPL];
        unpack<ST, EPL>(k, kf);
#pragma unroll
        for (int j = 0; j < QN; ++j) {
            float part = 0.0f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) part += qf[j][e] * kf[e];
            part = row_sum<LPR>(part);
            if constexpr (Q) part *= e4m3_scale(byte);
            d[j] = clamped ? clamped_logit(part * p.scale + (partner ? bias[j] : shift[j]), p.clamp) * kLog2e
                           : part * c2 + (partner ? bias[j] * kLog2e : 0.0f);
        }
    };

    // The new row (row group 0) and the partner (row group 1), by the wavefront
    // whose turn comes after the last chunk.
    if (range == 0 && w == nchunks % WAVES) {
        const int jp = partner_of(t, p.k, p.pi);
        const int pe = jp >= 0 ? page_of(g, s, g.by_page.div(jp)) : -1;
        const bool par = rg == 1 && pe >= 0;
        uint4 kx = make_uint4(0, 0, 0, 0), vx = kx;
        unsigned kxb = 127, vxb = 127;
        if (par) {
            const int64_t row = pe * per_page + kv + (jp - g.by_page.div(jp) * g.page);
            kx = ld16(kc + row * RB);
            vx = ld16(vc + row * RB);
            if constexpr (Q) {
                kxb = g.k_exp[row];
                vxb = g.v_exp[row];
            }
        }
        const T *kn = (const T *)p.k_new + ((int64_t)s * p.Hk + hk) * D, *vn = (const T *)p.v_new + ((int64_t)s * p.Hk + hk) * D;
        float f[EPL];
        load_new(kn, rotary, f);
        if constexpr (Q) {
            auto quantised = [&](unsigned &byte) __attribute__((always_inline)) {
                unsigned a = 0;
#pragma unroll
                for (int e = 0; e < EPL; ++e) a = max(a, finite_bits(f[e]));
                byte = e4m3_byte(row_max<LPR>(a));
                const float inv = e4m3_inverse(byte);
                return make_uint4(e4m3_pack4(f, inv), e4m3_pack4(f + 4, inv), e4m3_pack4(f + 8, inv), e4m3_pack4(f + 12, inv));
            };
            unsigned kby, vby;
            const uint4 kq = quantised(kby);
            load_new(vn, false, f);
            const uint4 vq = quantised(vby);
            if (!par) {
                kx = kq;
                vx = vq;
                kxb = kby;
                vxb = vby;
            }
        } else if (!par) {
            vx = ld16(vn + sub * EPL);
            kx = rotary ? __builtin_bit_cast(uint4, narrowed<T, EPL>(f)) : ld16(kn + sub * EPL);
        }
        const bool entered = rg == 0 || par;
        float d[QN], vf[EPL];
        logits(kx, kxb, rg == 1, d);
        unpack<ST, EPL>(vx, vf);
#pragma unroll
        for (int j = 0; j < QN; ++j) {
            if (!entered) continue;
            m[j] = d[j];
            const float pr = __builtin_amdgcn_exp2f(d[j] - (d[j] == -INFINITY ? 0.0f : d[j]));   // 1, or NaN
            l[j] = pr;
            const float pv = Q ? pr * e4m3_scale(vxb) : pr;
#pragma unroll
            for (int e = 0; e < EPL; ++e) acc[j][e] = pv * vf[e];
        }
        if (rg == 0 && g0 == 0) {   // no row read here is row t
            const uint32_t slot = g.by_page.div(t);
            const int64_t row = page_of(g, s, slot) * per_page + kv + (t - slot * g.page);
            *reinterpret_cast<uint4 *>((uint8_t *)g.k + sub * 16 + row * RB) = kx;
            *reinterpret_cast<uint4 *>((uint8_t *)g.v + sub * 16 + row * RB) = vx;
            if (Q && sub == 0) {
                g.k_exp[row] = (uint8_t)kxb;
                g.v_exp[row] = (uint8_t)vxb;
            }
        }
    }

    for (int ch = w; ch < nchunks; ch += WAVES) {
        if (ch != w) {
            load(ch, there);
            if (ch + WAVES < nchunks) look_up(ch + WAVES);
        }
        float sc[CH][QN], top[QN];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            logits(kr[c], kb[c], false, sc[c]);
#pragma unroll
            for (int j = 0; j < QN; ++j) {
                sc[c][j] = there[c] ? sc[c][j] : -INFINITY;
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
                for (int e = 0; e < EPL; ++e) acc[j][e] *= a;
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            // rows that are not there may hold anything
            if (!there[c]) vr[c] = make_uint4(0, 0, 0, 0);
            const float vs = Q && there[c] ? e4m3_scale(vb[c]) : 1.0f;
            float vf[EPL];
            unpack<ST, EPL>(vr[c], vf);
#pragma unroll
            for (int j = 0; j < QN; ++j) {
                const float pr = __builtin_amdgcn_exp2f(sc[c][j] - (m[j] == -INFINITY ? 0.0f : m[j]));
                l[j] += pr;
                const float pv = Q ? pr * vs : pr;
#pragma unroll
                for (int e = 0; e < EPL; ++e) acc[j][e] += pv * vf[e];
            }
        }
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
        for (int e = 0; e < EPL; ++e) acc[j][e] *= f;
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1) {
            l[j] += __shfl_xor(l[j], o);
#pragma unroll
            for (int e = 0; e < EPL; ++e) acc[j][e] += __shfl_xor(acc[j][e], o);
        }
        if (rg == 0) {
#pragma unroll
            for (int e = 0; e < EPL; ++e) s_acc[w][j][sub * EPL + e] = acc[j][e];
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
        if (PART) {
            const int64_t at = (int64_t)range * p.S * p.H + first_head + j;
            p.part_o[at * D + e] = o;
            if (e == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(M, L);
        } else {
            ((T *)p.out)[first_head * D + i] = (T)(o / L);
            if (e == 0 && p.lse) {
                const FusionBias fb = fusion_bias(p.gate[s * p.gss + (hk * G + g0 + j) * p.gsh], clamped);
                p.lse[first_head + j] = (M + __log2f(L)) * kLn2 + fb.lse_shift;
            }
        }
    }
    if (!PART && p.len_out && hk == 0 && g0 == 0 && tid == 0) p.len_out[s] = t + 1;
}

// Joins the parts of a query head: every wavefront takes each WAVES-th, four at a
// time.
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void join_kernel(PagedStepParams p) {
    constexpr int EPL = D / 64, U = 4;
    __shared__ float s_m[WAVES], s_l[WAVES];
    __shared__ float s_o[WAVES][D];
    const DivMod head_of = divmod(blockIdx.x, p.H);
    const int s = (int)head_of.quot, h = (int)head_of.rem;
    const int tid = threadIdx.x, lane = __lane_id();
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t head = blockIdx.x, heads = (int64_t)p.S * p.H;
    const int t = p.len_in[s];
    if (!has_place(p.pages, s, t)) {
        if (tid < D) ((T *)p.out)[head * D + tid] = (T)NAN;
        if (p.lse && tid == 0) p.lse[head] = NAN;
        if (p.len_out && h == 0 && tid == 0) p.len_out[s] = t;
        return;
    }
    const int n = ranges_of(p, t - window_lo(t, p.k));
    float M = -INFINITY, L = 0.0f, o[EPL] = {};
    for (int x = w; x < n; x += WAVES * U) {
        float2 ml[U];
        float po[U][EPL];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = min(x + u * WAVES, n - 1) * heads + head;
            ml[u] = *reinterpret_cast<const float2 *>(p.part_ml + 2 * at);
#pragma unroll
            for (int e = 0; e < EPL; ++e) po[u][e] = p.part_o[at * D + lane + 64 * e];
        }
        float m_new = M;
#pragma unroll
        for (int u = 0; u < U; ++u) m_new = fmaxf(m_new, x + u * WAVES < n ? ml[u].x : -INFINITY);
        const float a = M == m_new ? 1.0f : __builtin_amdgcn_exp2f(M - m_new);
        M = m_new;
        L *= a;
#pragma unroll
        for (int e = 0; e < EPL; ++e) o[e] *= a;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (x + u * WAVES >= n) break;
            const float b = ml[u].x == M ? 1.0f : __builtin_amdgcn_exp2f(ml[u].x - M);
            L += ml[u].y * b;
#pragma unroll
            for (int e = 0; e < EPL; ++e) o[e] += po[u][e] * b;
        }
    }
#pragma unroll
    for (int e = 0; e < EPL; ++e) s_o[w][lane + 64 * e] = o[e];
    if (lane == 0) {
        s_m[w] = M;
        s_l[w] = L;
    }
    __syncthreads();
    if (tid < D) {
        float top = -INFINITY, sum = 0.0f, out = 0.0f;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) top = fmaxf(top, s_m[x]);
#pragma unroll
        for (int x = 0; x < WAVES; ++x) {
            const float f = s_m[x] == top ? 1.0f : __builtin_amdgcn_exp2f(s_m[x] - top);
            sum += s_l[x] * f;
            out += s_o[x][tid] * f;
        }
        ((T *)p.out)[head * D + tid] = (T)(out / sum);
        if (tid == 0) {
            if (p.lse) {
                const FusionBias fb = fusion_bias(p.gate[s * p.gss + h * p.gsh], p.clamp > 0.0f);
                p.lse[head] = (top + __log2f(sum)) * kLn2 + fb.lse_shift;
            }
            if (p.len_out && h == 0) p.len_out[s] = t + 1;
        }
    }
}

template <typename T, int D>
hipError_t launch_join_d(const PagedStepParams &p, hipStream_t stream) {
    const dim3 grid((unsigned)(p.S * p.H));
    return p.parts > 32 ? launch_kernel(join_kernel<T, D, 16>, grid, dim3(1024), stream, p)
                        : launch_kernel(join_kernel<T, D, 4>, grid, dim3(256), stream, p);
}

template <typename T>
hipError_t launch_join(const PagedStepParams &p, hipStream_t stream) {
    return p.D == 64 ? launch_join_d<T, 64>(p, stream) : launch_join_d<T, 128>(p, stream);
}

template <typename T, typename ST, int D, int QN>
hipError_t launch_q(const PagedStepParams &p, hipStream_t stream) {
    const int G = p.H / p.Hk, q_groups = (G + QN - 1) / QN;
    const int64_t groups = (int64_t)p.S * p.Hk * q_groups;
    if (p.parts) {
        const hipError_t e = launch_kernel(decode_paged_kernel<T, ST, D, QN, true, 4, 4>, dim3((unsigned)(groups * p.parts)),
                                           dim3(256), stream, p, q_groups);
        return e != hipSuccess ? e : launch_join<T>(p, stream);
    }
    return launch_kernel(decode_paged_kernel<T, ST, D, QN, false, 4, 4>, dim3((unsigned)groups), dim3(256), stream, p, q_groups);
}

template <typename T, typename ST, int D>
hipError_t launch_d(const PagedStepParams &p, hipStream_t stream) {
    const int G = p.H / p.Hk;
    if (G == 1) return launch_q<T, ST, D, 1>(p, stream);
    if (G == 2) return launch_q<T, ST, D, 2>(p, stream);
    return launch_q<T, ST, D, 4>(p, stream);
}

template <typename T, typename ST>
hipError_t launch_t(const PagedStepParams &p, hipStream_t stream) {
    return p.D == 64 ? launch_d<T, ST, 64>(p, stream) : launch_d<T, ST, 128>(p, stream);
}

}  // namespace

void plan_decode_paged(PagedStepParams &p, bool bf16) {
    const int64_t n = (int64_t)p.S * p.Hk, rows = longest_window(p);
    p.parts = p.range = 0;
    if (rows <= 1024 || n >= 4096) return;
    int64_t r = std::clamp<int64_t>((rows * n / 768 + 127) & ~(int64_t)127, 256, 1024);
    if (getenv("PI_RANGE")) r = atoi(getenv("PI_RANGE"));
    const int64_t parts = std::min<int64_t>((rows + r - 1) / r, std::max<int64_t>(1, 4096 / n));
    if (parts < 2) return;
    p.range = (int)r;
    p.parts = (int)parts;
}

hipError_t launch_decode_paged(const PagedStepParams &p, bool bf16, hipStream_t stream) {
    if ((p.pages.k_exp || bf16) && (p.H / p.Hk > 1 || getenv("PI_TILES"))) {
        const hipError_t e = launch_decode_paged_tiles(p, bf16, stream);
        if (e != hipSuccess || !p.parts) return e;
        return bf16 ? launch_join<__bf16>(p, stream) : launch_join<float>(p, stream);
    }
    if (p.pages.k_exp) return bf16 ? launch_t<__bf16, e4m3>(p, stream) : launch_t<float, e4m3>(p, stream);
    return bf16 ? launch_t<__bf16, __bf16>(p, stream) : launch_t<float, float>(p, stream);
}

}  // namespace pi_attn
