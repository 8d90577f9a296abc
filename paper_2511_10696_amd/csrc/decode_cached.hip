// decode_cached.hip -- the decode step over quantised caches and the one behind
// a shared prefix: causal pi-Attention of one new row a sequence, caches in the
// working type (float32 or bf16) or e4m3 (e4m3.h), fp32 arithmetic, D = 64 or
// 128.
//
// With t = plen + len_in[s], the working set W_t (Sec. 3.5, eq. online_ws) is
// the window's rows max(0, t - k)..t - 1, the partner t - pi and the new row,
// which is appended to the sequence's own cache (quantised first, and attended
// as it is stored).  Rows below plen lie in the prefix, the others in the own
// cache.  The softmax is joined from parts: the prefix rows of the windows are
// taken chunk by chunk for all sequences at once (prefix_rows.hip), each chunk
// leaving (max, sum, weighted values) for every sequence and head; one
// work-group per (s, h) here takes the own rows, the partner and the new row,
// and the parts like rows whose weight is the part's sum.
//
// Own rows as in decode.hip: 16 bytes a lane, so a load instruction reads 1 KiB
// of whole rows, CH of them of keys and of values in flight in each wavefront.
// A quantised row's scale moves into its score and into its weight, both exact
// (powers of two); codes become floats two an instruction.
//
// Few (s, h) with long windows: a work-group per range of own rows, each
// leaving a part, and a last launch that joins them.  Short prefixes: read with
// the own rows, in the same launch.
//
// What bounds it: HBM with many long windows (64 sequences of 32 heads, D = 128,
// k = 512, e4m3: 274 MB in 45 us, 6.1 TB/s; 90 from bf16 caches), one launch and
// two round trips with few (one sequence 6.3 us, 3.5 of them an empty launch).
#include <algorithm>

#include "cached.h"
#include "decode_rows.h"
#include "e4m3.h"
#include "pi_common.h"

namespace pi_attn {

namespace {

template <typename ST>
constexpr bool kQuantised = false;
template <>
constexpr bool kQuantised<e4m3> = true;

// What a lane holds of a row.
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

// EPL consecutive elements of a row in the working type, from their loads.
template <typename T, int EPL>
__device__ inline void wide_f32(const uint4 (&u)[EPL * sizeof(T) / 16], float (&f)[EPL]) {
    constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < EPL / N; ++i) {
        float x[N];
        to_f32<T>(u[i], x);
#pragma unroll
        for (int e = 0; e < N; ++e) f[i * N + e] = x[e];
    }
}

// A new row in the caches' type: the lane's codes, and the row's byte.
template <int LPR>
__device__ inline uint4 quantise16(const float (&x)[16], unsigned &byte) {
    unsigned a = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) a = max(a, finite_bits(x[e]));
    byte = e4m3_byte(row_max<LPR>(a));
    const float inv = e4m3_inverse(byte);
    return make_uint4(e4m3_pack4(x, inv), e4m3_pack4(x + 4, inv), e4m3_pack4(x + 8, inv), e4m3_pack4(x + 12, inv));
}

// What a launch does of a step: all of it, where no prefix row is in a window
// (ALONE), where they were taken in parts (WHOLE) or are read here, by each
// sequence for itself (DIRECT); one range of own rows (RANGE: a part), or of
// prefix and own rows (DIRECT_RANGE); or the join of the parts (JOIN).
enum { ALONE, WHOLE, DIRECT, RANGE, DIRECT_RANGE, JOIN };

template <typename T, typename ST, int D, bool CLAMP, int MODE, int WAVES, int CH, bool ONCE>
__global__ __launch_bounds__(64 * WAVES) void decode_cached_kernel(CachedParams p) {
    using R = Row<ST, D>;
    constexpr bool Q = kQuantised<ST>;
    constexpr bool PART = MODE == RANGE || MODE == DIRECT_RANGE;
    constexpr bool BOTH = MODE == DIRECT || MODE == DIRECT_RANGE;   // window rows in either table
    constexpr int LPR = R::LPR, RPI = R::RPI, EPL = R::EPL;
    constexpr int RPC = RPI * CH;   // rows per chunk

    __shared__ float s_m[WAVES], s_l[WAVES];
    __shared__ float s_acc[WAVES][D];

    const DecodeParams &d = p.d;
    const DivMod range_of = divmod(blockIdx.x, PART ? p.own_parts : 1);
    const int64_t sh = range_of.quot;
    const int range = (int)range_of.rem;
    const DivMod head_of = divmod(range_of.quot, d.H);
    const int s = (int)head_of.quot, h = (int)head_of.rem;
    const int64_t n_sh = (int64_t)d.S * d.H;
    const int tid = threadIdx.x, lane = __lane_id();
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int sub = lane % LPR, rg = lane / LPR;
    T *out = (T *)d.out + sh * D;

    constexpr int WIDE = EPL * (int)sizeof(T) / 16;   // loads of a lane's elements in the working type
    const int n = d.len_in[s];   // own rows
    auto load_wide = [&](const void *row, uint4 (&u)[WIDE]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < WIDE; ++i) u[i] = ld16((const T *)row + sh * D + sub * EPL + i * (EPL / WIDE));
    };
    uint4 qw[WIDE];
    if constexpr (MODE != JOIN) load_wide(d.q_new, qw);
    const FusionBias fb = fusion_bias(d.gate[s * d.gss + h * d.gsh], CLAMP);

    if (n < 0 || n >= d.cap) {
        if (PART) return;
        for (int i = tid; i < D; i += 64 * WAVES) out[i] = (T)NAN;
        if (tid == 0) {
            if (d.lse) d.lse[sh] = NAN;
            if (d.len_out && h == 0) d.len_out[s] = n;
        }
        return;
    }
    const int t = p.plen + n;
    const int lo = window_lo(t, d.k);

    float m = -INFINITY, l = 0.0f;
    float acc[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[e] = 0.0f;
    // Raises the maximum to that of the row groups' logits.
    auto raise = [&](float cmax) __attribute__((always_inline)) {
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1) cmax = fmaxf(cmax, __shfl_xor(cmax, o));
        const float m_new = fmaxf(m, cmax);
        const float m_use = m_new == -INFINITY ? 0.0f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m - m_use);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int e = 0; e < EPL; ++e) acc[e] *= alpha;
        return m_use;
    };

    if constexpr (MODE != JOIN) {
        const int64_t head = sh * (int64_t)d.cap;
        uint8_t *kc = (uint8_t *)d.k_cache + (head * D + sub * EPL) * sizeof(ST);
        uint8_t *vc = (uint8_t *)d.v_cache + (head * D + sub * EPL) * sizeof(ST);
        constexpr int64_t RB = D * sizeof(ST);   // bytes of a row

        float qf[EPL];
        wide_f32<T, EPL>(qw, qf);
        const float c2 = d.scale * kLog2e;

        // window rows first + [0, nwin): own rows, or (BOTH) positions
        const int first = BOTH ? lo : max(lo - p.plen, 0);
        const int nwin = (BOTH ? t : n) - first;
        const int64_t shared = h * p.pcap;
        const uint8_t *kp = (const uint8_t *)p.k_prefix + (shared * D + sub * EPL) * sizeof(ST);
        const uint8_t *vp = (const uint8_t *)p.v_prefix + (shared * D + sub * EPL) * sizeof(ST);
        const int all = (nwin + RPC - 1) / RPC;
        // this launch's chunks
        const int per = PART ? (all + p.own_parts - 1) / p.own_parts : all;
        const int chunk0 = min(range * per, all), nchunks = min(per, all - chunk0);

        uint4 kr[CH], vr[CH];
        unsigned kb[CH], vb[CH];
        // Slots past the window read its last row again (and count as zeros below).
        auto load = [&](int ch) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                int64_t row = first + min(ch * RPC + c * RPI + rg, nwin - 1);
                const uint8_t *ka = kc, *va = vc;
                const uint8_t *kea = p.k_exp + head, *vea = p.v_exp + head;
                if constexpr (BOTH) {
                    const bool own = row >= p.plen;
                    row = own ? row - p.plen : row;
                    ka = own ? ka : kp;
                    va = own ? va : vp;
                    kea = own ? kea : p.k_prefix_exp + shared;
                    vea = own ? vea : p.v_prefix_exp + shared;
                }
                kr[c] = ONCE ? ld16_once(ka + row * RB) : ld16(ka + row * RB);
                vr[c] = ONCE ? ld16_once(va + row * RB) : ld16(va + row * RB);
                if constexpr (Q) {
                    kb[c] = kea[row];
                    vb[c] = vea[row];
                }
            }
        };
        // logit (log2 units) of a row from this lane's part of it
        auto logit = [&](uint4 k, unsigned byte, float bias) __attribute__((always_inline)) {
            float kf[EPL];
            unpack<ST, EPL>(k, kf);
            float part = 0.0f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) part += qf[e] * kf[e];
            part = row_sum<LPR>(part);
            if constexpr (Q) part *= e4m3_scale(byte);
            if constexpr (CLAMP) return clamped_logit(part * d.scale + bias, d.clamp) * kLog2e;
            return part * c2 + bias * kLog2e;
        };

        // The slot of the new row (row group 0) and the partner (row group 1),
        // by the wavefront whose turn comes after the last chunk.
        const bool extra = range == 0 && w == nchunks % WAVES;   // wave-uniform
        const int jp = partner_of(t, d.k, d.pi);
        const bool par = rg == 1 && jp >= 0;
        uint4 kx = make_uint4(0, 0, 0, 0), vx = kx;
        unsigned kxb = 127, vxb = 127;
        uint4 kw[WIDE], vw[WIDE];
        if (extra) {
            load_wide(d.k_new, kw);
            load_wide(d.v_new, vw);
        }
        if (extra && par) {
            const bool own = jp >= p.plen;
            const int64_t row = own ? jp - p.plen : jp;
            kx = ld16((own ? kc : kp) + row * RB);
            vx = ld16((own ? vc : vp) + row * RB);
            if constexpr (Q) {
                kxb = (own ? p.k_exp + head : p.k_prefix_exp + shared)[row];
                vxb = (own ? p.v_exp + head : p.v_prefix_exp + shared)[row];
            }
        }
        if (w < nchunks) load(chunk0 + w);
        if (extra) {
            if constexpr (Q) {
                float kn[EPL], vn[EPL];
                wide_f32<T, EPL>(kw, kn);
                wide_f32<T, EPL>(vw, vn);
                unsigned kby, vby;
                const uint4 kq = quantise16<LPR>(kn, kby), vq = quantise16<LPR>(vn, vby);
                if (!par) {
                    kx = kq;
                    vx = vq;
                    kxb = kby;
                    vxb = vby;
                }
            } else if (!par) {
                kx = kw[0];
                vx = vw[0];
            }
            const float v = logit(kx, kxb, rg == 1 ? fb.partner : fb.local);
            const bool entry = rg == 0 || par;
            const float sc = entry ? v : -INFINITY;
            m = sc;
#pragma unroll
            for (int o = LPR; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
            const float pr = __builtin_amdgcn_exp2f(sc - (m == -INFINITY ? 0.0f : m));
            l = pr;
            float vf[EPL];
            unpack<ST, EPL>(vx, vf);
            if (entry) {
                const float pv = Q ? pr * e4m3_scale(vxb) : pr;
#pragma unroll
                for (int e = 0; e < EPL; ++e) acc[e] = pv * vf[e];
            }
            // append the new row as own row n (no row read here is row n)
            if (rg == 0) {
                *reinterpret_cast<uint4 *>(kc + n * RB) = kx;
                *reinterpret_cast<uint4 *>(vc + n * RB) = vx;
                if (Q && sub == 0) {
                    p.k_exp[head + n] = (uint8_t)kxb;
                    p.v_exp[head + n] = (uint8_t)vxb;
                }
            }
        }
        for (int i = w; i < nchunks; i += WAVES) {
            const int ch = chunk0 + i;
            if (i != w) load(ch);
            float sc[CH];
            float cmax = -INFINITY;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const float v = logit(kr[c], kb[c], fb.local);
                sc[c] = ch * RPC + c * RPI + rg < nwin ? v : -INFINITY;
                cmax = fmaxf(cmax, sc[c]);
            }
            const float m_use = raise(cmax);
            if ((ch + 1) * RPC > nwin) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    if (ch * RPC + c * RPI + rg >= nwin) vr[c] = make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const float pr = __builtin_amdgcn_exp2f(sc[c] - m_use);
                l += pr;
                const float pv = Q ? pr * e4m3_scale(vb[c]) : pr;
                float vf[EPL];
                unpack<ST, EPL>(vr[c], vf);
#pragma unroll
                for (int e = 0; e < EPL; ++e) acc[e] += pv * vf[e];
            }
        }
    }

    // The parts: of the prefix chunks that this window meets, and (JOIN) of the
    // ranges of own rows.
    // (Loaded before the rows they would be there by now, and cost the registers of
    // a wavefront a SIMD: 40 us as it is, 43 so, 64 sequences of 32 heads behind
    // 4096 e4m3 rows, 128 own ones.)
    const int parts = MODE == WHOLE || MODE == JOIN ? p.chunks + (MODE == JOIN ? p.own_parts : 0) : 0;
    for (int x = w * RPI; x < parts; x += WAVES * RPI) {
        const int y = x + rg;
        const bool there = y < parts && (y >= p.chunks || (lo < p.plen && lo < chunk_end(p, y)));
        const int64_t at = (int64_t)y * n_sh + sh;
        float2 ml = make_float2(-INFINITY, 0.0f);
        f32x4 o[EPL / 4];
#pragma unroll
        for (int i = 0; i < EPL / 4; ++i) o[i] = f32x4{};
        if (there) {
            ml = *reinterpret_cast<const float2 *>(p.part_ml + 2 * at);
#pragma unroll
            for (int i = 0; i < EPL / 4; ++i)
                o[i] = *reinterpret_cast<const f32x4 *>(p.part_o + at * D + sub * EPL + 4 * i);
        }
        const float m_use = raise(ml.x);
        const float f = __builtin_amdgcn_exp2f(ml.x - m_use);
        l += f * ml.y;
#pragma unroll
        for (int i = 0; i < EPL / 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[4 * i + e] += f * o[i][e];
    }

    // Merge the row groups of the wavefront (lanes with the same sub).
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1) {
        l += __shfl_xor(l, o);
#pragma unroll
        for (int e = 0; e < EPL; ++e) acc[e] += __shfl_xor(acc[e], o);
    }
    if (rg == 0) {
#pragma unroll
        for (int e = 0; e < EPL; ++e) s_acc[w][sub * EPL + e] = acc[e];
        if (sub == 0) {
            s_m[w] = m;
            s_l[w] = l;
        }
    }
    __syncthreads();

    for (int i = tid; i < D; i += 64 * WAVES) {
        float M = -INFINITY;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) M = fmaxf(M, s_m[x]);
        float L = 0.0f, o = 0.0f;
#pragma unroll
        for (int x = 0; x < WAVES; ++x) {
            const float f = s_m[x] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(s_m[x] - M);
            L += s_l[x] * f;
            o += s_acc[x][i] * f;
        }
        if (PART) {
            const int64_t at = (int64_t)(p.chunks + range) * n_sh + sh;
            p.part_o[at * D + i] = o;
            if (i == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(M, L);
        } else {
            out[i] = (T)(o / L);
            if (i == 0) {
                if (d.lse) d.lse[sh] = (M + __log2f(L)) * kLn2 + fb.lse_shift;
                if (d.len_out && h == 0) d.len_out[s] = n + 1;
            }
        }
    }
}

// ONCE, by the bytes of a step's window rows, as in decode.hip: they are read
// once, and kept in the caches they only push out what is there.
constexpr int64_t kKeepBytes = 12 << 20;

template <typename T, typename ST, int D, bool CLAMP, int MODE, int WAVES, int CH>
hipError_t launch_n(const CachedParams &p, hipStream_t stream) {
    const int64_t n = (int64_t)p.d.S * p.d.H;
    constexpr bool kMany = MODE != DIRECT && MODE != DIRECT_RANGE && MODE != JOIN;   // window rows of its own, and many
    const bool once = kMany && 2 * n * std::min(p.d.k, p.d.cap) * D * (int64_t)sizeof(ST) > kKeepBytes;
    const int64_t groups = n * (MODE == RANGE || MODE == DIRECT_RANGE ? p.own_parts : 1);
    return launch_kernel(once ? decode_cached_kernel<T, ST, D, CLAMP, MODE, WAVES, CH, kMany>
                              : decode_cached_kernel<T, ST, D, CLAMP, MODE, WAVES, CH, false>,
                         dim3((unsigned)groups), dim3(64 * WAVES), stream, p);
}

// Wavefronts and chunk size, by the load instructions of a window's keys and the
// launch: a few (s, h) by the chain of one wavefront, a chip full of them by the
// wavefronts that it holds and by what a work-group costs beside its rows.  us,
// 8 wavefronts of 4 slots, 4 of 4 and 2 of 4, e4m3, D = 128: 512 (s, h) of 128
// rows (16 loads) 7.1, 7.1 and 8.0, of 512 rows 13.4, 14.8 (of 2 slots) and 18.0;
// 2048 of 32 rows 16.4, 8.4 and 7.9, of 128 rows 21.3, 16.8 and 15.2, of 256 rows
// 29.1, 26.6 and 24.8, of 512 rows 46.8, 47 and 47.4, of 1024 rows 87.0, - and
// 92.0.  With the parts of a prefix, 2048 (s, h): of 256 rows 44.7, 42.5 and 36.5,
// of 512 rows 48.0, - and 41.3; bf16 of 256 rows 50.5, - and 48.4.
// The other types and D, the rule's choice first: from 2048 (s, h) on, 2 wavefronts
// and 4, e4m3 D = 64 of 65 rows 8.0 and 8.5, of 257 16.1 and 16.9, float32 over
// e4m3 D = 128 of 129 15.5 and 17.0, parts of a bf16 prefix D = 128 of 129 50 and
// 51, of a float32 one D = 64 60.6 and 58.0.  From 33 loads on, 8 and 4: e4m3 D =
// 64, 256 (s, h) of 1025 rows 9.6 and 10.8, bf16 behind chunks D = 128, 128 of 257
// 22.3 and 23.3, float32 D = 64 18.3 and 19.6; the prefix's rows too, bf16 D = 128,
// 32 of 520 7.3 and 9.6, float32 D = 64 32 of 420 5.1 and 6.0; 2048 of 513 45.5 and
// 44.9.  From 5 loads on, up to 1024 (s, h), 4 wavefronts of 4 and 2 of 2: e4m3 D =
// 128 of 41 rows 32 (s, h) 4.2 and 4.7, 1024 6.5 and 6.2; D = 64 256 of 100 4.4 and
// 5.4, float32 over e4m3 4.3 and 5.3.
template <typename T, typename ST, int D, bool CLAMP>
hipError_t launch_w(const CachedParams &p, hipStream_t stream) {
    const int64_t n = (int64_t)p.d.S * p.d.H;
    const int rows = std::min(p.d.k, p.d.cap) + (p.direct ? p.near : 0);
    const int loads = (rows + Row<ST, D>::RPI - 1) / Row<ST, D>::RPI;
    const bool many = n >= 2048;
    if (p.own_parts) {
        const hipError_t e = p.direct ? launch_n<T, ST, D, CLAMP, DIRECT_RANGE, 4, 4>(p, stream)
                                      : launch_n<T, ST, D, CLAMP, RANGE, 4, 4>(p, stream);
        return e != hipSuccess ? e : launch_n<T, ST, D, CLAMP, JOIN, 4, 4>(p, stream);
    }
    if (p.direct) {
        return loads > 32 ? launch_n<T, ST, D, CLAMP, DIRECT, 8, 4>(p, stream)
                          : launch_n<T, ST, D, CLAMP, DIRECT, 4, 4>(p, stream);
    }
    if (p.chunks) {
        if (many && loads <= 64) return launch_n<T, ST, D, CLAMP, WHOLE, 2, 4>(p, stream);
        return loads > 32 ? launch_n<T, ST, D, CLAMP, WHOLE, 8, 4>(p, stream)
                          : launch_n<T, ST, D, CLAMP, WHOLE, 4, 4>(p, stream);
    }
    if (loads > 32) return launch_n<T, ST, D, CLAMP, ALONE, 8, 4>(p, stream);
    if (many && loads > 2) return launch_n<T, ST, D, CLAMP, ALONE, 2, 4>(p, stream);
    if (loads > 8 || (loads > 4 && n <= 1024)) return launch_n<T, ST, D, CLAMP, ALONE, 4, 4>(p, stream);
    return launch_n<T, ST, D, CLAMP, ALONE, 2, 2>(p, stream);
}

template <typename T, typename ST>
hipError_t launch_t(const CachedParams &p, hipStream_t stream) {
    const bool clamp = p.d.clamp > 0.0f;
    if (p.d.D == 64) return clamp ? launch_w<T, ST, 64, true>(p, stream) : launch_w<T, ST, 64, false>(p, stream);
    return clamp ? launch_w<T, ST, 128, true>(p, stream) : launch_w<T, ST, 128, false>(p, stream);
}

}  // namespace

// Whether the sequences read the prefix's rows for themselves, with their own: as
// long as one (s, h) has a chain of few loads, and all of them together little
// more than the launch that is saved.  us, by chunks and so: bf16 D = 64, 64
// (s, h) 1024 rows 8.7 and 7.3, 2048 rows 8.8 and 10.5; D = 128, 128 (s, h) 512
// rows 9.8 and 7.2, 1024 rows 9.9 and 11.0; e4m3 D = 128, 128 (s, h) 1024 rows
// 10.3 and 9.7, 2048 rows 10.9 and 15.0; 2048 (s, h): bf16 D = 64 128 rows (67 MB
// in all) 12.9 and 9.2, 256 rows 13.2 and 15.0; e4m3 D = 64 256 rows (67 MB) 15.3
// and 13.4, 512 rows 16.0 and 22.2.
bool read_directly(const CachedParams &p, int element_bytes) {
    const int64_t bytes = 2 * (int64_t)p.near * p.d.D * element_bytes;   // keys and values of an (s, h)
    return bytes <= 300 << 10 && (int64_t)p.d.S * p.d.H * bytes <= 100 << 20;
}

// Ranges of own rows that a step is split into: where a few (s, h) have long
// chains of loads, which a second launch costs less than; enough for 512
// work-groups, of 64 KB at least.  us, whole and split, e4m3, D = 128: 32 (s, h)
// of 1600 rows 13.5 and 11.1, of 16384 rows 99.4 and 27.8; 64 of 2048 17.0 and
// 13.1, 128 of 2048 18.3 and 18.2; 256 of 2048 24.5 and 28.2, of 8192 80.9 and
// 85.0; 1024 and 2048 work-groups the same but for 256 (s, h) and one.  Behind 200
// prefix rows that are read with them: 32 (s, h) of 16384 rows 112.8 and 32.7, of
// 1700 15.6 and 11.1, 128 of 1600 15.2 and 15.7, of 4000 35.6 and 31.0; bf16 32 of
// 8000 81.6 and 29.7, of 1000 12.8 and 10.0.
int own_parts(const CachedParams &p, int element_bytes) {
    const int64_t n = (int64_t)p.d.S * p.d.H, own = std::min(p.d.k, p.d.cap - 1);
    const int64_t bytes = 2 * own * p.d.D * element_bytes;   // keys and values of an (s, h)
    if (bytes < 384 << 10 || n > 128) return 0;
    return (int)std::min<int64_t>(512 / n, bytes >> 16);
}

// At most `most` chunks of whole tiles, as even as they can be.
int64_t even_chunks(const CachedParams &p, int64_t most) {
    const int64_t tiles = (p.near + p.tile - 1) / p.tile, per = (tiles + most - 1) / most;
    return (tiles + per - 1) / per;
}

// The sizes of the parts, by the problem's sizes alone (the lengths lie in
// device memory).
void plan_decode_cached(CachedParams &p, bool bf16) {
    p.near = std::min(p.d.k, p.plen);
    p.tile = p.chunks = p.own_parts = 0;
    p.direct = false;
    if (p.near > 0 && !read_directly(p, bf16 ? 2 : 4)) {
        // the most chunks that any caches' type takes: of 64 rows, two a CU
        const int queries = prefix_shape(p, bf16).queries;
        const int64_t side = (int64_t)p.d.H * ((p.d.S + queries - 1) / queries);
        p.tile = 64;
        p.chunks = (int)even_chunks(p, std::max<int64_t>(1, 512 / side));
    }
    p.own_parts = own_parts(p, bf16 ? 2 : 4);
}

hipError_t launch_decode_cached(const CachedParams &planned, bool bf16, hipStream_t stream) {
    CachedParams p = planned;
    if ((int64_t)p.d.S * p.d.H == 0) return hipSuccess;
    if (p.near > 0 && read_directly(p, p.k_exp ? 1 : bf16 ? 2 : 4)) {
        p.direct = true;
        p.chunks = 0;
    }
    p.own_parts = own_parts(p, p.k_exp ? 1 : bf16 ? 2 : 4);
    if (p.chunks) {
        const PrefixShape shape = prefix_shape(p, bf16);
        const int64_t side = (int64_t)p.d.H * ((p.d.S + shape.queries - 1) / shape.queries);
        p.tile = shape.tile;
        p.chunks = (int)even_chunks(p, std::min<int64_t>(p.chunks, std::max<int64_t>(1, 256 * shape.per_cu / side)));
        const hipError_t e = launch_prefix(p, bf16, stream);
        if (e != hipSuccess) return e;
    }
    if (p.k_exp) return bf16 ? launch_t<__bf16, e4m3>(p, stream) : launch_t<float, e4m3>(p, stream);
    return bf16 ? launch_t<__bf16, __bf16>(p, stream) : launch_t<float, float>(p, stream);
}

}  // namespace pi_attn
