// rotate.hip -- rotary positions of queries and keys (rotary.h), and their
// backward, the transpose: float32 or bf16 rows in and out, D = 64 or 128, fp32
// arithmetic, one rounding at the end.
//
// A wavefront takes a few positions (as many as one load instruction covers, a
// lane holding both halves of its pairs) and walks over heads with the cosines
// and sines that it forms once; q's and k's heads are one list.  A lane reads all
// that it writes over before it writes, so that a result may take its input's
// place.
//
// What bounds it: HBM, rows read and written once.
#include <algorithm>

#include "half_rows.h"
#include "paged.h"
#include "pi_common.h"

namespace pi_attn {

namespace {

constexpr int WAVES = 4;
constexpr int U = 4;   // heads whose loads are in flight together

template <typename TI, typename TO, int D, bool ONCE>
__global__ __launch_bounds__(64 * WAVES) void rotate_kernel(RotateParams p) {
    using R = HalfRow<TI, D>;
    constexpr int EPL = R::EPL;
    const int lane = __lane_id(), sub = lane % R::LPR, rg = lane / R::LPR;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * WAVES + (threadIdx.x >> 6));
    const uint32_t tile = p.by_splits.div(wave);
    const uint32_t r = tile * R::RPI + rg;
    if (r >= p.rows) return;
    const uint32_t b = p.by_n.div(r), n = r - b * p.N;
    const int h0 = (int)(wave - tile * p.splits) * p.per, h1 = min(h0 + p.per, p.H + p.Hk);

    const TI *q = (const TI *)p.q + b * p.qsb + n * p.qsn + sub * EPL;
    const TI *k = (const TI *)p.k + b * p.ksb + n * p.ksn + sub * EPL;
    TO *qo = (TO *)p.q_out + b * p.oqsb + n * p.oqsn + sub * EPL;
    TO *ko = (TO *)p.k_out + b * p.oksb + n * p.oksn + sub * EPL;
    float2 cs[EPL];
    bool turned[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
        const int i = sub * EPL + e;
        cs[e] = cos_sin_of(p.r, i, b, n, (int)n);
        if (p.back) cs[e].y = -cs[e].y;
        turned[e] = i < p.r.pairs;
    }
    for (int h = h0; h < h1; h += U) {
        Piece<TI, EPL> lo[U], hi[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int hh = min(h + u, h1 - 1);
            const TI *x = hh < p.H ? q + hh * p.qsh : k + (hh - p.H) * p.ksh;
            lo[u] = load_piece<TI, EPL, ONCE>(x);
            hi[u] = load_piece<TI, EPL, ONCE>(x + D / 2);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int hh = h + u;
            if (hh >= h1) break;
            float a[EPL], c[EPL];
            widen<TI, EPL>(lo[u], a);
            widen<TI, EPL>(hi[u], c);
#pragma unroll
            for (int e = 0; e < EPL; ++e) turn(a[e], c[e], cs[e], turned[e]);
            TO *y = hh < p.H ? qo + hh * p.oqsh : ko + (hh - p.H) * p.oksh;
            store_piece<TO, EPL, ONCE>(narrowed<TO, EPL>(a), y);
            store_piece<TO, EPL, ONCE>(narrowed<TO, EPL>(c), y + D / 2);
        }
    }
}

template <typename TI, typename TO, int D>
hipError_t launch_d(RotateParams p, hipStream_t stream) {
    using R = HalfRow<TI, D>;
    const int heads = p.H + p.Hk;
    const int64_t tiles = ((int64_t)p.rows + R::RPI - 1) / R::RPI;
    p.splits = (int)std::clamp<int64_t>(8192 / tiles, 1, (heads + U - 1) / U);
    p.per = ((heads + p.splits - 1) / p.splits + U - 1) / U * U;
    p.splits = (heads + p.per - 1) / p.per;
    p.by_splits = Divisor(p.splits);
    const int64_t groups = (tiles * p.splits + WAVES - 1) / WAVES;
    if (groups >= 1 << 24) return hipErrorInvalidConfiguration;   // 2^32 threads
    return launch_kernel(rotate_kernel<TI, TO, D, false>, dim3((unsigned)groups), dim3(64 * WAVES), stream, p);
}

template <typename TI, typename TO>
hipError_t launch_t(const RotateParams &p, hipStream_t stream) {
    return p.D == 64 ? launch_d<TI, TO, 64>(p, stream) : launch_d<TI, TO, 128>(p, stream);
}

}  // namespace

hipError_t launch_rotate(const RotateParams &p, bool bf16_in, bool bf16_out, hipStream_t stream) {
    if (bf16_in) return bf16_out ? launch_t<__bf16, __bf16>(p, stream) : launch_t<__bf16, float>(p, stream);
    return bf16_out ? launch_t<float, __bf16>(p, stream) : launch_t<float, float>(p, stream);
}

}  // namespace pi_attn
