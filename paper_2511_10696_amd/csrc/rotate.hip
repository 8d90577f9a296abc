// rotate.hip -- rotary positions of queries and keys (rotary.h), and their
// backward, the transpose: float32 or bf16 rows in and out, D = 64 or 128, fp32
// arithmetic, one rounding at the end.
//
// A wavefront takes a few positions (as many as one load instruction covers, a
// lane holding both halves of its pairs) and four heads, with the cosines and sines
// that it forms once; q's and k's heads are one list.  A lane reads all that it writes
// over before it writes, so that a result may take its input's place.
//
// What bounds it: HBM, rows read and written once.  Wavefronts that are next to each
// other take neighbours in memory: the heads of a position where these lie together
// ([B][N][H][D], 8192 positions of 4 x 40 heads, bf16, D = 128: 110 us, 671 MB at 6.1
// TB/s, and 123 the other way), the positions of a head otherwise ([B][H][N][D], 4 x
// 32 heads: 89 us and 109).  More heads a wavefront, walked one group after the other,
// save cosines and lose memory streams: one sequence of 32768, float32 to bf16, 333 us
// with all 64 heads, 291 with four.  A plain copy reaches 4.9 TB/s.
#include <algorithm>

#include "half_rows.h"
#include "paged.h"
#include "pi_common.h"

namespace pi_attn {

namespace {

constexpr int WAVES = 4;
constexpr int U = 4;   // heads of a wavefront, their loads in flight together

template <typename TI, typename TO, int D, bool ONCE>
__global__ __launch_bounds__(64 * WAVES) void rotate_kernel(RotateParams p) {
    using R = HalfRow<TI, D>;
    constexpr int EPL = R::EPL;
    const int lane = __lane_id(), sub = lane % R::LPR, rg = lane / R::LPR;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * WAVES + (threadIdx.x >> 6));
    uint32_t tile, group;
    p.order.place(wave, tile, group);
    const uint32_t r = tile * R::RPI + rg;
    if (tile >= p.order.tiles || r >= p.rows) return;
    const uint32_t b = p.by_n.div(r), n = r - b * p.N;
    const int h0 = (int)group * U, heads = p.H + p.Hk;

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
    Piece<TI, EPL> lo[U], hi[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = min(h0 + u, heads - 1);
        const TI *x = h < p.H ? q + h * p.qsh : k + (h - p.H) * p.ksh;
        lo[u] = load_piece<TI, EPL, ONCE>(x);
        hi[u] = load_piece<TI, EPL, ONCE>(x + D / 2);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = h0 + u;
        if (h >= heads) break;
        float a[EPL], c[EPL];
        widen<TI, EPL>(lo[u], a);
        widen<TI, EPL>(hi[u], c);
#pragma unroll
        for (int e = 0; e < EPL; ++e) turn(a[e], c[e], cs[e], turned[e]);
        TO *y = h < p.H ? qo + h * p.oqsh : ko + (h - p.H) * p.oksh;
        store_piece<TO, EPL, ONCE>(narrowed<TO, EPL>(a), y);
        store_piece<TO, EPL, ONCE>(narrowed<TO, EPL>(c), y + D / 2);
    }
}

// Rows are not kept in the caches from 192 MB on, read and written, where a lane's
// halves lie in different lines of 128 bytes: 131 MB 14.5 us kept and 17.7 not, 262 MB
// (float32) 46.8 and 45.7, 537 MB 95 and 89; bf16 at D = 64 (halves of 64 bytes) 537 MB
// 97 and 108.
constexpr int64_t kKeepBytes = 192 << 20;

template <typename TI, typename TO, int D>
hipError_t launch_d(RotateParams p, hipStream_t stream) {
    using R = HalfRow<TI, D>;
    const int heads = p.H + p.Hk;
    const int64_t tiles = ((int64_t)p.rows + R::RPI - 1) / R::RPI, groups = ((int64_t)heads + U - 1) / U;
    const bool heads_first = p.H > 0 ? p.qsh < p.qsn : p.ksh < p.ksn;
    p.order = WaveOrder(heads_first, (uint32_t)tiles, (uint32_t)groups);
    constexpr bool kWide = D / 2 * sizeof(TI) >= 128;
    const bool once = kWide && (int64_t)p.rows * heads * D * (int64_t)(sizeof(TI) + sizeof(TO)) > kKeepBytes;
    return launch_in_order<WAVES>(once ? rotate_kernel<TI, TO, D, kWide> : rotate_kernel<TI, TO, D, false>, p, stream);
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
