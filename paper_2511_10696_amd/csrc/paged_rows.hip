// paged_rows.hip -- rows of keys and values into and out of a paged cache:
// float32 or bf16 rows, pages in the same type or quantised (e4m3.h), D = 64 or
// 128.  A store turns the keys by their positions on the way (rotary.h), in fp32,
// with one rounding to what the page holds.
//
// A wavefront takes a few rows (as many as one load instruction covers) and two heads,
// looks the rows' pages up and forms their cosines and sines once.
//
// What bounds it: HBM, rows read and written once.  Wavefronts that are next to each
// other take neighbours in memory: the heads of a row where these lie together
// ([S][n][H][D], 8 prompts of 3000 to 6000 rows of 16 heads, turned, bf16, D = 128: 101
// us, 590 MB at 5.8 TB/s, and 114 the other way), the rows of a head otherwise ([S][H]
// [n][D], 4 of 16000 rows of 8 heads into e4m3: 71 us, 394 MB, and 78).  All heads a
// wavefront, walked two at a time: 121 and 75.  A plain copy reaches 4.9 TB/s.
#include <algorithm>

#include "e4m3.h"
#include "half_rows.h"
#include "paged.h"
#include "pi_common.h"

namespace pi_attn {

namespace {

constexpr int WAVES = 4;
constexpr int U = 2;   // heads of a wavefront, their keys' and values' loads in flight together

// What a lane does for its row, all heads alike.
struct Place {
    bool wanted;      // its position is within the table's reach, and the row in the count
    uint32_t s, i;    // sequence and row of k and v
    int at;           // its position
    int entry;        // the table's, not looked at before page() is asked
    uint32_t slot;

    template <int RPI>
    __device__ bool find(const PagedRowsParams &p, uint32_t tile, int rg) {
        const uint32_t r = tile * RPI + rg;
        if (tile >= p.order.tiles || r >= p.rows) return false;
        s = p.by_n.div(r);
        i = r - s * p.n;
        const int64_t pos = (int64_t)i + (p.start ? p.start[s] : 0);
        const Pages &g = p.pages;
        wanted = pos >= 0 && pos < (int64_t)g.page * g.max_pages && (!p.count || (int)i < p.count[s]);
        at = wanted ? (int)pos : 0;
        slot = g.by_page.div(at);
        entry = wanted ? g.table[(int64_t)s * g.max_pages + slot] : -1;
        return true;
    }
    __device__ int page(const Pages &g) const { return entry >= 0 && entry < g.n_pages ? entry : -1; }
    // Cache row of head 0; head h's is h * page further on.
    __device__ int64_t first(const PagedRowsParams &p) const {
        const Pages &g = p.pages;
        return (int64_t)max(page(g), 0) * p.Hk * g.page + (at - slot * g.page);
    }
};

// LD, SD: what is loaded, or stored, is not kept in the caches.
template <typename T, bool QUANT, int D, bool LD, bool SD>
__global__ __launch_bounds__(64 * WAVES) void paged_store_kernel(PagedRowsParams p) {
    using R = HalfRow<T, D>;
    constexpr int EPL = R::EPL;
    const int lane = __lane_id(), sub = lane % R::LPR, rg = lane / R::LPR;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * WAVES + (threadIdx.x >> 6));
    uint32_t tile, group;
    p.order.place(wave, tile, group);
    Place a;
    if (!a.find<R::RPI>(p, tile, rg) || !a.wanted) return;   // a row's lanes alike
    const int h0 = (int)group * U;
    const int64_t from = a.s * p.sb + a.i * p.sn + sub * EPL;
    const T *k = (const T *)p.k + from, *v = (const T *)p.v + from;

    Piece<T, EPL> kl[U], kh[U], vl[U], vh[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t x = min(h0 + u, p.Hk - 1) * p.sh;
        kl[u] = load_piece<T, EPL, LD>(k + x);
        kh[u] = load_piece<T, EPL, LD>(k + x + D / 2);
        vl[u] = load_piece<T, EPL, LD>(v + x);
        vh[u] = load_piece<T, EPL, LD>(v + x + D / 2);
    }
    float2 cs[EPL];
    bool turned[EPL];
    if (p.r.freq) {
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
            const int i = sub * EPL + e;
            cs[e] = cos_sin_of(p.r, i, a.s, a.i, a.at);
            turned[e] = i < p.r.pairs;
        }
    }
    const Pages &g = p.pages;
    if (a.page(g) < 0) return;
    const int64_t first = a.first(p);
    // A row's halves into head h's pages, as these hold them.
    auto put = [&](const Piece<T, EPL> &lo, const Piece<T, EPL> &hi, bool turns, int h, void *pages, uint8_t *exps)
        __attribute__((always_inline)) {
        const int64_t row = first + (int64_t)h * g.page;
        float x[EPL], y[EPL];
        if (QUANT || turns) {
            widen<T, EPL>(lo, x);
            widen<T, EPL>(hi, y);
        }
        if (turns) {
#pragma unroll
            for (int e = 0; e < EPL; ++e) turn(x[e], y[e], cs[e], turned[e]);
        }
        if constexpr (QUANT) {
            unsigned m = 0;
#pragma unroll
            for (int e = 0; e < EPL; ++e) m = max(m, max(finite_bits(x[e]), finite_bits(y[e])));
            const unsigned byte = e4m3_byte(row_max<R::LPR>(m));
            const float inv = e4m3_inverse(byte);
            Piece<uint8_t, EPL> cl, ch;
#pragma unroll
            for (int i = 0; i < EPL / 4; ++i) {
                cl.w[i] = e4m3_pack4(x + 4 * i, inv);
                ch.w[i] = e4m3_pack4(y + 4 * i, inv);
            }
            uint8_t *to = (uint8_t *)pages + row * D + sub * EPL;
            store_piece<uint8_t, EPL, SD>(cl, to);
            store_piece<uint8_t, EPL, SD>(ch, to + D / 2);
            if (sub == 0) exps[row] = (uint8_t)byte;
        } else {
            T *to = (T *)pages + row * D + sub * EPL;
            store_piece<T, EPL, SD>(turns ? narrowed<T, EPL>(x) : lo, to);
            store_piece<T, EPL, SD>(turns ? narrowed<T, EPL>(y) : hi, to + D / 2);
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (h0 + u >= p.Hk) break;
        put(kl[u], kh[u], p.r.freq != nullptr, h0 + u, g.k, g.k_exp);
        put(vl[u], vh[u], false, h0 + u, g.v, g.v_exp);
    }
}

template <typename T, bool QUANT, int D, bool LD, bool SD>
__global__ __launch_bounds__(64 * WAVES) void paged_load_kernel(PagedRowsParams p) {
    using R = HalfRow<T, D>;
    constexpr int EPL = R::EPL;
    using ST = typename std::conditional<QUANT, uint8_t, T>::type;   // what the pages hold
    const int lane = __lane_id(), sub = lane % R::LPR, rg = lane / R::LPR;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * WAVES + (threadIdx.x >> 6));
    uint32_t tile, group;
    p.order.place(wave, tile, group);
    Place a;
    if (!a.find<R::RPI>(p, tile, rg)) return;
    const bool there = a.page(p.pages) >= 0;
    const int64_t first = a.first(p);
    const int h0 = (int)group * U;
    const int64_t to = a.s * p.sb + a.i * p.sn + sub * EPL;
    T *k = (T *)p.k + to, *v = (T *)p.v + to;
    const Pages &g = p.pages;
    const ST *kp = (const ST *)g.k + sub * EPL, *vp = (const ST *)g.v + sub * EPL;
    auto out = [&](const Piece<ST, EPL> &x, unsigned byte, T *y) __attribute__((always_inline)) {
        if constexpr (QUANT) {
            const float scale = e4m3_scale(byte);
            float f[EPL];
#pragma unroll
            for (int i = 0; i < EPL / 4; ++i) e4m3_unpack4(x.w[i], f + 4 * i);
#pragma unroll
            for (int e = 0; e < EPL; ++e) f[e] *= scale;
            store_piece<T, EPL, SD>(narrowed<T, EPL>(f), y);
        } else {
            store_piece<T, EPL, SD>(x, y);
        }
    };
    Piece<ST, EPL> x[U][4];
    unsigned kb[U], vb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        kb[u] = vb[u] = 127;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[u][j] = Piece<ST, EPL>{};   // absent rows: zeros, in codes too
        if (there) {
            const int64_t row = first + (int64_t)min(h0 + u, p.Hk - 1) * g.page;
            x[u][0] = load_piece<ST, EPL, LD>(kp + row * D);
            x[u][1] = load_piece<ST, EPL, LD>(kp + row * D + D / 2);
            x[u][2] = load_piece<ST, EPL, LD>(vp + row * D);
            x[u][3] = load_piece<ST, EPL, LD>(vp + row * D + D / 2);
            if constexpr (QUANT) {
                kb[u] = g.k_exp[row];
                vb[u] = g.v_exp[row];
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (h0 + u >= p.Hk) break;
        const int64_t y = (h0 + u) * p.sh;
        out(x[u][0], kb[u], k + y);
        out(x[u][1], kb[u], k + y + D / 2);
        out(x[u][2], vb[u], v + y);
        out(x[u][3], vb[u], v + y + D / 2);
    }
}

// Rows are not kept in the caches from 128 MB on, read and written: 66 MB stored 13.9 us
// kept and 15.2 not, loaded 11.8 and 13.1; 229 MB 49.2 and 44.2, 47.8 and 41.9.  Loads of
// halves below 128 bytes share lines, and are kept: e4m3 to bf16, 361 MB, 65.4 us and 70.8.
constexpr int64_t kKeepBytes = 128 << 20;

template <typename T, bool QUANT, int D>
hipError_t launch_d(PagedRowsParams p, bool store, hipStream_t stream) {
    using R = HalfRow<T, D>;
    constexpr int NARROW = QUANT ? 1 : (int)sizeof(T);   // bytes of an element in the pages
    const int64_t tiles = ((int64_t)p.rows + R::RPI - 1) / R::RPI, groups = ((int64_t)p.Hk + U - 1) / U;
    p.order = WaveOrder(p.sh < p.sn, (uint32_t)tiles, (uint32_t)groups);
    const bool once = 2 * (int64_t)p.rows * p.Hk * D * (int64_t)(sizeof(T) + NARROW) > kKeepBytes;
    constexpr bool kStoreLd = D / 2 * sizeof(T) >= 128, kLoadLd = D / 2 * NARROW >= 128;
    if (store)
        return launch_in_order<WAVES>(once ? paged_store_kernel<T, QUANT, D, kStoreLd, true>
                                           : paged_store_kernel<T, QUANT, D, false, false>, p, stream);
    return launch_in_order<WAVES>(once ? paged_load_kernel<T, QUANT, D, kLoadLd, true>
                                       : paged_load_kernel<T, QUANT, D, false, false>, p, stream);
}

template <typename T>
hipError_t launch_t(const PagedRowsParams &p, bool store, hipStream_t stream) {
    if (p.pages.k_exp)
        return p.D == 64 ? launch_d<T, true, 64>(p, store, stream) : launch_d<T, true, 128>(p, store, stream);
    return p.D == 64 ? launch_d<T, false, 64>(p, store, stream) : launch_d<T, false, 128>(p, store, stream);
}

}  // namespace

hipError_t launch_paged_rows(const PagedRowsParams &p, bool store, bool bf16, hipStream_t stream) {
    return bf16 ? launch_t<__bf16>(p, store, stream) : launch_t<float>(p, store, stream);
}

}  // namespace pi_attn
