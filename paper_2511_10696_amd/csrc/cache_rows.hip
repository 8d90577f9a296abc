// cache_rows.hip -- rows into and out of the quantised caches (the format is
// in e4m3.h): float32 or bf16 rows, D = 64 or 128.
//
// A row is covered by the lanes of its 16-byte pieces in the working type, so
// the wide side is read or written in whole lines; a lane's 4 or 8 codes are
// one word or two.  A wavefront takes U load instructions of rows, the keys'
// and the values' alike, all of them in flight before the first is used.
//
// What bounds them: HBM, by bytes moved (a bf16 row of 256 bytes becomes 129).
#include "decode_rows.h"
#include "e4m3.h"
#include "kernels.h"

namespace pi_attn {

namespace {

constexpr int WAVES = 4;

// Row r of S x H x n: sequence, head, index.
struct Place {
    int s, h, i;
};

__device__ inline Place place(uint32_t r, const CacheRowsParams &p) {
    const uint32_t sh = p.by_n.div(r), s = p.by_h.div(sh);
    return Place{(int)s, (int)(sh - s * p.H), (int)(r - sh * p.n)};
}

// Cache row of the place, -1 where there is none.
__device__ inline int64_t cache_row(const Place &a, const CacheRowsParams &p) {
    const int64_t at = (int64_t)a.i + (p.start ? p.start[a.s] : 0);
    const bool there = at >= 0 && at < p.cap && (!p.count || a.i < p.count[a.s]);
    return there ? ((int64_t)a.s * p.H + a.h) * p.cap + at : -1;
}

// The codes of one lane: a word for each four elements.
template <int EPL>
struct Codes {
    unsigned w[EPL / 4];
};

template <typename T, int D>
__device__ inline void store_piece(uint4 raw, uint8_t *codes, uint8_t *bytes, int64_t row, int sub) {
    using R = Row<T, D>;
    float x[R::EPL];
    to_f32<T>(raw, x);
    unsigned a = 0;
#pragma unroll
    for (int e = 0; e < R::EPL; ++e) a = max(a, finite_bits(x[e]));
    const unsigned byte = e4m3_byte(row_max<R::LPR>(a));
    if (row < 0) return;
    const float inv = e4m3_inverse(byte);
    Codes<R::EPL> c;
#pragma unroll
    for (int i = 0; i < R::EPL / 4; ++i) c.w[i] = e4m3_pack4(x + 4 * i, inv);
    *reinterpret_cast<Codes<R::EPL> *>(codes + row * D + sub * R::EPL) = c;
    if (sub == 0) bytes[row] = (uint8_t)byte;
}

template <typename T, int D, int U>
__global__ __launch_bounds__(64 * WAVES) void store_kernel(CacheRowsParams p) {
    using R = Row<T, D>;
    const int lane = __lane_id(), sub = lane % R::LPR, rg = lane / R::LPR;
    const uint32_t r0 = (blockIdx.x * WAVES + (threadIdx.x >> 6)) * (U * R::RPI) + rg;
    uint4 k[U], v[U];
    int64_t row[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t r = r0 + u * R::RPI;
        row[u] = -1;
        k[u] = v[u] = make_uint4(0, 0, 0, 0);
        if (r < p.rows) {
            const Place a = place(r, p);
            row[u] = cache_row(a, p);
            if (row[u] >= 0) {
                const int64_t off = a.s * p.sb + a.h * p.sh + a.i * p.sn + sub * R::EPL;
                k[u] = ld16((const T *)p.k + off);
                v[u] = ld16((const T *)p.v + off);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        store_piece<T, D>(k[u], p.k_cache, p.k_exp, row[u], sub);
        store_piece<T, D>(v[u], p.v_cache, p.v_exp, row[u], sub);
    }
}

template <typename T, int EPL>
__device__ inline void load_piece(const Codes<EPL> &c, unsigned byte, T *to) {
    const float scale = e4m3_scale(byte);
    float x[EPL];
#pragma unroll
    for (int i = 0; i < EPL / 4; ++i) e4m3_unpack4(c.w[i], x + 4 * i);
    T y[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) y[e] = (T)(x[e] * scale);
    *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(y);
}

template <typename T, int D, int U>
__global__ __launch_bounds__(64 * WAVES) void load_kernel(CacheRowsParams p) {
    using R = Row<T, D>;
    const int lane = __lane_id(), sub = lane % R::LPR, rg = lane / R::LPR;
    const uint32_t r0 = (blockIdx.x * WAVES + (threadIdx.x >> 6)) * (U * R::RPI) + rg;
    Codes<R::EPL> k[U], v[U];
    unsigned kb[U], vb[U];
    int64_t off[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t r = r0 + u * R::RPI;
        off[u] = -1;
        k[u] = v[u] = Codes<R::EPL>{};   // absent rows: code 0, value 0
        kb[u] = vb[u] = 127;
        if (r < p.rows) {
            const Place a = place(r, p);
            const int64_t row = cache_row(a, p);
            off[u] = a.s * p.sb + a.h * p.sh + a.i * p.sn + sub * R::EPL;
            if (row >= 0) {
                k[u] = *reinterpret_cast<const Codes<R::EPL> *>(p.k_cache + row * D + sub * R::EPL);
                v[u] = *reinterpret_cast<const Codes<R::EPL> *>(p.v_cache + row * D + sub * R::EPL);
                kb[u] = p.k_exp[row];
                vb[u] = p.v_exp[row];
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (off[u] < 0) continue;
        load_piece<T, R::EPL>(k[u], kb[u], (T *)p.k + off[u]);
        load_piece<T, R::EPL>(v[u], vb[u], (T *)p.v + off[u]);
    }
}

template <typename T, int D, int U>
hipError_t launch_u(const CacheRowsParams &p, bool store, hipStream_t stream) {
    const uint32_t per = WAVES * U * Row<T, D>::RPI;
    return launch_kernel(store ? store_kernel<T, D, U> : load_kernel<T, D, U>, dim3((p.rows - 1) / per + 1),
                         dim3(64 * WAVES), stream, p);
}

template <typename T>
hipError_t launch_t(const CacheRowsParams &p, bool store, hipStream_t stream) {
    const bool many = p.rows >= 1 << 14;
    if (p.D == 64) return many ? launch_u<T, 64, 4>(p, store, stream) : launch_u<T, 64, 1>(p, store, stream);
    return many ? launch_u<T, 128, 4>(p, store, stream) : launch_u<T, 128, 1>(p, store, stream);
}

}  // namespace

hipError_t launch_cache_rows(const CacheRowsParams &p, bool store, bool bf16, hipStream_t stream) {
    return bf16 ? launch_t<__bf16>(p, store, stream) : launch_t<float>(p, store, stream);
}

}  // namespace pi_attn
