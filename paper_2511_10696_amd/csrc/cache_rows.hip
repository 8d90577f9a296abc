// cache_rows.hip -- rows into and out of the quantised caches (the format is
// in e4m3.h): float32 or bf16 rows, D = 64 or 128.
//
// A row is covered by the lanes of its 16-byte pieces in the working type, so
// the wide side is read or written in whole lines; a lane's 4 or 8 codes are
// one word or two.  A wavefront takes U load instructions of rows, the keys'
// and the values' alike, all of them in flight before the first is used.
//
// Many rows: a work-group takes a run of one head's.  The runs of a head follow
// one another, but with [S][n][H][D] storage of long prompts, of which the
// work-groups under way (some 2^17 rows) then hold few heads, that is every 32nd
// row of 256 bytes: there the heads of a run come first (one prompt of 32768 rows
// of 32 heads, D = 128: 181 -> 147 us stored, 208 -> 160 read; 16 of 2000, where
// the runs under way hold all heads, 134 and 142, 135 and 149).  Few rows, or few
// of each sequence: one after the other.
//
// What bounds them: HBM, by bytes moved (a bf16 row of 256 bytes becomes 129):
// 32 heads of 32768 rows of keys and values, D = 128, stored in 133 us (6.05 TB/s
// read and written, a plain copy 4.8), 16 sequences of 2000 read in 131.
// Large transfers leave the caches alone: what is read is not needed again, what
// is written is more than they hold.
#include <algorithm>

#include "cached.h"
#include "decode_rows.h"
#include "e4m3.h"
#include "pi_common.h"

namespace pi_attn {

namespace {

constexpr int WAVES = 4;

// Row of S x H x n: sequence, head, index; i is -1 past the last.
struct Place {
    int s, h, i;
};

// Of load instruction u of this lane's row group.  RUNS: runs of one head's rows.
template <int RPI, int U, bool RUNS>
__device__ inline Place place(int u, int rg, const CacheRowsParams &p) {
    const int w = threadIdx.x >> 6;
    const uint32_t group = p.first_group + blockIdx.x;
    if constexpr (RUNS) {
        const DivMod inner = divmod(group, p.heads_first ? p.H : p.runs);
        const DivMod outer = divmod(inner.quot, p.heads_first ? p.runs : p.H);
        const int h = (int)(p.heads_first ? inner.rem : outer.rem), run = (int)(p.heads_first ? outer.rem : inner.rem);
        const int i = run * (WAVES * U * RPI) + (w * U + u) * RPI + rg;
        return Place{(int)outer.quot, h, i < p.n ? i : -1};
    } else {
        const uint32_t r = (group * WAVES + w) * (U * RPI) + u * RPI + rg;
        if (r >= p.rows) return Place{0, 0, -1};
        const uint32_t sh = p.by_n.div(r), s = p.by_h.div(sh);
        return Place{(int)s, (int)(sh - s * p.H), (int)(r - sh * p.n)};
    }
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

template <typename T, int D, bool ONCE>
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
    unsigned *const to = reinterpret_cast<unsigned *>(codes + row * D + sub * R::EPL);
    if constexpr (ONCE) {
#pragma unroll
        for (int i = 0; i < R::EPL / 4; ++i) __builtin_nontemporal_store(c.w[i], to + i);
    } else {
        *reinterpret_cast<Codes<R::EPL> *>(to) = c;
    }
    if (sub == 0) bytes[row] = (uint8_t)byte;
}

template <typename T, int D, int U, bool RUNS, bool ONCE>
__global__ __launch_bounds__(64 * WAVES) void store_kernel(CacheRowsParams p) {
    using R = Row<T, D>;
    const int lane = __lane_id(), sub = lane % R::LPR, rg = lane / R::LPR;
    uint4 k[U], v[U];
    int64_t row[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Place a = place<R::RPI, U, RUNS>(u, rg, p);
        row[u] = a.i < 0 ? -1 : cache_row(a, p);
        k[u] = v[u] = make_uint4(0, 0, 0, 0);
        if (row[u] >= 0) {
            const int64_t off = a.s * p.sb + a.h * p.sh + a.i * p.sn + sub * R::EPL;
            k[u] = ONCE ? ld16_once((const T *)p.k + off) : ld16((const T *)p.k + off);
            v[u] = ONCE ? ld16_once((const T *)p.v + off) : ld16((const T *)p.v + off);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        store_piece<T, D, ONCE>(k[u], p.k_cache, p.k_exp, row[u], sub);
        store_piece<T, D, ONCE>(v[u], p.v_cache, p.v_exp, row[u], sub);
    }
}

template <typename T, int EPL, bool ONCE>
__device__ inline void load_piece(const Codes<EPL> &c, unsigned byte, T *to) {
    const float scale = e4m3_scale(byte);
    float x[EPL];
#pragma unroll
    for (int i = 0; i < EPL / 4; ++i) e4m3_unpack4(c.w[i], x + 4 * i);
    T y[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) y[e] = (T)(x[e] * scale);
    const raw16 out = *reinterpret_cast<const raw16 *>(y);
    if constexpr (ONCE) {
        __builtin_nontemporal_store(out, reinterpret_cast<raw16 *>(to));
    } else {
        *reinterpret_cast<raw16 *>(to) = out;
    }
}

template <typename T, int D, int U, bool RUNS, bool ONCE>
__global__ __launch_bounds__(64 * WAVES) void load_kernel(CacheRowsParams p) {
    using R = Row<T, D>;
    const int lane = __lane_id(), sub = lane % R::LPR, rg = lane / R::LPR;
    Codes<R::EPL> k[U], v[U];
    unsigned kb[U], vb[U];
    int64_t off[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Place a = place<R::RPI, U, RUNS>(u, rg, p);
        off[u] = -1;
        k[u] = v[u] = Codes<R::EPL>{};   // absent rows: code 0, value 0
        kb[u] = vb[u] = 127;
        if (a.i >= 0) {
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
        load_piece<T, R::EPL, ONCE>(k[u], kb[u], (T *)p.k + off[u]);
        load_piece<T, R::EPL, ONCE>(v[u], vb[u], (T *)p.v + off[u]);
    }
}

template <typename T, int D, int U, bool RUNS, bool ONCE>
hipError_t launch_n(CacheRowsParams p, bool store, hipStream_t stream) {
    constexpr uint32_t PER = WAVES * U * Row<T, D>::RPI;
    uint32_t groups = (p.rows - 1) / PER + 1;
    if (RUNS) {
        p.runs = ((uint32_t)p.n - 1) / PER + 1;
        groups = (uint32_t)p.S * p.H * p.runs;
        p.heads_first = p.sn > p.sh && (int64_t)p.n * p.H >= 1 << 18;
    }
    // a launch has fewer than 2^32 threads
    constexpr uint32_t kMost = 1u << 23;
    hipError_t e = hipSuccess;
    for (p.first_group = 0; e == hipSuccess && p.first_group < groups; p.first_group += kMost)
        e = launch_kernel(store ? store_kernel<T, D, U, RUNS, ONCE> : load_kernel<T, D, U, RUNS, ONCE>,
                          dim3(std::min(groups - p.first_group, kMost)), dim3(64 * WAVES), stream, p);
    return e;
}

// us, D = 128, rows one after the other: 32768 rows by one load instruction a
// lane 6.8 and 5.7 (stored, read), by four 7.8 and 6.4; 262144 rows 148 and 142
// as they come, 134 and 133 past the caches, but 96000 rows of D = 64 (55 MB) 15.5
// stored so, 16.4 past them; read, past them from the first sizes on: 17 MB 6.4
// and 4.9, 67 MB 21.3 and 15.7, 131 MB of float32 64.5 and 48.1.
constexpr int64_t kKeepStored = 96 << 20, kKeepLoaded = 12 << 20;

template <typename T, int D>
hipError_t launch_d(const CacheRowsParams &p, bool store, hipStream_t stream) {
    const int64_t wide = 2 * (int64_t)p.rows * D * sizeof(T), narrow = 2 * (int64_t)p.rows * (D + 1);
    const bool once = store ? wide + narrow > kKeepStored : wide > kKeepLoaded;
    if (p.rows >= 1 << 16 && p.n >= 64)
        return once ? launch_n<T, D, 4, true, true>(p, store, stream) : launch_n<T, D, 4, true, false>(p, store, stream);
    return once ? launch_n<T, D, 1, false, true>(p, store, stream) : launch_n<T, D, 1, false, false>(p, store, stream);
}

template <typename T>
hipError_t launch_t(const CacheRowsParams &p, bool store, hipStream_t stream) {
    return p.D == 64 ? launch_d<T, 64>(p, store, stream) : launch_d<T, 128>(p, store, stream);
}

}  // namespace

hipError_t launch_cache_rows(const CacheRowsParams &p, bool store, bool bf16, hipStream_t stream) {
    return bf16 ? launch_t<__bf16>(p, store, stream) : launch_t<float>(p, store, stream);
}

}  // namespace pi_attn
