// half_rows.h -- rows covered by a wavefront so that a lane holds both elements
// of a rotary pair: 16 bytes (or fewer, of a narrower type) from each half of
// the row, a row's lanes next to each other.
#pragma once

#include "decode_rows.h"

namespace pi_attn {

// T: the wide type, of which a lane holds EPL consecutive elements from each half.
template <typename T, int D>
struct HalfRow {
    static constexpr int EPL = 16 / (int)sizeof(T);
    static constexpr int LPR = D / 2 / EPL;           // lanes per row: 4, 8 or 16
    static constexpr int RPI = 64 / LPR;              // rows per load instruction
};

// Consecutive elements of one lane and half, as many bytes as their type takes.
template <typename T, int N>
struct alignas(sizeof(T) * N) Piece {
    unsigned w[sizeof(T) * N / 4];
};

template <typename T, int N, bool ONCE>
__device__ inline Piece<T, N> load_piece(const T *from) {
    Piece<T, N> r;
    constexpr int W = (int)sizeof(r) / 4;
    typedef unsigned vec __attribute__((ext_vector_type(W)));
    const vec x = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const vec *>(from))
                       : *reinterpret_cast<const vec *>(from);
#pragma unroll
    for (int i = 0; i < W; ++i) r.w[i] = x[i];
    return r;
}

template <typename T, int N, bool ONCE>
__device__ inline void store_piece(const Piece<T, N> &r, T *to) {
    constexpr int W = (int)sizeof(r) / 4;
    typedef unsigned vec __attribute__((ext_vector_type(W)));
    vec x;
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = r.w[i];
    if constexpr (ONCE) {
        __builtin_nontemporal_store(x, reinterpret_cast<vec *>(to));
    } else {
        *reinterpret_cast<vec *>(to) = x;
    }
}

template <typename T, int N>
__device__ inline void widen(const Piece<T, N> &r, float (&f)[N]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = __uint_as_float(r.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            f[2 * i] = __uint_as_float(r.w[i] << 16);
            f[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
        }
    }
}

template <typename T, int N>
__device__ inline Piece<T, N> narrowed(const float (&f)[N]) {
    Piece<T, N> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) r.w[i] = __float_as_uint(f[i]);
    } else {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const bf16x2 y = {(__bf16)f[2 * i], (__bf16)f[2 * i + 1]};
            r.w[i] = __builtin_bit_cast(unsigned, y);
        }
    }
    return r;
}

}  // namespace pi_attn
