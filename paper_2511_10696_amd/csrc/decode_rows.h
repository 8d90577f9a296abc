// decode_rows.h -- how the decode kernels cover rows with a wavefront: 16-byte
// pieces of consecutive rows, a row's lanes next to each other.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pi_attn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned raw16 __attribute__((ext_vector_type(4)));

template <typename T, int D>
struct Row {
    static constexpr int EPL = 16 / (int)sizeof(T);   // elements per lane
    static constexpr int LPR = D / EPL;               // lanes per row
    static constexpr int RPI = 64 / LPR;              // rows per load instruction
};

__device__ inline uint4 ld16(const void *p) { return *reinterpret_cast<const uint4 *>(p); }

// A load that does not keep its line in the caches.
__device__ inline uint4 ld16_once(const void *p) {
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const raw16 *>(p)));
}

template <typename T>
__device__ inline void to_f32(uint4 u, float (&f)[16 / sizeof(T)]) {
    if constexpr (sizeof(T) == 2) {
        const bf16x8 b = __builtin_bit_cast(bf16x8, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)b[i];
    } else {
        const f32x4 b = __builtin_bit_cast(f32x4, u);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = b[i];
    }
}

// Sum over the LPR lanes of a row, left in each of them: xor 1 and 2 inside
// quads, the mirrored half-row (8 lanes), the mirrored row (16), then the
// neighbouring row (32).
template <int LPR>
__device__ inline float row_sum(float x) {
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xF, 0xF, false));
    x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xF, 0xF, false));
    if constexpr (LPR >= 8) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xF, 0xF, false));
    if constexpr (LPR >= 16) x += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x140, 0xF, 0xF, false));
    if constexpr (LPR >= 32) x += __shfl_xor(x, 16);
    return x;
}

// The largest of the LPR lanes' whole numbers, the same way.
template <int LPR>
__device__ inline unsigned row_max(unsigned x) {
    x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, false));
    x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, false));
    if constexpr (LPR >= 8) x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xF, 0xF, false));
    if constexpr (LPR >= 16) x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xF, 0xF, false));
    if constexpr (LPR >= 32) x = max(x, (unsigned)__shfl_xor((int)x, 16));
    return x;
}

}  // namespace pi_attn
