// e4m3.h -- rows as the quantised caches hold them: D e4m3 codes (4 bits of
// exponent, 3 of mantissa, no infinities; largest 448) and one byte b, the
// scale 2^(b - 127).  With amax the row's largest finite magnitude, e = b - 127
// is the least integer from -126 on with amax <= 448 * 2^e, and the code of an
// element x is x * 2^-e rounded to the nearest, ties to even; an infinity or NaN
// is stored as NaN.  A scale that is a power of two costs no precision (a
// floating format's relative step does not depend on it) and makes every
// scaling exact: codes and bytes follow from the definition bit by bit, and a
// scale can be moved into a score, a weight or a rounded bf16 value without an
// error of its own.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pi_attn {

struct e4m3 {
    uint8_t code;
};

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr unsigned kInfBits = 0x7f800000u;

// The byte of a row from the bits of amax: 448 is 1.75 * 2^8, so a mantissa
// above 0x600000 (1.75) carries into the next exponent.
__device__ inline unsigned e4m3_byte(unsigned amax_bits) {
    return (unsigned)max((int)((amax_bits + 0x1fffffu) >> 23) - 8, 1);
}

__device__ inline float e4m3_scale(unsigned byte) { return __uint_as_float(byte << 23); }
__device__ inline float e4m3_inverse(unsigned byte) { return __uint_as_float((254u - byte) << 23); }

// The bits of |x|, 0 where x is not finite.
__device__ inline unsigned finite_bits(float x) {
    const unsigned a = __float_as_uint(x) & 0x7fffffffu;
    return a < kInfBits ? a : 0u;
}

// Four codes of x[0..3] * inv.
__device__ inline unsigned e4m3_pack4(const float *x, float inv) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = fabsf(x[i]) < INFINITY ? x[i] * inv : NAN;
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
}

// The values of four codes, without the scale.
__device__ inline void e4m3_unpack4(unsigned u, float *x) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, true);
    x[0] = lo.x;
    x[1] = lo.y;
    x[2] = hi.x;
    x[3] = hi.y;
}

}  // namespace pi_attn
