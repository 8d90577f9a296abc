// rotary.h -- rotary positions: pair i < P of a row, its elements i and i + D/2,
// is turned by the angle pos_a * freq_i, a the axis that the pair belongs to
// (one, or up to three: time, height and width); pairs from P on stay as they
// are.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pi_attn {

// pos == nullptr: the position of a row in its sequence, on every axis.
struct Rotary {
    const float *freq;              // [pairs], radians a position; nullptr: no rotation
    int pairs, end0, end1;          // axis 0 has pairs [0, end0), axis 1 [end0, end1), axis 2 the rest
    const int32_t *pos;
    int64_t psa, psb, psn;          // its element strides: axis, sequence, row
};

// cos and sin of pos * freq.  The angle is formed in turns and in 64 bits.  For |freq| <= 1
// and |pos| < 2^31 it is off by less than 2^-23 of a turn: 2^-25.5 by the constant (off by
// 2^-56.5), 2^-25 by its product with freq, 2^-25 by the turns (up to 2^28.4); up to a
// million positions 2^-34.  In 32 bits a position of 2^20 would be off by a hundredth of a
// turn.
__device__ inline float2 cos_sin(int pos, float freq) {
    constexpr double kTurns = 0.15915494309189535;   // 1 / (2 pi)
    const double turns = (double)pos * ((double)freq * kTurns);
    const float x = 2.0f * (float)(turns - __builtin_rint(turns));
    float s, c;
    sincospif(x, &s, &c);
    return make_float2(c, s);
}

// What pair i at row n of sequence b is turned by, once asked for (0 beyond the last
// pair), where the row is position `at` of its sequence.
struct Angle {
    float freq;
    int pos;
};
__device__ inline Angle angle_of(const Rotary &r, int i, int64_t b, int64_t n, int at) {
    if (!r.freq || i >= r.pairs) return Angle{0.0f, 0};
    const int axis = i < r.end0 ? 0 : i < r.end1 ? 1 : 2;
    return Angle{r.freq[i], r.pos ? r.pos[axis * r.psa + b * r.psb + n * r.psn] : at};
}
__device__ inline float2 cos_sin_of(const Rotary &r, int i, int64_t b, int64_t n, int at) {
    const Angle a = angle_of(r, i, b, n, at);
    return cos_sin(a.pos, a.freq);
}

// A pair (a, b) turned; pairs from r.pairs on are not touched, whatever they hold.
__device__ inline void turn(float &a, float &b, float2 cs, bool turned) {
    const float x = a * cs.x - b * cs.y, y = a * cs.y + b * cs.x;
    a = turned ? x : a;
    b = turned ? y : b;
}

}  // namespace pi_attn
