// Rotation of pairs of features by a token's position (gfx950): angles, and a pair turned.
//
// A pair turns by `position * frequency`, and only the fraction of a turn counts.  Frequencies are 64-bit fractions of a turn (2^-64 units), so the
// product with a position, its low 64 bits kept, is that fraction with nothing lost but the frequency's own rounding: position * 2^-65 turns,
// 2^-34 for the last position there is.  The top 32 bits, the nearest quarter turn taken off, are an angle of at most pi / 4 in fp32 (half
// a unit is 7e-10), and the Taylor series of sine and cosine around 0 up to x^9 and x^10 are within 2e-9 of them: an error of 2^-24 of the pair's length.
#pragma once
#include "gen.hpp"

namespace w4a4 {

struct RotaryArgs {
    const uint64_t *turns;                                         // [pairs]
    int pairs, interleaved;
    float magnitude;                                               // negative sines: the inverse
    int inverse;
};

struct Turn { float cos, sin; };

__device__ __forceinline__ Turn turn_of(uint64_t per, uint32_t position, float magnitude, int inverse) {
    const uint32_t f = (uint32_t)((per * position) >> 32);
    const uint32_t quarter = (f + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(f - (quarter << 30)) * 1.4629180792671596e-09f;   // 2 pi / 2^32
    const float z = x * x;
    float s = __fmaf_rn(z, 2.7557319224e-06f, -1.9841269841e-04f);                      // 1/9!, 1/7!
    s = __fmaf_rn(s, z, 8.3333333333e-03f);
    s = __fmaf_rn(s, z, -1.6666666667e-01f);
    s = __fmaf_rn(s * z, x, x);
    float c = __fmaf_rn(z, -2.7557319224e-07f, 2.4801587302e-05f);                      // 1/10!, 1/8!
    c = __fmaf_rn(c, z, -1.3888888889e-03f);
    c = __fmaf_rn(c, z, 4.1666666667e-02f);
    c = __fmaf_rn(c, z, -0.5f);
    c = __fmaf_rn(c, z, 1.0f);
    const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
    Turn t;
    t.cos = (((quarter + 1) & 2) ? -a : a) * magnitude;
    t.sin = (((quarter & 2) != 0) != (inverse != 0) ? -b : b) * magnitude;
    return t;
}
__device__ __forceinline__ float turned_a(Turn t, float a, float b) { return __fmaf_rn(a, t.cos, -(b * t.sin)); }
__device__ __forceinline__ float turned_b(Turn t, float a, float b) { return __fmaf_rn(b, t.cos, a * t.sin); }

// W4A4_OK, or what is wrong with a plan of angles for heads of `features`.
inline int rotary_check(const w4a4_rotary_angles *R, int features) {
    if (!R || !R->turns || R->pairs <= 0 || 2 * (long)R->pairs > features || !(R->magnitude > 0.0f) || !(R->magnitude < INFINITY)) return W4A4_ERR_INVALID_ARG;
    if ((R->interleaved != 0 && R->interleaved != 1) || (R->inverse != 0 && R->inverse != 1)) return W4A4_ERR_INVALID_ARG;
    return reinterpret_cast<uintptr_t>(R->turns) & 7 ? W4A4_ERR_UNSUPPORTED_SHAPE : W4A4_OK;
}
inline RotaryArgs rotary_args(const w4a4_rotary_angles *R) { return RotaryArgs{R->turns, R->pairs, R->interleaved, R->magnitude, R->inverse}; }

// out[t, h, :] = x[t, h, :] turned by positions[t]; arguments checked by the caller (rotary.hip).
int rotary_launch(const void *x, int dtype, int tokens, int heads, int features, long ldx, const int32_t *positions, const RotaryArgs &r, void *out, long ldo, hipStream_t st);

}  // namespace w4a4
