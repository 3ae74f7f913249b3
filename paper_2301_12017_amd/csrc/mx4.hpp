// What the kernels of microscaled 4-bit floating point share (gfx950).
//
// A number is E2M1 (sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6) times a power of two that it shares with 31
// neighbours of its row.  Planes of 128 numbers: 64 bytes of codes and one word of four exponents (plus 127) for each row.
#pragma once
#include "gen.hpp"

namespace w4a4 {

typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float v2f_t __attribute__((ext_vector_type(2)));

constexpr int kPlane = 128;                                        // numbers of a row in a plane
constexpr int kPlaneBytes = 64;

inline int mx4_planes(int K) { return (K + kPlane - 1) / kPlane; }

// 2^(e - 127) for the byte e; NaN for 255.
__device__ __forceinline__ float mx4_scale(uint32_t e) {
    const uint32_t bits = e ? e << 23 : 0x00400000u;
    return __builtin_bit_cast(float, e == 255 ? 0x7FC00000u : bits);
}

// GELU for bf16 results, max(x, 0) - |x| Phi(-|x|).  A bf16 number has fp32's range, so that Phi counts relatively all the way to where it ends, not to fp16's last number:
// log2 Phi(-t) is a polynomial of degree 9 in t, fitted evenly to [0, 13.35] (3.3e-5, or 2.3e-5 of Phi).  Its fp32 steps add 5.0e-5 at most (half a step of each
// partial sum, at the t behind it), measured 4.3e-5 of GELU in all: 8e-5, a 24th of the smallest half step of bf16, wherever |GELU| is 2^-122 or more.  Below that Phi leaves fp32's normal
// numbers, and the result may be 0.  Behind 13.3 the polynomial falls on, and x's own size times 2^-inf is 0: x needs no clamp.  (fp16's form, degree 5, is off by 0.3 % at -5 and
// 14 % at -7; the four steps more take 16384 x 16384 x 1024 from 226 to 239 us, 12288 x 4096 x 1024 from 54 to 57.)
__device__ __forceinline__ float mx4_gelu_bf16(float x) {
    const float t = fabsf(x);
    float q = -1.858528553e-09f;
    q = __fmaf_rn(q, t, 1.366808533e-07f);
    q = __fmaf_rn(q, t, -4.417262062e-06f);
    q = __fmaf_rn(q, t, 8.302903734e-05f);
    q = __fmaf_rn(q, t, -1.016221242e-03f);
    q = __fmaf_rn(q, t, 8.645871654e-03f);
    q = __fmaf_rn(q, t, -5.390371382e-02f);
    q = __fmaf_rn(q, t, -4.588583112e-01f);
    q = __fmaf_rn(q, t, -1.150948524e+00f);
    q = __fmaf_rn(q, t, -1.000032663e+00f);
    return __fmaf_rn(-t, __builtin_amdgcn_exp2f(q), __int_as_float(max(__float_as_int(x), 0)));
}

// GELU of two finite sums as 16-bit numbers; fp16 by the form of the library's fp16 stores (9e-5 of what is a normal number of fp16).
template <bool BF16>
__device__ __forceinline__ uint32_t mx4_gelu2(float a, float b) {
    if constexpr (BF16) return from_float<true>(mx4_gelu_bf16(a)) | (uint32_t)from_float<true>(mx4_gelu_bf16(b)) << 16;
    else return gelu_erf_half2(a, b);
}
// ... of a sum that is an infinity or a NaN (which that form makes NaN of)
__device__ __forceinline__ float mx4_gelu_limit(float y) { return y < 0.0f ? 0.0f : y; }

// A sum as it is stored, GELU applied where asked for.
template <bool BF16>
__device__ __forceinline__ uint16_t mx4_result(float y, bool gelu) {
    if (!gelu) return from_float<BF16>(y);
    return fabsf(y) < INFINITY ? (uint16_t)mx4_gelu2<BF16>(y, y) : from_float<BF16>(mx4_gelu_limit(y));
}

// Tiles of a product.  A problem of M x N and `planes` of K takes about  start + plane * planes + (more * planes + tile) * (tiles / CUs - 1, not below 0)  us
// by tiles of one kind: small ones bring the operands of a small problem to more CUs (42 to 52 KB a us come into a CU by the constants, whatever is asked for at once), large ones
// bring less in all.  Past the `held` tiles of a CU the count lies halfway between tiles and whole rounds of them.
// A kind whose workgroups are more than a launch takes is none.
struct MX4Way {
    int bm, bn, threads, held;                                     // threads: of a workgroup; held: by a CU at once; 0: not counted in rounds
    float start, plane, more, tile, gelu;                          // gelu: more of `tile` where there is one
    bool tail;                                                     // a last round of up to a quarter is taken in quarters of tiles
};
inline long mx4_way_tiles(const MX4Way &w, int M, int N) { return (((long)M + w.bm - 1) / w.bm) * (((long)N + w.bn - 1) / w.bn); }
inline bool mx4_launches(const MX4Way &w, int M, int N) { return grid_fits(mx4_way_tiles(w, M, N), w.threads); }
inline bool mx4_any_launches(const MX4Way *ways, int count, int M, int N) {
    for (int i = 0; i < count; ++i)
        if (mx4_launches(ways[i], M, N)) return true;
    return false;
}
inline int mx4_way(const MX4Way *ways, int count, int M, int N, int planes, int act, int cus) {
    int best = -1;
    float least = INFINITY;
    for (int i = 0; i < count; ++i) {
        const MX4Way &w = ways[i];
        if (!mx4_launches(w, M, N)) continue;
        const long tiles = mx4_way_tiles(w, M, N), left = tiles % cus;
        float r = (float)tiles / (float)cus;
        if (w.held && r > (float)w.held) {
            const long round = (long)w.held * cus, rounds = (tiles + round - 1) / round;
            r = w.tail && 4 * left <= cus ? (float)(tiles / cus) + (left ? 0.4f : 0.0f) : 0.5f * (r + (float)(rounds * w.held));
        }
        const float us = w.start + w.plane * (float)planes + (r > 1.0f ? (w.more * (float)planes + w.tile + (act == W4A4_ACT_GELU ? w.gelu : 0.0f)) * (r - 1.0f) : 0.0f);
        if (us < least) least = us, best = i;
    }
    return best;
}

// W4A4_OK, or what is wrong with an operand.
inline int mx4_check(const w4a4_mx4 *Q) {
    if (!Q || Q->rows < 0 || Q->K <= 0) return W4A4_ERR_INVALID_ARG;
    if (Q->rows && (!Q->q || !Q->scale)) return W4A4_ERR_INVALID_ARG;
    if (Q->K % 32 || Q->K > 1 << 30 || !aligned16(Q->q) || (reinterpret_cast<uintptr_t>(Q->scale) & 3)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    return W4A4_OK;
}

}  // namespace w4a4
