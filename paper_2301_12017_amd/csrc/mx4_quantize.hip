// Rows of 16-bit numbers to microscaled 4-bit floating point, and back.
//
//   E = min(max(floor(log2(max |x|)) - 2, -127), 127)   of 32 neighbours      code = x / 2^E at the nearest E2M1 number, ties to even
//
// The largest magnitude lies in [4, 8) units then; what passes 6 becomes 6.  The exponent of a 16-bit number is a field of its bits
// (of its fp32 form for fp16, whose subnormal numbers are normal there), so nothing is computed to find E, and dividing by a power of two rounds
// nothing: codes are the definition's bit for bit.  The conversion instruction divides, rounds and saturates by itself, two numbers a time.
//
// Four lanes have a block, eight numbers each: sixteen bytes in, four out, both consecutive over a wave.  A wave takes four rows (one where
// there are few) of 512 numbers, so that a lane of sixteen has four rows' scale words, which lie together.
//
// Memory bounds it: 12288 x 4096 25 us = 5.1 TB/s of 127 MB (eight rows a wave, or loads and stores past the caches: slower), back 20.6.
#include "mx4.hpp"

namespace w4a4 {
namespace {

struct QuantArgs {
    const uint16_t *x;
    uint8_t *q;
    uint32_t *scale;
    int rows, K;
    long ldx;
};

template <bool BF16>
__device__ __forceinline__ uint32_t quantize8(u32x4_t w, uint32_t &byte) {
    // largest magnitude of the block, as bits
    typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));
    ushort2_t m = {0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(ushort2_t, w[j] & 0x7FFF7FFFu));
    uint32_t most = max((uint32_t)m[0], (uint32_t)m[1]);
    most = max(most, dpp_fetch<0xB1>(most));
    most = max(most, dpp_fetch<0x4E>(most));
    const bool bad = most >= (BF16 ? 0x7F80u : 0x7C00u);           // an infinity or a NaN: the block is NaN
    const int e = (int)(__builtin_bit_cast(uint32_t, to_float<BF16>((uint16_t)most)) >> 23) - 2;
    byte = bad ? 255u : (uint32_t)max(e, 0);
    const float by = __builtin_bit_cast(float, byte << 23);        // (the instruction reads the exponent's field alone; 0 is 2^-127)
    uint32_t c = 0;
    const uint32_t x[4] = {w[0], w[1], w[2], w[3]};                // (a bit cast of a vector's element takes its first one)
#define PAIR(J)                                                                                                                               \
    if constexpr (BF16) c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x[J]), by, J);                          \
    else c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(half2_t, x[J]), by, J);
    PAIR(0) PAIR(1) PAIR(2) PAIR(3)
#undef PAIR
    return bad ? 0u : c;
}

// R rows of a wave, 512 numbers of each.
template <bool BF16, int R>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(QuantArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int cols = (a.K + 511) / 512;                            // workgroups of a row of them follow each other
    const long r0 = ((long)(blockIdx.x / cols) * 4 + wave) * R;
    const int k = blockIdx.x % cols * 512 + lane * 8, c = k / kPlane, planes = (a.K + kPlane - 1) / kPlane;
    if (r0 >= a.rows || c >= planes) return;                       // (sixteen lanes together)
    u32x4_t w[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        w[i] = u32x4_t{0, 0, 0, 0};
        if (k < a.K && r0 + i < a.rows) w[i] = *reinterpret_cast<const u32x4_t *>(a.x + (r0 + i) * a.ldx + k);
    }
    uint32_t words[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        uint32_t byte;
        const uint32_t codes = quantize8<BF16>(w[i], byte);
        uint32_t s = k < a.K ? byte << (8 * (lane >> 2 & 3)) : 0u; // the same in the four lanes of a block
        s |= dpp_fetch<0x141>(s);                                  // half-row mirror: blocks 0 and 1, 2 and 3
        s |= dpp_fetch<0x140>(s);                                  // row mirror: the two halves
        words[i] = s;
        if (r0 + i < a.rows) *reinterpret_cast<uint32_t *>(a.q + ((long)c * a.rows + r0 + i) * kPlaneBytes + k % kPlane / 2) = codes;
    }
    if ((lane & 15) == 0) {
        uint32_t *to = a.scale + (long)c * a.rows + r0;
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (r0 + i < a.rows) to[i] = words[i];
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t *q, const uint32_t *scale, int rows, int K, uint16_t *x) {
    constexpr int R = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int cols = (K + 511) / 512;
    const long r0 = ((long)(blockIdx.x / cols) * 4 + wave) * R;
    const int k = blockIdx.x % cols * 512 + lane * 8, c = k / kPlane;
    if (r0 >= rows || k >= K) return;
    uint32_t codes[R], s[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const long at = (long)c * rows + min(r0 + i, (long)rows - 1);
        codes[i] = *reinterpret_cast<const uint32_t *>(q + at * kPlaneBytes + k % kPlane / 2);
        s[i] = scale[at];
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (r0 + i >= rows) break;
        const float by = mx4_scale(s[i] >> (8 * (lane >> 2 & 3)) & 255);
        u32x4_t o;
#define PAIR(J)                                                                                                                               \
    {                                                                                                                                         \
        const v2f_t v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], 1.0f, J);                                                          \
        o[J] = from_float<BF16>(v[0] * by) | (uint32_t)from_float<BF16>(v[1] * by) << 16;                                                     \
        o[J] |= (codes[i] >> (8 * J) & 0x08u) << 12 | (codes[i] >> (8 * J) & 0x80u) << 24;      /* (the conversion loses a zero's sign) */     \
    }
        PAIR(0) PAIR(1) PAIR(2) PAIR(3)
#undef PAIR
        *reinterpret_cast<u32x4_t *>(x + (r0 + i) * K + k) = o;
    }
}

}  // namespace
}  // namespace w4a4

using namespace w4a4;

extern "C" int w4a4_mx4_quantize(const void *X, int dtype, int ldx, const w4a4_mx4 *out, void *stream) {
    if (const int rc = mx4_check(out)) return rc;
    if ((dtype != W4A4_F16 && dtype != W4A4_BF16) || ldx < out->K) return W4A4_ERR_INVALID_ARG;
    if (out->rows == 0) return W4A4_OK;
    if (!X) return W4A4_ERR_INVALID_ARG;
    if (ldx % 8 || !aligned16(X)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const QuantArgs a{static_cast<const uint16_t *>(X), out->q, out->scale, out->rows, out->K, ldx};
    const int cols = (a.K + 511) / 512;
    const bool few = (long)a.rows * cols < 4096;
    const int per = few ? 4 : 16;                                  // rows of a workgroup (us by 4 | 16: 3 x 1024 1.9 | 2.1, 512 x 4096 2.4 | 2.5, 12288 x 4096 26 | 25)
    const long groups = ((long)a.rows + per - 1) / per * cols;
    if (!grid_fits(groups, 256)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const dim3 grid((unsigned)groups);
    auto run = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, as_stream(stream), a); };
    if (dtype == W4A4_BF16) few ? run(mx4_quantize_kernel<true, 1>) : run(mx4_quantize_kernel<true, 4>);
    else few ? run(mx4_quantize_kernel<false, 1>) : run(mx4_quantize_kernel<false, 4>);
    return launch_status();
}

extern "C" int w4a4_mx4_dequantize(const w4a4_mx4 *Q, int dtype, void *X, void *stream) {
    if (const int rc = mx4_check(Q)) return rc;
    if (dtype != W4A4_F16 && dtype != W4A4_BF16) return W4A4_ERR_INVALID_ARG;
    if (Q->rows == 0) return W4A4_OK;
    if (!X) return W4A4_ERR_INVALID_ARG;
    const long groups = ((long)Q->rows + 15) / 16 * ((Q->K + 511) / 512);
    if (!aligned16(X) || !grid_fits(groups, 256)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const dim3 grid((unsigned)groups);
    auto run = [&](auto kern) {
        hipLaunchKernelGGL(kern, grid, dim3(256), 0, as_stream(stream), Q->q, Q->scale, Q->rows, Q->K, static_cast<uint16_t *>(X));
    };
    if (dtype == W4A4_BF16) run(mx4_dequantize_kernel<true>);
    else run(mx4_dequantize_kernel<false>);
    return launch_status();
}
