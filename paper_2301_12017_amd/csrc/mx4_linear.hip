// Linear layers whose operands are both microscaled 4-bit floating point.
//
//   y[m,n] = act( sum_blocks 2^(ea[m,b] + ew[n,b]) * sum_{k in b} a[m,k] w[n,k]  + bias[n] )
//
// The matrix instruction takes codes and exponents as they are: 128 numbers of 16 rows, a lane one block of one row, sixteen bytes of codes
// and a byte of exponent.  A plane's rows follow each other, so such an operand is a kilobyte of consecutive memory.
//
// This file's kernel takes what has too few tiles for the one in LDS (mx4_tiles.hip): a chain of first loads, a product, a sum over eight waves.  5 tokens
// 1024 x 1024 2.7 us, of which a launch is 2.1.
#include "mx4.hpp"
#include "mx4_linear.hpp"

namespace w4a4 {
namespace {

__device__ __forceinline__ v8i_t operand(u32x4_t x) { return v8i_t{(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0}; }

// Few tokens: MT x NT tiles of 16 x 16, the waves of a workgroup have a part of K each and add up in LDS, in their order.
template <bool BF16, int MT, int NT, int NW>
__global__ __launch_bounds__(NW * 64) void mx4_linear_few_kernel(MX4LinearArgs a) {
    extern __shared__ float red[];                                 // [NW][MT * NT * 4][64]
    constexpr int AHEAD = 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, kg = lane >> 4;
    const int m0 = blockIdx.x / a.tiles_n * (16 * MT), n0 = blockIdx.x % a.tiles_n * (16 * NT);
    const int each = (a.planes + NW - 1) / NW, c0 = wave * each, c1 = min(c0 + each, a.planes);
    const int rows = min(16 * MT, a.M - m0), cols = min(16 * NT, a.N - n0);
    const int n = threadIdx.x % (16 * NT);                         // the channel of the results that the thread finishes
    const uint16_t bias = a.bias ? a.bias[min(n0 + n, a.N - 1)] : 0;
    struct Stage {
        u32x4_t x[MT], w[NT];
        uint32_t sx[MT], sw[NT];
    } st[AHEAD];
    auto load = [&](Stage &s, int c) {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const size_t at = (size_t)c * a.M + min(m0 + 16 * t + row, a.M - 1);
            s.x[t] = *reinterpret_cast<const u32x4_t *>(a.a + at * kPlaneBytes + 16 * kg);
            s.sx[t] = a.sa[at];
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const size_t at = (size_t)c * a.N + min(n0 + 16 * t + row, a.N - 1);
            s.w[t] = *reinterpret_cast<const u32x4_t *>(a.w + at * kPlaneBytes + 16 * kg);
            s.sw[t] = a.sw[at];
        }
    };
    float4_t acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = float4_t{0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < AHEAD; ++p)
        if (c0 + p < c1) load(st[p], c0 + p);
    for (int c = c0; c < c1; c += AHEAD) {
#pragma unroll
        for (int p = 0; p < AHEAD; ++p) {
            if (c + p >= c1) break;
            Stage &s = st[p];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    acc[i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(s.x[i]), operand(s.w[t]), acc[i][t], 4, 4, 0, (int)(s.sx[i] >> (8 * kg)), 0,
                                                                                 (int)(s.sw[t] >> (8 * kg)));
            if (c + p + AHEAD < c1) load(s, c + p + AHEAD);
        }
    }
    constexpr int REGS = MT * NT * 4;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) red[(wave * REGS + (i * NT + t) * 4 + e) * 64 + lane] = acc[i][t][e];
    __syncthreads();
    if (n >= cols) return;
    for (int m = threadIdx.x / (16 * NT); m < rows; m += NW * 64 / (16 * NT)) {
        const int reg = ((m >> 4) * NT + (n >> 4)) * 4 + (m & 3), from = ((m & 15) >> 2) * 16 + (n & 15);
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) y += red[(w * REGS + reg) * 64 + from];
        a.out[(size_t)(m0 + m) * a.N + n0 + n] = mx4_result<BF16>(y + to_float<BF16>(bias), a.act == W4A4_ACT_GELU);
    }
}

// The constants are fitted to 90 to 178 sizes each, of 1 to 20000 tokens; over 215 sizes the choice is 2.4 % above the best, 28 % at worst.
// (us of 16384 x 16384 x 1024 without GELU | with it, from 64 x 128 on: 254 | 292, 202 | 241, 195 | 229, 205 | 264.)
constexpr int kFew = 3;                                            // the first of them are this file's, the others an MX4Tile each
constexpr MX4Way kWays[] = {{16, 16, 512, 0, 1.99f, 0.042f, 0.041f, 0.205f, 0.00f},
                            {16, 32, 512, 0, 2.10f, 0.056f, 0.061f, 0.551f, 0.00f},
                            {32, 32, 512, 0, 2.26f, 0.070f, 0.079f, 0.820f, 0.00f},
                            {64, 64, 512, 1, 4.11f, 0.100f, 0.114f, 3.401f, 0.10f},
                            {64, 128, 256, 4, 2.75f, 0.267f, 0.147f, 0.932f, 0.28f},
                            {128, 128, 256, 3, 3.28f, 0.288f, 0.198f, 2.149f, 0.60f},
                            {128, 256, 256, 2, 4.16f, 0.454f, 0.399f, 3.798f, 1.40f},
                            {256, 256, 512, 1, 5.85f, 0.625f, 0.851f, 9.643f, 3.50f, true}};

template <bool BF16, int MT, int NT, int NW>
int launch_few(MX4LinearArgs a, hipStream_t st) {
    auto kern = mx4_linear_few_kernel<BF16, MT, NT, NW>;
    constexpr size_t lds = (size_t)NW * MT * NT * 4 * 64 * sizeof(float);
    a.tiles_n = (int)(((long)a.N + 16 * NT - 1) / (16 * NT));
    const long tiles = (long)a.tiles_n * (((long)a.M + 16 * MT - 1) / (16 * MT));     // (mx4_way has asked whether they are a launch)
    hipLaunchKernelGGL(kern, dim3((unsigned)tiles), dim3(NW * 64), lds, st, a);
    return launch_status();
}

template <bool BF16>
int pick(const MX4LinearArgs &a, hipStream_t st) {
    // (the tiles in LDS have 32-bit offsets into a row of tiles' results)
    const int ways = a.N < 1 << 22 ? (int)(sizeof(kWays) / sizeof(kWays[0])) : kFew;
    if (!mx4_any_launches(kWays, ways, a.M, a.N)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    static KernelState ks;
    const int cus = prepare_kernel(reinterpret_cast<const void *>(mx4_linear_few_kernel<BF16, 1, 1, 8>), 0, ks);
    if (cus < 0) return W4A4_ERR_HIP;
    const int way = mx4_way(kWays, ways, a.M, a.N, a.planes, a.act, cus);
    switch (way) {
        case 0: return launch_few<BF16, 1, 1, 8>(a, st);
        case 1: return launch_few<BF16, 1, 2, 8>(a, st);
        case 2: return launch_few<BF16, 2, 2, 8>(a, st);
        default: return mx4_tiles(a, BF16 ? W4A4_BF16 : W4A4_F16, static_cast<MX4Tile>(way - kFew), st);
    }
}

}  // namespace
}  // namespace w4a4

using namespace w4a4;

extern "C" int w4a4_mx4_linear(const w4a4_mx4 *A, const w4a4_mx4 *W, const void *bias, int act, int dtype, void *out, void *stream) {
    if (const int rc = mx4_check(A)) return rc;
    if (const int rc = mx4_check(W)) return rc;
    if (A->K != W->K || W->rows == 0 || (dtype != W4A4_F16 && dtype != W4A4_BF16) || (act != W4A4_ACT_NONE && act != W4A4_ACT_GELU)) return W4A4_ERR_INVALID_ARG;
    if (A->rows == 0) return W4A4_OK;
    if (!out) return W4A4_ERR_INVALID_ARG;
    if (W->rows % 8 || !aligned16(out) || (bias && !aligned16(bias))) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const MX4LinearArgs a{A->q, W->q, A->scale, W->scale, static_cast<const uint16_t *>(bias), static_cast<uint16_t *>(out), A->rows, W->rows, mx4_planes(A->K), act, 0, 0, 0};
    return dtype == W4A4_BF16 ? pick<true>(a, as_stream(stream)) : pick<false>(a, as_stream(stream));
}
