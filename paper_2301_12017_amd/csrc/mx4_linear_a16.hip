// Linear layers of few tokens: fp16 or bf16 activations as they are, weights in microscaled 4-bit floating point.
//
//   y[m,n] = act( sum_blocks 2^e[n,b] * sum_{k in b} w[n,k] x[m,k]  + bias[n] )
//
// A weight's 17/32 byte is read once for every 16 or 32 tokens, so the bytes of W bound a call of few.  Its codes become 16-bit numbers by a conversion instruction, two
// at a time and exact (the exponents stay out: they pass what fp16 holds); 32 of them are one matrix instruction, whose sums in
// fp32 go into the total with the block's power of two.
//
// A wave has some planes of K for itself.  It reads a plane of 16 channels as one kilobyte: a lane has a block, four words of eight codes.  The four lanes
// that share a channel change words (two lane swaps a pair), so that each instruction has one block of all 16 channels and a row of x is read 64 bytes
// at a time.  What is on its way is held in registers, two planes of it; the waves' sums are added up in LDS, in their order.
//
// What bounds it is how fast bytes come into a CU, its channels' codes and all of x: 42 KB a us by the constants of the tiles of 32 x 64 below, where a stream out of L2 reaches 110
// and more.  32 tokens 16000 x 4096 take 14 us, of whose 395 KB a workgroup 256 are x.  16 tokens 264 x 5504 take 6.9 us, 3.9 without the loads of x; leaving out conversion, exponents
// or products changes 2 to 7 %, and three or four planes on their way instead of two, or DMA into LDS instead of registers, were no faster.
#include "gemm_common.hpp"
#include "mx4.hpp"

namespace w4a4 {
namespace {

// words (lane group g, j) -> (lane group j, word g) for the four groups of sixteen lanes
__device__ __forceinline__ u32x4_t transpose_groups(u32x4_t w) {
    const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap((unsigned)a[0], (unsigned)b[0], false, false);
    const auto d = __builtin_amdgcn_permlane16_swap((unsigned)a[1], (unsigned)b[1], false, false);
    return u32x4_t{(unsigned)c[0], (unsigned)c[1], (unsigned)d[0], (unsigned)d[1]};
}

struct A16Args {
    const uint16_t *x;
    const uint8_t *w;
    const uint32_t *sw;
    const uint16_t *bias;
    uint16_t *out;
    int M, N, K, ldx, act, tiles_n;
};

template <bool BF16>
__device__ __forceinline__ u32x4_t numbers8(uint32_t w) {          // eight codes as 16-bit numbers
    u32x4_t o;
#define PAIR(J)                                                                                                                               \
    if constexpr (BF16) o[J] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, J));                           \
    else o[J] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, J));
    PAIR(0) PAIR(1) PAIR(2) PAIR(3)
#undef PAIR
    return o;
}

template <bool BF16, int MT, int NT, int NW, int AHEAD>
__global__ __launch_bounds__(NW * 64, NW / 4) void mx4_linear_a16_kernel(A16Args a) {
    extern __shared__ float red[];                                 // [NW][MT * NT * 4][64]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, kg = lane >> 4;
    const int m0 = blockIdx.x / a.tiles_n * (16 * MT), n0 = blockIdx.x % a.tiles_n * (16 * NT);
    const int planes = (a.K + kPlane - 1) / kPlane, each = (planes + NW - 1) / NW, c0 = wave * each, c1 = min(c0 + each, planes);
    struct Stage {
        u32x4_t w[NT], x[MT][4];
        uint32_t s[NT];
    } st[AHEAD];
    // Rows of x whose bytes at the same place lie in the same half of a cache line are read in turn, one its first 64 bytes of 128, the next its second
    // ones.  (All rows of a lane are alike: sixteen rows are a multiple of 128 bytes.)
    const int half = ((uint32_t)((reinterpret_cast<uintptr_t>(a.x) + (size_t)(m0 + col) * a.ldx * 2) >> 6) ^ (uint32_t)col) & 1 ? 32 : 0;
    // Everything comes through descriptors, outside of which zeros are read: rows of x behind the last one, their numbers behind K, planes of other waves.
    // (Loads under a condition would be waited for at once, where the two ways meet.)
    const __amdgpu_buffer_rsrc_t xr = make_rsrc(a.x + (size_t)m0 * a.ldx, (uint32_t)(((long)min(16 * MT, a.M - m0) - 1) * a.ldx + a.K) * 2);
    const int rows = min(16 * MT, a.M - m0), cols = min(16 * NT, a.N - n0);
    const int n = threadIdx.x % (16 * NT);                         // the channel of the results that the thread finishes
    const uint16_t bias = __builtin_amdgcn_raw_buffer_load_b16(make_rsrc(a.bias, a.bias ? (uint32_t)a.N * 2 : 0), (int)((uint32_t)(n0 + n) * 2), 0, 0);
    int xo[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) xo[t] = 16 * t + col < rows ? ((16 * t + col) * a.ldx + 8 * kg) * 2 : (int)kPoison;
    auto load = [&](Stage &s, int c) {
        const size_t at = (size_t)c * a.N + n0;
        const __amdgpu_buffer_rsrc_t w = make_rsrc(a.w + at * kPlaneBytes, c < c1 ? (uint32_t)cols * kPlaneBytes : 0), e = make_rsrc(a.sw + at, c < c1 ? (uint32_t)cols * 4 : 0);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            s.w[t] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(w, (16 * t + col) * kPlaneBytes + 16 * kg, 0, 0));
            s.s[t] = __builtin_amdgcn_raw_buffer_load_b32(e, (16 * t + col) * 4, 0, 0);
        }
        const int left = c < c1 ? a.K - c * kPlane : 0;
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = 32 * j ^ half;
                s.x[t][j] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(xr, k < left ? xo[t] + (c * kPlane + k) * 2 : (int)kPoison, 0, 0));
            }
    };
    float4_t tot[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) tot[i][t] = float4_t{0, 0, 0, 0};
    auto compute = [&](const Stage &s) {
        u32x4_t x[MT][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i][j][e] = half ? s.x[i][j ^ 1][e] : s.x[i][j][e];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const u32x4_t w4 = transpose_groups(s.w[t]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u32x4_t w = numbers8<BF16>(w4[j]);
                const float by = mx4_scale(s.s[t] >> (8 * j) & 255);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const float4_t sum = mfma16<BF16>(x[i][j], w, float4_t{0, 0, 0, 0});
#pragma unroll
                    for (int e = 0; e < 4; ++e) tot[i][t][e] = __fmaf_rn(sum[e], by, tot[i][t][e]);
                }
            }
            if (NT > 1) __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (c0 < c1) {
#pragma unroll
        for (int p = 0; p < AHEAD; ++p) load(st[p], c0 + p);
        for (int c = c0; c < c1; c += AHEAD) {
#pragma unroll
            for (int p = 0; p < AHEAD; ++p) {
                if (p == 0 || c + p < c1) compute(st[p]);
                load(st[p], c + p + AHEAD);                        // (zeros behind the last one)
            }
        }
    }
    constexpr int REGS = MT * NT * 4;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) red[(wave * REGS + (i * NT + t) * 4 + e) * 64 + lane] = tot[i][t][e];
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

template <bool BF16, int MT, int NT, int NW>
int launch(A16Args a, hipStream_t st) {
    auto kern = mx4_linear_a16_kernel<BF16, MT, NT, NW, 2>;
    constexpr size_t lds = (size_t)NW * MT * NT * 4 * 64 * sizeof(float);
    a.tiles_n = (int)(((long)a.N + 16 * NT - 1) / (16 * NT));
    const long tiles = (long)a.tiles_n * (((long)a.M + 16 * MT - 1) / (16 * MT));     // (mx4_way has asked whether they are a launch)
    static KernelState ks;
    if (prepare_kernel(reinterpret_cast<const void *>(kern), lds, ks) < 0) return W4A4_ERR_HIP;
    hipLaunchKernelGGL(kern, dim3((unsigned)tiles), dim3(NW * 64), lds, st, a);
    return launch_status();
}

// Tokens and channels of a tile, waves that share K.  Fitted to 200 sizes of 1 to 64 tokens each; over 200 with weights that no cache holds the choice is 2.2 % above the
// best of nine kinds, 32 % at worst.  us of the kinds in their order: one token 4096 x 4096 5.5, 4.8, ..; 32 tokens 16000 x 4096 (23 by the third), 20, 19, 32, 17; 64 tokens
// 32000 x 768 (28), 17, 22, 16, 22.
constexpr MX4Way kWays[] = {{16, 16, 256, 0, 2.405f, 0.114f, 0.099f, 0.224f, 0.0f}, {16, 16, 512, 0, 2.596f, 0.087f, 0.103f, 0.448f, 0.0f}, {16, 32, 512, 0, 2.743f, 0.129f, 0.143f, 0.756f, 0.0f},
                            {16, 64, 256, 0, 3.126f, 0.273f, 0.218f, 0.531f, 0.0f}, {16, 64, 512, 0, 3.301f, 0.206f, 0.229f, 1.126f, 0.0f}, {32, 64, 128, 0, 3.390f, 0.808f, 0.293f, 1.070f, 0.0f},
                            {32, 64, 512, 0, 3.698f, 0.296f, 1.413f, 0.000f, 0.0f}};

template <bool BF16>
int pick(const A16Args &a, hipStream_t st) {
    constexpr int ways = (int)(sizeof(kWays) / sizeof(kWays[0]));
    if (!mx4_any_launches(kWays, ways, a.M, a.N)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    static KernelState ks;
    const int cus = prepare_kernel(reinterpret_cast<const void *>(mx4_linear_a16_kernel<BF16, 1, 1, 8, 2>), 0, ks);
    if (cus < 0) return W4A4_ERR_HIP;
    switch (mx4_way(kWays, ways, a.M, a.N, mx4_planes(a.K), a.act, cus)) {
        case 0: return launch<BF16, 1, 1, 4>(a, st);
        case 1: return launch<BF16, 1, 1, 8>(a, st);
        case 2: return launch<BF16, 1, 2, 8>(a, st);
        case 3: return launch<BF16, 1, 4, 4>(a, st);
        case 4: return launch<BF16, 1, 4, 8>(a, st);
        case 5: return launch<BF16, 2, 4, 2>(a, st);
        default: return launch<BF16, 2, 4, 8>(a, st);
    }
}

}  // namespace
}  // namespace w4a4

using namespace w4a4;

extern "C" int w4a4_mx4_linear_a16(const void *X, int dtype, int M, int ldx, const w4a4_mx4 *W, const void *bias, int act, void *out, void *stream) {
    if (const int rc = mx4_check(W)) return rc;
    if (M < 0 || ldx < W->K || W->rows == 0 || (dtype != W4A4_F16 && dtype != W4A4_BF16) || (act != W4A4_ACT_NONE && act != W4A4_ACT_GELU)) return W4A4_ERR_INVALID_ARG;
    if (M == 0) return W4A4_OK;
    if (!X || !out) return W4A4_ERR_INVALID_ARG;
    if (W->rows % 8 || ldx % 8 || ldx >= 1 << 24 || !aligned16(X) || !aligned16(out) || (bias && !aligned16(bias))) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const A16Args a{static_cast<const uint16_t *>(X), W->q, W->scale, static_cast<const uint16_t *>(bias), static_cast<uint16_t *>(out), M, W->rows, W->K, ldx, act, 0};
    return dtype == W4A4_BF16 ? pick<true>(a, as_stream(stream)) : pick<false>(a, as_stream(stream));
}
