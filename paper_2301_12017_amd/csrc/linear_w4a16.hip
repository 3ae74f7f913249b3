// Linear layers of few tokens: fp16 or bf16 activations times 4-bit weights (token generation).
//
//   y[m,n] = act( sum_g scale[n,g] * sum_{k in g} c[n,k] x[m,k]  (+ zero[n,g] * sum_{k in g} x[m,k])  + bias[n] )
//
// A weight is read once, four bits of it, so the bytes of W bound the call.  The codes become operands of the 16-bit matrix
// instruction without an arithmetic conversion: u = code (unsigned) or code + 8 (symmetric; the top bit of the nibble flipped) is
//   fp16: the bit pattern itself, a subnormal number u * 2^-24 (the matrix instruction takes those; 2^24 goes into the scale);
//   bf16: the pattern 0x4300 | u, the number 128 + u.
// Products with them are exact and summed in fp32.  What is added to the codes (8, 128, 136) leaves again by a matrix instruction
// whose other operand is that constant, negative: its result is where the sum of the products begins, so that the sum
// does not have to cancel it later; it is one instruction for all tiles of channels.  Sums go into the fp32 total at the end of
// a group, and every 128 codes at the latest: with the offset in them they are up to 50 times larger than the result.
//
// A wave holds NT tiles of 16 channels x MT of 16 tokens and reads chunks of 128 codes of K, 16 bytes (32 codes) a lane, straight
// into registers; the waves of a workgroup take turns over K and add up through LDS.  The order of K inside an instruction
// is free as long as both operands agree: (w >> 4j) & 0x000F000F gives codes j and j + 4 of a word, so the pairs of x are
// put in that order.  Groups that are not whole chunks (32, 64, 96, ...): the four words of the four lanes that share a row
// change places (two lane swaps a pair), so that each instruction reads 32 consecutive codes and a sum never crosses a group.
#include "gen.hpp"

namespace w4a4 {
namespace {

struct W4A16Args {
    const uint16_t *x;
    const uint8_t *q;
    const float *scale, *zero;
    const uint16_t *bias;
    uint16_t *out;
    int M, N, K, ldx, group, ng, act;
};

// x0 .. x7 as (x0,x4), (x1,x5), (x2,x6), (x3,x7)
__device__ __forceinline__ u32x4_t pair_up(u32x4_t x) {
    return u32x4_t{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
                   __builtin_amdgcn_perm(x[3], x[1], 0x05040100u), __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
}

// words (lane group g, j) -> (lane group j, word g) for the four groups of sixteen lanes
__device__ __forceinline__ u32x4_t transpose_groups(u32x4_t w) {
    const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap((unsigned)a[0], (unsigned)b[0], false, false);
    const auto d = __builtin_amdgcn_permlane16_swap((unsigned)a[1], (unsigned)b[1], false, false);
    return u32x4_t{(unsigned)c[0], (unsigned)c[1], (unsigned)d[0], (unsigned)d[1]};
}

template <bool BF16, bool ASYM>
__device__ __forceinline__ u32x4_t codes8(uint32_t w) {
    constexpr uint32_t kOr = BF16 ? 0x43004300u : 0u;
    if (!ASYM) w ^= 0x88888888u;
    return u32x4_t{(w & 0x000F000Fu) | kOr, ((w >> 4) & 0x000F000Fu) | kOr, ((w >> 8) & 0x000F000Fu) | kOr, ((w >> 12) & 0x000F000Fu) | kOr};
}

// SMALL: groups that are not a multiple of 128 codes.
template <bool BF16, bool ASYM, bool SMALL, int MT, int NT, int NW, int PF>
__global__ __launch_bounds__(NW * 64) void linear_w4a16_kernel(W4A16Args a) {
    extern __shared__ float red[];                                 // [NW][MT * NT * 4][64]
    constexpr int FOLDS = SMALL ? 4 : 1;                           // sums per chunk that get a scale of their own
    constexpr uint32_t kOne = BF16 ? 0x3F803F80u : 0x3C003C00u;
    constexpr uint32_t kOff = BF16 ? 0xC308C308u : 0x80088008u;    // -136; -8 * 2^-24
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
    const int n0 = blockIdx.x * (16 * NT), m0 = blockIdx.y * (16 * MT);
    const int chunks = (a.K + 127) >> 7;

    struct Stage {
        u32x4_t w[NT], x[MT][4];
        float s[NT][FOLDS], z[NT][ASYM ? FOLDS : 1];
    } st[PF];
    const uint8_t *wp[NT];
    const float *sp[NT], *zp[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int n = min(n0 + 16 * t + col, a.N - 1);
        wp[t] = a.q + (size_t)n * (a.K >> 1);
        sp[t] = a.scale + (size_t)n * a.ng;
        if (ASYM) zp[t] = a.zero + (size_t)n * a.ng;
    }
    const uint16_t *xp[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) xp[t] = a.x + (size_t)min(m0 + 16 * t + col, a.M - 1) * a.ldx;

    auto load = [&](Stage &s, int c) {
        const int left = a.K - 128 * c;                            // codes from here on: below 128 in the last chunk only
        const bool in = 32 * kg < left;
        const int wo = 64 * c + (in ? 16 * kg : 0);
#pragma unroll
        for (int t = 0; t < NT; ++t) s.w[t] = *reinterpret_cast<const u32x4_t *>(wp[t] + wo);
#pragma unroll
        for (int f = 0; f < FOLDS; ++f) {
            const int k = 128 * c + 32 * f;
            const int g = a.group && k < a.K ? k / a.group : 0;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                s.s[t][f] = sp[t][g];
                if (ASYM) s.z[t][f] = zp[t][g];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = SMALL ? 32 * j + 8 * kg : 32 * kg + 8 * j;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                s.x[t][j] = u32x4_t{0, 0, 0, 0};
                if (k < left) s.x[t][j] = *reinterpret_cast<const u32x4_t *>(xp[t] + 128 * c + k);
            }
        }
    };

    float4_t tot[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) tot[i][t] = float4_t{0, 0, 0, 0};

    auto compute = [&](Stage &s) {
        if (SMALL)
#pragma unroll
            for (int t = 0; t < NT; ++t) s.w[t] = transpose_groups(s.w[t]);
#pragma unroll
        for (int f = 0; f < FOLDS; ++f) {
            constexpr int STEPS = 4 / FOLDS;
            u32x4_t xr[MT][STEPS];
            float4_t first[MT], sx[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                first[i] = sx[i] = float4_t{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < STEPS; ++j) {
                    xr[i][j] = pair_up(s.x[i][f * STEPS + j]);
                    if (ASYM) sx[i] = mfma16<BF16>(xr[i][j], u32x4_t{kOne, kOne, kOne, kOne}, sx[i]);
                    else first[i] = mfma16<BF16>(xr[i][j], u32x4_t{kOff, kOff, kOff, kOff}, first[i]);
                }
                if (ASYM && BF16)
#pragma unroll
                    for (int e = 0; e < 4; ++e) first[i][e] = -128.0f * sx[i][e];
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float4_t acc[MT];
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[i] = first[i];
#pragma unroll
                for (int j = 0; j < STEPS; ++j) {
                    const u32x4_t w = codes8<BF16, ASYM>(s.w[t][f * STEPS + j]);
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[i] = mfma16<BF16>(xr[i][j], w, acc[i]);
                }
                const float sc = BF16 ? s.s[t][f] : s.s[t][f] * 16777216.0f;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        tot[i][t][e] = __fmaf_rn(acc[i][e], sc, tot[i][t][e]);
                        if (ASYM) tot[i][t][e] = __fmaf_rn(sx[i][e], s.z[t][f], tot[i][t][e]);
                    }
            }
        }
    };

#pragma unroll
    for (int p = 0; p < PF; ++p)
        if (wave + p * NW < chunks) load(st[p], wave + p * NW);
    for (int c = wave; c < chunks; c += PF * NW) {
#pragma unroll
        for (int p = 0; p < PF; ++p) {
            const int at = c + p * NW;
            if (at < chunks) {
                compute(st[p]);
                if (at + PF * NW < chunks) load(st[p], at + PF * NW);
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
    const int rows = min(16 * MT, a.M - m0), cols = min(16 * NT, a.N - n0);
    for (int o = threadIdx.x; o < rows * 16 * NT; o += NW * 64) {
        const int m = o / (16 * NT), n = o % (16 * NT);
        if (n >= cols) continue;
        const int reg = ((m >> 4) * NT + (n >> 4)) * 4 + (m & 3), from = ((m & 15) >> 2) * 16 + (n & 15);
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) y += red[(w * REGS + reg) * 64 + from];
        if (a.bias) y += to_float<BF16>(a.bias[n0 + n]);
        if (a.act == W4A4_ACT_GELU) y = gelu_erf(y);
        a.out[(size_t)(m0 + m) * a.N + n0 + n] = from_float<BF16>(y);
    }
}

template <bool BF16, bool ASYM, bool SMALL, int MT, int NT, int NW, int PF>
int launch(const W4A16Args &a, hipStream_t st) {
    auto kern = linear_w4a16_kernel<BF16, ASYM, SMALL, MT, NT, NW, PF>;
    constexpr size_t lds = (size_t)NW * MT * NT * 4 * 64 * sizeof(float);
    static KernelState ks;
    if (prepare_kernel(reinterpret_cast<const void *>(kern), lds, ks) < 0) return W4A4_ERR_HIP;
    const dim3 grid((a.N + 16 * NT - 1) / (16 * NT), (a.M + 16 * MT - 1) / (16 * MT));
    hipLaunchKernelGGL(kern, grid, dim3(NW * 64), lds, st, a);
    return launch_status();
}

template <bool BF16, bool ASYM, bool SMALL>
int pick(const W4A16Args &a, hipStream_t st) {
    if (a.M <= 16) return a.N >= 8192 ? launch<BF16, ASYM, SMALL, 1, 2, 8, 2>(a, st) : launch<BF16, ASYM, SMALL, 1, 1, 8, 2>(a, st);
    if (a.M <= 32) return a.N >= 8192 ? launch<BF16, ASYM, SMALL, 2, 4, 4, 2>(a, st) : launch<BF16, ASYM, SMALL, 2, 1, 8, 2>(a, st);
    return a.N >= 8192 ? launch<BF16, ASYM, SMALL, 4, 4, 4, 1>(a, st) : launch<BF16, ASYM, SMALL, 4, 1, 8, 1>(a, st);
}

}  // namespace
}  // namespace w4a4

using namespace w4a4;

extern "C" int w4a4_linear_w4a16(const void *X, int dtype, int M, int K, int ldx, const w4a4_weight *W, const void *bias, int act,
                                 void *out, void *stream) {
    if (!W || M < 0 || ldx < K || W->K != K || K <= 0 || W->N <= 0 || W->group < 0) return W4A4_ERR_INVALID_ARG;
    if (dtype != W4A4_F16 && dtype != W4A4_BF16) return W4A4_ERR_INVALID_ARG;
    if (act != W4A4_ACT_NONE && act != W4A4_ACT_GELU) return W4A4_ERR_INVALID_ARG;
    if (W->mode != W4A4_SYM && W->mode != W4A4_ASYM) return W4A4_ERR_INVALID_ARG;
    if (M == 0) return W4A4_OK;
    if (!X || !out || !W->q || !W->scale || (W->mode == W4A4_ASYM && !W->zero)) return W4A4_ERR_INVALID_ARG;
    if (W->layout != W4A4_LAYOUT_CANONICAL) return W4A4_ERR_UNSUPPORTED_SHAPE;
    if (K % 32 || W->N % 8 || ldx % 8 || (W->group && (W->group % 32 || K % W->group))) return W4A4_ERR_UNSUPPORTED_SHAPE;
    if (!aligned16(X) || !aligned16(W->q) || !aligned16(out) || (bias && !aligned16(bias))) return W4A4_ERR_UNSUPPORTED_SHAPE;
    if (M > 65535 * 16) return W4A4_ERR_UNSUPPORTED_SHAPE;         // (rows of the grid)
    const W4A16Args a{static_cast<const uint16_t *>(X), W->q, W->scale, W->zero, static_cast<const uint16_t *>(bias),
                      static_cast<uint16_t *>(out), M, W->N, K, ldx, W->group, W->group ? K / W->group : 1, act};
    const bool small = W->group % 128 != 0;
    hipStream_t st = as_stream(stream);
    auto typed = [&](auto bf16) {
        constexpr bool BF = decltype(bf16)::value;
        if (W->mode == W4A4_ASYM) return small ? pick<BF, true, true>(a, st) : pick<BF, true, false>(a, st);
        return small ? pick<BF, false, true>(a, st) : pick<BF, false, false>(a, st);
    };
    return dtype == W4A4_BF16 ? typed(std::true_type{}) : typed(std::false_type{});
}
