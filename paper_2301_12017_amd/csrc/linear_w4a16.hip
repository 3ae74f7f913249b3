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
// into registers, codes two chunks ahead and x, which comes out of L2, one; the waves of a workgroup have a part of K each, which they add up through LDS.  The four
// words of the four lanes that share a row then change places (two lane swaps a pair), so that each instruction takes 32 consecutive
// codes: a sum never crosses a group (of any multiple of 32), and a row of x is read 64 bytes at a time (without the swaps its
// four lanes read 64 bytes apart, 32 cache lines a load instead of 16).  Inside eight codes the order is free as long as both
// operands agree: (w >> 4j) & 0x000F000F gives codes j and j + 4 of a word, so the pairs of x are put in that order.
//
// Measured (kernel trace, median): 32 tokens of 4096 to 16384 channels, groups of 128 with zeros, 18.4 us, its 39 MB at 2.1 TB/s: two waves
// a SIMD, which wait half of their cycles (vector ALU 23 %, matrix pipe 9 %); without the loads of x, which come out of L2, it is 14.2 (64
// tokens 4096 x 4096: 14.0 and 8.9).  5 tokens 4096 x 4096 5.7 us and one token 768 x 768 3.3 us, mostly launch, first loads and the sum over waves.
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

// One result as the definition has it, code by code.  For sums that are no finite number: an infinity in x would meet its own negative in what takes
// the offset out of the codes, and a bf16 number past 2^120 passes fp32 with the offset's factor.
template <bool BF16, bool ASYM>
__device__ __forceinline__ float code_by_code(const W4A16Args &a, int m, int n) {
    const uint16_t *x = a.x + (size_t)m * a.ldx;
    const uint8_t *q = a.q + (size_t)n * (a.K >> 1);
    const int group = a.group ? a.group : a.K;
    float y = 0.0f;
    for (int g = 0; g < a.ng; ++g) {
        const float scale = a.scale[(size_t)n * a.ng + g], zero = ASYM ? a.zero[(size_t)n * a.ng + g] : 0.0f;
        for (int k = g * group; k < (g + 1) * group && y == y; k += 8) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(q + (k >> 1));
            const u32x4_t v = *reinterpret_cast<const u32x4_t *>(x + k);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float c = ASYM ? (float)(w >> (4 * j) & 15) : (float)((int)(w << (28 - 4 * j)) >> 28);
                y = __fmaf_rn(ASYM ? __fmaf_rn(c, scale, zero) : c * scale, to_float<BF16>((uint16_t)(v[j / 2] >> (16 * (j % 2)))), y);
            }
        }
    }
    return y;
}

struct __attribute__((packed, aligned(4))) Floats4 { float v[4]; };   // (rows of scales begin at any float)

// SMALL: groups that are not a multiple of 128 codes.
template <bool BF16, bool ASYM, bool SMALL, int MT, int NT, int NW>
__global__ __launch_bounds__(NW * 64, NW / 4) void linear_w4a16_kernel(W4A16Args a) {
    extern __shared__ float red[];                                 // [NW][MT * NT * 4][64]
    constexpr int FOLDS = SMALL ? 4 : 1, AHEAD = 2;                // sums per chunk that get a scale of their own; chunks requested ahead
    constexpr uint32_t kOne = BF16 ? 0x3F803F80u : 0x3C003C00u;
    constexpr uint32_t kOff = BF16 ? 0xC308C308u : 0x80088008u;    // -136; -8 * 2^-24
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, kg = lane >> 4;
    const int n0 = blockIdx.x * (16 * NT), m0 = blockIdx.y * (16 * MT);
    const int chunks = (a.K + 127) >> 7, each = (chunks + NW - 1) / NW, c0 = wave * each, c1 = min(c0 + each, chunks);

    // (x of rows behind the last one keeps what the registers hold)
    struct Stage {
        u32x4_t w[NT];
        float s[NT][SMALL ? 4 : 1], z[NT][SMALL && ASYM ? 4 : 1];  // (small groups)
    } st[AHEAD];
    const uint8_t *wp[NT];
    const float *sp[NT], *zp[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int n = min(n0 + 16 * t + col, a.N - 1);
        wp[t] = a.q + (size_t)n * (a.K >> 1);
        sp[t] = a.scale + (size_t)n * a.ng;
        if (ASYM) zp[t] = a.zero + (size_t)n * a.ng;
    }
    u32x4_t x[MT][4];
    const uint16_t *xp[MT];
    bool on[MT];
    // Rows whose bytes at the same place lie in the same half of a cache line are read in turn, one its first 64 bytes of 128, the next its
    // second ones: 16 lanes at once would else ask for one half only.  (All rows of a lane are alike: sixteen rows are a multiple of 128 bytes.)
    // us with | without, N x K: 64 tokens 4096 x 4096 14.0 | 19.7, 16000 x 4096 25.5 | 29.2, 32 tokens 4096 x 4096 8.5 | 11.1, 5 tokens 5.7 | 5.7, 2048 tokens
    // 373 | 550; the tiles of 32 tokens and 64 channels have no registers for it (16384 x 4096 19.4 | 18.2).
    constexpr bool TURNS = !(MT == 2 && NT == 4);
    const uint32_t half = TURNS && ((uint32_t)((reinterpret_cast<uintptr_t>(a.x) + (size_t)(m0 + col) * a.ldx * 2) >> 6) ^ (uint32_t)col) & 1 ? 32 : 0;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = m0 + 16 * t + col;
        on[t] = m < a.M;
        xp[t] = a.x + (size_t)(on[t] ? m : 0) * a.ldx + 8 * kg;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[t][j] = u32x4_t{0, 0, 0, 0};
    }
    float s4[NT][4], z4[NT][4];                                    // groups of whole chunks: the scales of four
    auto load4 = [&](int c) {                                      // of chunks c .. c + 3
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (a.group == 128 && c + 3 < a.ng) {
                const Floats4 f = *reinterpret_cast<const Floats4 *>(sp[t] + c);
#pragma unroll
                for (int j = 0; j < 4; ++j) s4[t][j] = f.v[j];
                if (ASYM) {
                    const Floats4 g = *reinterpret_cast<const Floats4 *>(zp[t] + c);
#pragma unroll
                    for (int j = 0; j < 4; ++j) z4[t][j] = g.v[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int g = a.group ? min(128 * (c + j) / a.group, a.ng - 1) : 0;
                    s4[t][j] = sp[t][g];
                    if (ASYM) z4[t][j] = zp[t][g];
                }
            }
        }
    };

    auto load = [&](Stage &s, int c) {
        const int left = a.K - 128 * c;                            // codes from here on: below 128 in the last chunk only
        const int wo = 64 * c + (32 * kg < left ? 16 * kg : 0);
#pragma unroll
        for (int t = 0; t < NT; ++t) s.w[t] = *reinterpret_cast<const u32x4_t *>(wp[t] + wo);
        if constexpr (SMALL) {
            if (a.group == 32 && 4 * c + 3 < a.ng) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const Floats4 f = *reinterpret_cast<const Floats4 *>(sp[t] + 4 * c);
#pragma unroll
                    for (int j = 0; j < 4; ++j) s.s[t][j] = f.v[j];
                    if constexpr (ASYM) {
                        const Floats4 g = *reinterpret_cast<const Floats4 *>(zp[t] + 4 * c);
#pragma unroll
                        for (int j = 0; j < 4; ++j) s.z[t][j] = g.v[j];
                    }
                }
            } else {
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    const int g = min((128 * c + 32 * f) / a.group, a.ng - 1);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        s.s[t][f] = sp[t][g];
                        if constexpr (ASYM) s.z[t][f] = zp[t][g];
                    }
                }
            }
        }
    };
    auto load_x = [&](int c) {
        const int left = a.K - 128 * c;
        if (left >= 128) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
                if (on[t])
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[t][j] = *reinterpret_cast<const u32x4_t *>(xp[t] + 128 * c + (32 * j ^ half));
        } else {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[t][j] = u32x4_t{0, 0, 0, 0};
                    const int k = 32 * j ^ half;
                    if (k < left) x[t][j] = *reinterpret_cast<const u32x4_t *>(xp[t] + 128 * c + k);
                }
        }
    };

    float4_t tot[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) tot[i][t] = float4_t{0, 0, 0, 0};

    auto compute = [&](Stage &s, int next, auto scale, auto zero) {
        u32x4_t xr[MT][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                u32x4_t v[2];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[0][e] = half ? x[i][j + 1][e] : x[i][j][e];
                    v[1][e] = half ? x[i][j][e] : x[i][j + 1][e];
                }
                xr[i][j] = pair_up(v[0]);
                xr[i][j + 1] = pair_up(v[1]);
            }
        __builtin_amdgcn_sched_barrier(0);                         // (else their registers are needed twice)
        if (next < c1) load_x(next);
        constexpr int STEPS = 4 / FOLDS;
        float4_t first[FOLDS][MT], sx[FOLDS][MT];
#pragma unroll
        for (int f = 0; f < FOLDS; ++f)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                first[f][i] = sx[f][i] = float4_t{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < STEPS; ++j) {
                    if (ASYM) sx[f][i] = mfma16<BF16>(xr[i][f * STEPS + j], u32x4_t{kOne, kOne, kOne, kOne}, sx[f][i]);
                    else first[f][i] = mfma16<BF16>(xr[i][f * STEPS + j], u32x4_t{kOff, kOff, kOff, kOff}, first[f][i]);
                }
            }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const u32x4_t w4 = transpose_groups(s.w[t]);
#pragma unroll
            for (int f = 0; f < FOLDS; ++f) {
                float4_t acc[MT];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    acc[i] = first[f][i];
                    if (ASYM && BF16)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][e] = -128.0f * sx[f][i][e];
                }
#pragma unroll
                for (int j = 0; j < STEPS; ++j) {
                    const u32x4_t w = codes8<BF16, ASYM>(w4[f * STEPS + j]);
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[i] = mfma16<BF16>(xr[i][f * STEPS + j], w, acc[i]);
                }
                const float sc = BF16 ? scale(t, f) : scale(t, f) * 16777216.0f;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        tot[i][t][e] = __fmaf_rn(acc[i][e], sc, tot[i][t][e]);
                        if (ASYM) tot[i][t][e] = __fmaf_rn(sx[f][i][e], zero(t, f), tot[i][t][e]);
                    }
            }
            if (NT > 1) __builtin_amdgcn_sched_barrier(0);
        }
    };

    if (c0 < c1) {
        if (!SMALL) load4(c0);
#pragma unroll
        for (int p = 0; p < AHEAD; ++p)
            if (c0 + p < c1) load(st[p], c0 + p);
        load_x(c0);
        for (int c = c0; c < c1; c += 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (c + j >= c1) break;
                Stage &s = st[j % AHEAD];
                if constexpr (SMALL) compute(s, c + j + 1, [&](int t, int f) { return s.s[t][f]; }, [&](int t, int f) { return s.z[t][f]; });
                else compute(s, c + j + 1, [&](int t, int) { return s4[t][j]; }, [&](int t, int) { return z4[t][j]; });
                if (c + j + AHEAD < c1) load(s, c + j + AHEAD);
            }
            if (!SMALL && a.group && c + 4 < c1) load4(c + 4);
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
    auto results = [&](auto f) {                                   // f(m, n, sum over the waves) for the thread's results
        for (int o = threadIdx.x; o < rows * 16 * NT; o += NW * 64) {
            const int m = o / (16 * NT), n = o % (16 * NT);
            if (n >= cols) continue;
            const int reg = ((m >> 4) * NT + (n >> 4)) * 4 + (m & 3), from = ((m & 15) >> 2) * 16 + (n & 15);
            float y = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) y += red[(w * REGS + reg) * 64 + from];
            f(m0 + m, n0 + n, y);
        }
    };
    auto finish = [&](int m, int n, float y) {
        if (a.bias) y += to_float<BF16>(a.bias[n]);
        if (a.act == W4A4_ACT_GELU && y == y) y = gelu_erf(y);     // (which takes a NaN with its sign bit set for a negative number)
        a.out[(size_t)m * a.N + n] = from_float<BF16>(y);
    };
    bool finite = true;
    results([&](int m, int n, float y) {
        finish(m, n, y);
        finite &= fabsf(y) < INFINITY;
    });
    if (finite) return;
    results([&](int m, int n, float y) {                           // (a loop of its own: inside the first one 64 tokens 16000 x 4096 took 26.1 us, not 25.5)
        if (!(fabsf(y) < INFINITY)) finish(m, n, code_by_code<BF16, ASYM>(a, m, n));
    });
}

template <bool BF16, bool ASYM, bool SMALL, int MT, int NT, int NW>
int launch(const W4A16Args &a, hipStream_t st) {
    auto kern = linear_w4a16_kernel<BF16, ASYM, SMALL, MT, NT, NW>;
    constexpr size_t lds = (size_t)NW * MT * NT * 4 * 64 * sizeof(float);
    static KernelState ks;
    if (prepare_kernel(reinterpret_cast<const void *>(kern), lds, ks) < 0) return W4A4_ERR_HIP;
    const dim3 grid((a.N + 16 * NT - 1) / (16 * NT), (a.M + 16 * MT - 1) / (16 * MT));
    hipLaunchKernelGGL(kern, grid, dim3(NW * 64), lds, st, a);
    return launch_status();
}

// Tiles of channels a wave: as many as leave a workgroup for three quarters of the CUs (x is read once per workgroup, and costs as many
// load instructions as the codes of four tiles; more tiles than that leave CUs without work).  us at one | two | four tiles, N x K:
//   1 token 16000 x 4096 13.0 | 10.7 | 10.8, 5 tokens 4096 x 4096 5.4 | 6.3 | 9.6, 16 tokens 16000 x 11008 58 | 40 | 32,
//   32 tokens 16384 x 4096 41 | 25 | 17.6, 20 tokens 4096 x 4096 8.5 | 9.8 | 13.4, 64 tokens 16000 x 4096 71 | 42 | 29.
// (before rows of x were read in turn, which takes 5 to 30 % off from 12 tokens on, and does not change the order).
// Four tiles of four times sixteen tokens take the registers of a SIMD for one wave.  Small groups have four sums a chunk, whose
// operands leave room for one tile (24 tokens 2000 x 8000 in groups of 32: 17 us, two tiles 47), for two where tokens are few.
template <bool BF16, bool ASYM, bool SMALL, int MT>
int pick(const W4A16Args &a, hipStream_t st) {
    const int tiles = a.N / 16;
    if constexpr (!SMALL)
        if (tiles >= 4 * 192) return launch<BF16, ASYM, SMALL, MT, 4, MT == 4 ? 4 : 8>(a, st);
    if constexpr (!SMALL || MT == 1)
        if (tiles >= 2 * 192) return launch<BF16, ASYM, SMALL, MT, 2, MT == 4 ? 4 : 8>(a, st);
    return launch<BF16, ASYM, SMALL, MT, 1, 8>(a, st);
}
template <bool BF16, bool ASYM, bool SMALL>
int pick(const W4A16Args &a, hipStream_t st) {
    if (a.M <= 16) return pick<BF16, ASYM, SMALL, 1>(a, st);
    if constexpr (!SMALL)
        if (a.M > 32) return pick<BF16, ASYM, SMALL, 4>(a, st);
    return pick<BF16, ASYM, SMALL, 2>(a, st);
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
