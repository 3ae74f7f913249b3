// New keys and values into the 8-bit cache, and rows of the cache back out.
//
// A block of a head has one scale: the largest magnitude that has been written into it since its first slot was, over 127.  A
// write whose range passes it raises the scale, and the codes that stay are re-scaled (code * old / new, to nearest even).
//
// The new tokens of one block stand together in `slots`, so a wave owns a (block, head) and one of keys or values: it finds the
// run of tokens, takes their range, settles the scale and writes, without atomics and without another wave to wait for.  Keys
// are rows of D codes; values are stored by feature, so that a lane gathers a feature of up to sixteen tokens and writes their
// codes as one 16-byte piece.  Memory bounds it: a token's row is read once (16 of them wait in registers between the two
// passes) and written once at half the width.
#include "gen.hpp"

namespace w4a4 {
namespace {

constexpr int kPiece = 16;                                         // tokens of a run that a wave takes at once

struct AppendArgs {
    int8_t *k, *v;
    float *k_scale, *v_scale;
    const uint16_t *x[2];                                          // new keys, new values
    long ld[2];
    const int32_t *slots;
    int T, blocks, H, shift, tile;
};

// Code of x: NaN is stored as 0, what passes the range (an infinity) as its end.
__device__ __forceinline__ int code8(float x, float inv) {
    const float t = fminf(fmaxf(x * inv, -127.0f), 127.0f);        // (a NaN gives -127 here)
    return x != x ? 0 : (int)rintf(t);
}
__device__ __forceinline__ float finite_abs(float x) {             // infinities and NaN do not count for a range
    const float y = fabsf(x);
    return y <= 3.4028234e38f ? y : 0.0f;
}

// D features, two neighbouring ones per lane and step of 128.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void kv8_append_kernel(AppendArgs a) {
    constexpr int F = (D + 127) / 128;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int which = blockIdx.y * 4 + wave;                       // 0 .. H-1: keys of a head, H .. 2H-1: values
    if (which >= 2 * a.H) return;
    const bool val = which >= a.H;
    const int h = val ? which - a.H : which, block = 1 << a.shift;
    const int t_first = blockIdx.x * a.tile, t_last = min(t_first + a.tile, a.T);
    const uint16_t *x = a.x[val] + h * D + 2 * lane;
    const long ld = a.ld[val];
    float *scales = val ? a.v_scale : a.k_scale;
    auto block_of = [&](int t) {                                   // -1: a token that is not stored
        const int s = a.slots[t];
        return s >= 0 && (s >> a.shift) < a.blocks ? s >> a.shift : -1;
    };

    for (int t0 = t_first; t0 < t_last; ++t0) {
        const int b = block_of(t0);
        if (b < 0 || (t0 > 0 && block_of(t0 - 1) == b)) continue;  // (not the first token of its run)
        int t1 = t0 + 1;
        while (t1 < a.T && block_of(t1) == b) ++t1;

        // the range of the run, its first slot
        float wide = 0.0f;
        bool first = false;
        for (int t = t0; t < t1; ++t) {
            first |= (a.slots[t] & (block - 1)) == 0;
#pragma unroll
            for (int f = 0; f < F; ++f)
                if (128 * f + 2 * lane < D) {
                    const uint32_t w = *reinterpret_cast<const uint32_t *>(x + t * ld + 128 * f);
                    wide = fmaxf(wide, fmaxf(finite_abs(to_float<BF16>((uint16_t)w)), finite_abs(to_float<BF16>((uint16_t)(w >> 16)))));
                }
        }
        wide = lanes_reduce<64>(wide, [](float p, float q) { return fmaxf(p, q); });
        const size_t unit = (size_t)b * a.H + h;
        const float had = scales[unit], was = first ? 0.0f : had;
        float now = fmaxf(was, wide / 127.0f);
        if (now < 1.1754943508e-38f) now = 0.0f;                   // (its reciprocal would not be a number)
        const float inv = now > 0.0f ? 1.0f / now : 0.0f;
        int8_t *codes = (val ? a.v : a.k) + unit * D * block;
        if (!first && now != was) {                                // what stays of the block
            const float ratio = now > 0.0f ? was / now : 0.0f;
            for (int i = 16 * lane; i < D * block; i += 16 * 64) {
                u32x4_t p = *reinterpret_cast<const u32x4_t *>(codes + i);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t o = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o |= ((uint32_t)(int)rintf((float)(int8_t)(p[j] >> (8 * e)) * ratio) & 0xFFu) << (8 * e);
                    p[j] = o;
                }
                *reinterpret_cast<u32x4_t *>(codes + i) = p;
            }
            __threadfence();                                       // the new codes of other lanes come behind these
        }
        if (lane == 0 && now != had) scales[unit] = now;
        for (int t = t0; t < t1; ++t) {
            const int off = a.slots[t] & (block - 1);
#pragma unroll
            for (int f = 0; f < F; ++f)
                if (128 * f + 2 * lane < D) {
                    const uint32_t w = *reinterpret_cast<const uint32_t *>(x + t * ld + 128 * f);
                    const int c0 = code8(to_float<BF16>((uint16_t)w), inv), c1 = code8(to_float<BF16>((uint16_t)(w >> 16)), inv);
                    const int d = 128 * f + 2 * lane;
                    if (val) {
                        codes[(size_t)d * block + off] = (int8_t)c0;
                        codes[(size_t)(d + 1) * block + off] = (int8_t)c1;
                    } else {
                        *reinterpret_cast<uint16_t *>(codes + (size_t)off * D + d) = (uint16_t)((c0 & 0xFF) | (c1 & 0xFF) << 8);
                    }
                }
        }
    }
}

struct ReadArgs {
    const int8_t *k, *v;
    const float *k_scale, *v_scale;
    uint16_t *out[2];
    const int32_t *slots;
    int T, blocks, H, shift;
};

template <bool BF16, int D>
__global__ __launch_bounds__(256) void kv8_read_kernel(ReadArgs a) {
    constexpr int F = (D + 127) / 128;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int which = blockIdx.y * 4 + wave;
    if (which >= 2 * a.H) return;
    const bool val = which >= a.H;
    const int h = val ? which - a.H : which, block = 1 << a.shift;
    const int t0 = blockIdx.x * kPiece, t1 = min(t0 + kPiece, a.T);
    for (int t = t0; t < t1; ++t) {
        const int slot = a.slots[t], b = slot >> a.shift, off = slot & (block - 1);
        const bool there = slot >= 0 && b < a.blocks;
        const size_t unit = there ? (size_t)b * a.H + h : 0;
        const int8_t *codes = (val ? a.v : a.k) + unit * D * block;
        const float scale = there ? (val ? a.v_scale : a.k_scale)[unit] : 0.0f;
        uint16_t *out = a.out[val] + ((size_t)t * a.H + h) * D;
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int d = 128 * f + 2 * lane;
            if (d < D) {
                int c0 = 0, c1 = 0;
                if (there) {
                    c0 = val ? codes[(size_t)d * block + off] : codes[(size_t)off * D + d];
                    c1 = val ? codes[(size_t)(d + 1) * block + off] : codes[(size_t)off * D + d + 1];
                }
                *reinterpret_cast<uint32_t *>(out + d) = from_float<BF16>((float)c0 * scale) | (uint32_t)from_float<BF16>((float)c1 * scale) << 16;
            }
        }
    }
}

template <typename F>
int by_features(int D, F f) {
    switch (D) {
        case 64: return f(std::integral_constant<int, 64>{});
        case 96: return f(std::integral_constant<int, 96>{});
        case 128: return f(std::integral_constant<int, 128>{});
        default: return f(std::integral_constant<int, 256>{});
    }
}

}  // namespace

int kv8_cache_check(const w4a4_kv8_cache *C) {
    if (!C || C->blocks < 0 || C->heads <= 0 || C->features <= 0 || C->block <= 0) return W4A4_ERR_INVALID_ARG;
    if (C->blocks && (!C->k || !C->v || !C->k_scale || !C->v_scale)) return W4A4_ERR_INVALID_ARG;
    const int D = C->features;
    if (!kv8_block_ok(C->block) || (D != 64 && D != 96 && D != 128 && D != 256) || C->heads > 1024) return W4A4_ERR_UNSUPPORTED_SHAPE;
    if ((long)C->blocks * C->block > 0x7fffffffL) return W4A4_ERR_UNSUPPORTED_SHAPE;
    if (!aligned16(C->k) || !aligned16(C->v)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    return W4A4_OK;
}

}  // namespace w4a4

using namespace w4a4;

extern "C" int w4a4_kv8_append(const w4a4_kv8_cache *C, const void *K, const void *V, int dtype, int tokens, int ldk, int ldv,
                               const int32_t *slots, void *stream) {
    if (const int rc = kv8_cache_check(C)) return rc;
    if (tokens < 0 || (dtype != W4A4_F16 && dtype != W4A4_BF16)) return W4A4_ERR_INVALID_ARG;
    const int row = C->heads * C->features;
    if (ldk < row || ldv < row) return W4A4_ERR_INVALID_ARG;
    if (tokens == 0) return W4A4_OK;
    if (!K || !V || !slots) return W4A4_ERR_INVALID_ARG;
    if (ldk % 8 || ldv % 8 || !aligned16(K) || !aligned16(V)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    AppendArgs a{C->k, C->v, C->k_scale, C->v_scale, {static_cast<const uint16_t *>(K), static_cast<const uint16_t *>(V)}, {ldk, ldv},
                 slots, tokens, C->blocks, C->heads, __builtin_ctz(C->block), tokens <= 512 ? 1 : kPiece};
    const dim3 grid((tokens + a.tile - 1) / a.tile, (2 * C->heads + 3) / 4);
    return by_features(C->features, [&](auto d) {
        constexpr int D = decltype(d)::value;
        if (dtype == W4A4_BF16) hipLaunchKernelGGL((kv8_append_kernel<true, D>), grid, dim3(256), 0, as_stream(stream), a);
        else hipLaunchKernelGGL((kv8_append_kernel<false, D>), grid, dim3(256), 0, as_stream(stream), a);
        return launch_status();
    });
}

extern "C" int w4a4_kv8_read(const w4a4_kv8_cache *C, const int32_t *slots, int tokens, int dtype, void *K, void *V, void *stream) {
    if (const int rc = kv8_cache_check(C)) return rc;
    if (tokens < 0 || (dtype != W4A4_F16 && dtype != W4A4_BF16)) return W4A4_ERR_INVALID_ARG;
    if (tokens == 0) return W4A4_OK;
    if (!slots || !K || !V) return W4A4_ERR_INVALID_ARG;
    if (!aligned16(K) || !aligned16(V)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const ReadArgs a{C->k, C->v, C->k_scale, C->v_scale, {static_cast<uint16_t *>(K), static_cast<uint16_t *>(V)}, slots, tokens,
                     C->blocks, C->heads, __builtin_ctz(C->block)};
    const dim3 grid((tokens + kPiece - 1) / kPiece, (2 * C->heads + 3) / 4);
    return by_features(C->features, [&](auto d) {
        constexpr int D = decltype(d)::value;
        if (dtype == W4A4_BF16) hipLaunchKernelGGL((kv8_read_kernel<true, D>), grid, dim3(256), 0, as_stream(stream), a);
        else hipLaunchKernelGGL((kv8_read_kernel<false, D>), grid, dim3(256), 0, as_stream(stream), a);
        return launch_status();
    });
}
