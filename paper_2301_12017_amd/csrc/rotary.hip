// Heads of features turned by their tokens' positions.
//
//   a' = m (a cos(p f) - b sin(p f)),  b' = m (b cos(p f) + a sin(p f))    for each pair (a, b) of features, p the position, f the pair's frequency
//
// A unit of work is one token's piece of a head that turns within itself: eight neighbouring features (pairs of neighbours), eight and the
// eight that they pair with (halves of the turned part), or one feature and its partner where the halves are no multiple of eight.  A thread
// keeps its piece and takes head after head, so that angles are found once for all heads; neighbouring threads have neighbouring pieces and
// heads.  Features behind the turned part are copied.
#include "rotary.hpp"

namespace w4a4 {
namespace {

struct Args {
    const uint16_t *x;
    uint16_t *out;
    const int32_t *positions;
    long ldx, ldo;
    int tokens, heads, features;
    int units, side, share;                                        // pieces of a head; heads that a workgroup takes at once, of `share` tokens
    RotaryArgs r;
};

enum { NEIGHBOURS, HALVES, SINGLE };

template <bool BF16>
__device__ __forceinline__ float half_of(u32x4_t w, int j) { return to_float<BF16>((uint16_t)(w[j / 2] >> (16 * (j % 2)))); }
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float a, float b) { return from_float<BF16>(a) | (uint32_t)from_float<BF16>(b) << 16; }

template <bool BF16, int WAY>
__global__ __launch_bounds__(256) void rotary_kernel(Args a) {
    constexpr int V = WAY == SINGLE ? 1 : 8, T = WAY == NEIGHBOURS ? 4 : V, B = 4;          // features of a unit (and of its partner); its angles; heads at once
    const int unit = threadIdx.x % a.units, group = threadIdx.x / a.units, pairs = a.r.pairs;
    const int sub = group / a.side, h0 = group % a.side;
    const long t = (long)blockIdx.x * a.share + sub;
    if (sub >= a.share || t >= a.tokens) return;
    const int position = a.positions[t];
    // first feature, and first feature of the partners (none: the same again)
    const int mine = WAY == NEIGHBOURS ? 8 * unit : V * unit < pairs ? V * unit : V * unit + pairs;
    const bool turns = position >= 0 && (WAY == NEIGHBOURS ? 2 * T * unit < 2 * pairs : V * unit < pairs);
    const int other = WAY != NEIGHBOURS && V * unit < pairs ? mine + pairs : mine;
    Turn angle[T];
    if (turns)
#pragma unroll
        for (int i = 0; i < T; ++i) {
            const int p = T * unit + i;
            angle[i] = turn_of(a.r.turns[min(p, pairs - 1)], (uint32_t)position, a.r.magnitude, a.r.inverse);
        }
    const uint16_t *x = a.x + t * a.ldx;
    uint16_t *out = a.out + t * a.ldo;
    for (int h = h0; h < a.heads; h += a.side * B) {
        if constexpr (WAY == SINGLE) {
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int at = (h + b * a.side) * a.features;
                if (h + b * a.side >= a.heads) break;
                const uint16_t u = x[at + mine], v = x[at + other];
                if (turns) {
                    const float p = to_float<BF16>(u), q = to_float<BF16>(v);
                    out[at + mine] = from_float<BF16>(turned_a(angle[0], p, q));
                    out[at + other] = from_float<BF16>(turned_b(angle[0], p, q));
                } else {
                    out[at + mine] = u;
                    if (other != mine) out[at + other] = v;
                }
            }
        } else {
            u32x4_t u[B], v[B];
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int at = (h + b * a.side) * a.features;
                if (h + b * a.side >= a.heads) break;
                u[b] = *reinterpret_cast<const u32x4_t *>(x + at + mine);
                if (WAY == HALVES) v[b] = *reinterpret_cast<const u32x4_t *>(x + at + other);
            }
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int at = (h + b * a.side) * a.features;
                if (h + b * a.side >= a.heads) break;
                if (turns) {
                    if constexpr (WAY == NEIGHBOURS) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float p = half_of<BF16>(u[b], 2 * i), q = half_of<BF16>(u[b], 2 * i + 1);
                            if (4 * unit + i < pairs) u[b][i] = pack2<BF16>(turned_a(angle[i], p, q), turned_b(angle[i], p, q));
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            const float p0 = half_of<BF16>(u[b], i), q0 = half_of<BF16>(v[b], i), p1 = half_of<BF16>(u[b], i + 1), q1 = half_of<BF16>(v[b], i + 1);
                            u[b][i / 2] = pack2<BF16>(turned_a(angle[i], p0, q0), turned_a(angle[i + 1], p1, q1));
                            v[b][i / 2] = pack2<BF16>(turned_b(angle[i], p0, q0), turned_b(angle[i + 1], p1, q1));
                        }
                    }
                }
                *reinterpret_cast<u32x4_t *>(out + at + mine) = u[b];
                if (WAY == HALVES && other != mine) *reinterpret_cast<u32x4_t *>(out + at + other) = v[b];
            }
        }
    }
}

}  // namespace

int rotary_launch(const void *x, int dtype, int tokens, int heads, int features, long ldx, const int32_t *positions, const RotaryArgs &r, void *out, long ldo, hipStream_t st) {
    const int way = r.interleaved ? NEIGHBOURS : r.pairs % 8 == 0 ? HALVES : SINGLE;
    const int units = way == NEIGHBOURS ? features / 8 : way == HALVES ? (features - r.pairs) / 8 : features - r.pairs;      // at most 255
    const int groups = 256 / units, side = groups < heads ? groups : heads;
    int share = groups / side;
    while (share > 1 && (tokens + share - 1) / share < 512) --share;                  // (few tokens: a CU for each)
    const Args a{static_cast<const uint16_t *>(x), static_cast<uint16_t *>(out), positions, ldx, ldo, tokens, heads, features, units, side, share, r};
    const dim3 grid((unsigned)(((long)tokens + share - 1) / share));
    auto run = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a); };
    if (dtype == W4A4_BF16) way == NEIGHBOURS ? run(rotary_kernel<true, NEIGHBOURS>) : way == HALVES ? run(rotary_kernel<true, HALVES>) : run(rotary_kernel<true, SINGLE>);
    else way == NEIGHBOURS ? run(rotary_kernel<false, NEIGHBOURS>) : way == HALVES ? run(rotary_kernel<false, HALVES>) : run(rotary_kernel<false, SINGLE>);
    return launch_status();
}

}  // namespace w4a4

using namespace w4a4;

extern "C" int w4a4_rotary(const void *X, int dtype, int tokens, int heads, int features, int ldx, const int32_t *positions, const w4a4_rotary_angles *R,
                           void *out, int ldo, void *stream) {
    if (tokens < 0 || heads <= 0 || features <= 0 || (dtype != W4A4_F16 && dtype != W4A4_BF16)) return W4A4_ERR_INVALID_ARG;
    if ((long)heads * features > ldx || (long)heads * features > ldo) return W4A4_ERR_INVALID_ARG;
    if (const int rc = rotary_check(R, features)) return rc;
    if (features % 8 || features > 256 || ldx % 8 || ldo % 8) return W4A4_ERR_UNSUPPORTED_SHAPE;
    if (tokens == 0) return W4A4_OK;
    if (!X || !out || !positions) return W4A4_ERR_INVALID_ARG;
    if (X == out && ldx != ldo) return W4A4_ERR_INVALID_ARG;
    if (!aligned16(X) || !aligned16(out)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    return rotary_launch(X, dtype, tokens, heads, features, ldx, positions, rotary_args(R), out, ldo, as_stream(stream));
}
