// Rotation of pairs of features by a token's position (gfx950): angles, a pair turned, heads of tokens turned.
//
// A pair turns by `position * frequency`, and only the fraction of a turn counts.  Frequencies are 64-bit fractions of a turn (2^-64 units), so the
// product with a position, its low 64 bits kept, is that fraction with nothing lost but the frequency's own rounding: position * 2^-65 turns,
// 2^-34 for the last position there is.  Its top 32 bits, rounded (half a unit is 7e-10), the nearest quarter turn taken off, are an angle x of at most pi / 4 in fp32.
//
// In units of 2^-24 of the pair's length: x is off by 0.39 (its conversion), 0.37 (2 pi in fp32) and 0.5 (their product); the Taylor series of sine and cosine around 0 up to
// x^9 and x^10 by 2e-9 = 0.03 and, through the roundings of their steps, sine by 0.7 and cosine by 0.9.  That is 2.5 at most in all, 2.02 measured over 6 million
// fractions.  A turned number is a product, rounded, in a sum, rounded once: 1.6 more where x is largest, and a magnitude that is not 1 another 1.
#pragma once
#include "gen.hpp"

namespace w4a4 {

struct RotaryArgs {
    const uint64_t *turns;                                         // [pairs]
    int pairs, interleaved;
    float magnitude;
    int inverse;                                                   // by the opposite angles
};

struct Turn { float cos, sin; };

__device__ __forceinline__ Turn turn_of(uint64_t per, uint32_t position, float magnitude, int inverse) {
    const uint32_t f = (uint32_t)((per * position + 0x80000000u) >> 32);
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

// How the pieces of a head turn: eight neighbouring features within themselves (pairs of neighbours), eight or four and those that they pair with
// (halves of the turned part), or one feature and its partner where the halves are no multiple of four.
enum RotaryWay { kRotaryNeighbours, kRotaryHalves8, kRotaryHalves4, kRotarySingle };

// Heads of tokens turned, by workgroups of 256.  A thread keeps its piece of a head and takes several heads, so that angles are found once for them;
// neighbouring threads have neighbouring pieces and heads.
struct RotaryWork {
    const uint16_t *x;
    uint16_t *out;
    const int32_t *positions;
    long ldx, ldo;
    int tokens, heads, features;
    int way, units, paired;                                        // pieces of a head; the first of them that are not turned and come two at a time
    int side, share;                                               // threads that have a token's heads between them, tokens at once
    RotaryArgs r;
};

template <int V>
struct Piece;
template <>
struct Piece<8> { typedef u32x4_t T; };
template <>
struct Piece<4> { typedef u32x2_t T; };
template <>
struct Piece<1> { typedef uint16_t T; };

template <bool BF16, int V>
__device__ __forceinline__ float piece_get(typename Piece<V>::T w, int j) {
    if constexpr (V == 1) return to_float<BF16>(w);
    else return to_float<BF16>((uint16_t)(w[j / 2] >> (16 * (j % 2))));
}

// Tokens t0 .. t0 + count - 1, B heads of a thread at once.
template <bool BF16, int WAY, int B>
__device__ __forceinline__ void rotary_tokens(const RotaryWork &a, long t0, int count) {
    constexpr int V = WAY == kRotarySingle ? 1 : WAY == kRotaryHalves4 ? 4 : 8, T = WAY == kRotaryNeighbours ? 4 : V;   // features of a piece; its angles
    constexpr bool HALVES = WAY != kRotaryNeighbours;
    typedef typename Piece<V>::T P;
    const int unit = threadIdx.x % a.units, group = threadIdx.x / a.units, pairs = a.r.pairs, sub = group / a.side, h0 = group % a.side;
    if (sub >= a.share) return;
    // first features of the piece and of its partner; of what does not turn a piece and its other half, or a piece alone
    const int still = HALVES ? unit - pairs / V : 0, rest = a.features - 2 * pairs;
    const bool on = HALVES ? still < 0 : 4 * unit < pairs;
    const int mine = !HALVES ? 8 * unit : on ? V * unit : 2 * pairs + V * still;
    const int other = HALVES && on ? mine + pairs : HALVES && a.paired ? mine + rest / 2 : mine;
    uint64_t per[T];
#pragma unroll
    for (int i = 0; i < T; ++i) per[i] = a.r.turns[min(T * unit + i, pairs - 1)];
    for (long t = t0 + sub; t < t0 + count; t += a.share) {
        const int position = a.positions[t];
        const uint16_t *x = a.x + t * a.ldx;
        uint16_t *out = a.out + t * a.ldo;
        Turn angle[T];
        for (int h = h0; h < a.heads; h += a.side * B) {
            P u[B], v[B];
#pragma unroll
            for (int b = 0; b < B; ++b) {                          // (heads behind the last one: the last again)
                const uint16_t *p = x + (long)min(h + b * a.side, a.heads - 1) * a.features;
                u[b] = *reinterpret_cast<const P *>(p + mine);
                if (HALVES) v[b] = *reinterpret_cast<const P *>(p + other);
            }
            if (h == h0 && on)
#pragma unroll
                for (int i = 0; i < T; ++i) angle[i] = turn_of(per[i], (uint32_t)position, a.r.magnitude, a.r.inverse);
#pragma unroll
            for (int b = 0; b < B; ++b) {
                if (on && position >= 0) {
                    if constexpr (WAY == kRotaryNeighbours) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float p = piece_get<BF16, V>(u[b], 2 * i), q = piece_get<BF16, V>(u[b], 2 * i + 1);
                            const uint32_t w = from_float<BF16>(turned_a(angle[i], p, q)) | (uint32_t)from_float<BF16>(turned_b(angle[i], p, q)) << 16;
                            if (4 * unit + i < pairs) u[b][i] = w;
                        }
                    } else if constexpr (V == 1) {
                        const float p = to_float<BF16>(u[b]), q = to_float<BF16>(v[b]);
                        u[b] = from_float<BF16>(turned_a(angle[0], p, q));
                        v[b] = from_float<BF16>(turned_b(angle[0], p, q));
                    } else {
#pragma unroll
                        for (int i = 0; i < V; i += 2) {
                            const float p0 = piece_get<BF16, V>(u[b], i), q0 = piece_get<BF16, V>(v[b], i), p1 = piece_get<BF16, V>(u[b], i + 1), q1 = piece_get<BF16, V>(v[b], i + 1);
                            u[b][i / 2] = from_float<BF16>(turned_a(angle[i], p0, q0)) | (uint32_t)from_float<BF16>(turned_a(angle[i + 1], p1, q1)) << 16;
                            v[b][i / 2] = from_float<BF16>(turned_b(angle[i], p0, q0)) | (uint32_t)from_float<BF16>(turned_b(angle[i + 1], p1, q1)) << 16;
                        }
                    }
                }
                if (h + b * a.side < a.heads) {
                    uint16_t *p = out + (long)(h + b * a.side) * a.features;
                    *reinterpret_cast<P *>(p + mine) = u[b];
                    if (HALVES && other != mine) *reinterpret_cast<P *>(p + other) = v[b];
                }
            }
        }
    }
}

// W4A4_OK, or what is wrong with a plan of angles for heads of `features`.
inline int rotary_check(const w4a4_rotary_angles *R, int features) {
    if (!R || !R->turns || R->pairs <= 0 || 2 * (long)R->pairs > features || !(R->magnitude > 0.0f) || !(R->magnitude < INFINITY)) return W4A4_ERR_INVALID_ARG;
    if ((R->interleaved != 0 && R->interleaved != 1) || (R->inverse != 0 && R->inverse != 1)) return W4A4_ERR_INVALID_ARG;
    return reinterpret_cast<uintptr_t>(R->turns) & 7 ? W4A4_ERR_UNSUPPORTED_SHAPE : W4A4_OK;
}
inline RotaryArgs rotary_args(const w4a4_rotary_angles *R) { return RotaryArgs{R->turns, R->pairs, R->interleaved, R->magnitude, R->inverse}; }

// B: heads of a thread at once.
inline RotaryWork rotary_work(const void *x, int tokens, int heads, int features, long ldx, const int32_t *positions, const RotaryArgs &r, void *out, long ldo, int B) {
    RotaryWork a{static_cast<const uint16_t *>(x), static_cast<uint16_t *>(out), positions, ldx, ldo, tokens, heads, features, 0, 0, 0, 0, 0, r};
    a.way = r.interleaved ? kRotaryNeighbours : r.pairs % 8 == 0 ? kRotaryHalves8 : r.pairs % 4 == 0 && features % 4 == 0 ? kRotaryHalves4 : kRotarySingle;
    const int V = a.way == kRotarySingle ? 1 : a.way == kRotaryHalves4 ? 4 : 8, rest = features - 2 * r.pairs;
    a.paired = !r.interleaved && rest % (2 * V) == 0;
    a.units = r.interleaved ? features / 8 : r.pairs / V + (a.paired ? rest / 2 : rest) / V;                     // at most 255
    const int groups = 256 / a.units, want = (heads + B - 1) / B;
    a.side = want < groups ? want : groups;
    a.share = groups / a.side;
    return a;
}

// All tokens of `a`, which was made for `heads` (1 or 4) at once (rotary.hip).
int rotary_launch(const RotaryWork &a, int dtype, int heads, hipStream_t st);

}  // namespace w4a4
