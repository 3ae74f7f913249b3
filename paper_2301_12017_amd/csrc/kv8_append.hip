// New keys and values into the 8-bit cache, and rows of the cache back out.
//
// A block of a head has one scale: the largest magnitude that has been written into it since its first slot was, over 127.  A
// write whose range passes it raises the scale, and the codes that stay are re-scaled (code * old / new, to nearest even).
//
// The new tokens of one block stand together in `slots`, so a wave owns a (block, head) and one of keys or values: it finds the
// run of tokens, takes their range, settles the scale and writes, without atomics and without another wave to wait for.
// Keys are rows of D codes: eight features a lane, sixteen bytes in and eight out.  Values are stored by feature: a lane takes
// two neighbouring features (one where D is 64) of sixteen tokens and writes each feature's codes as one sixteen-byte
// piece of the block.  A run of at most sixteen tokens is read once, a longer one a second time out of L2.
//
// Long runs: 12005 tokens of 8 heads of 128 features in blocks of 16, fp16, 25 us = 2.9 TB/s of 74 MB (22 where the rows are in a cache).  A wave takes its runs one after the
// other, and in each the rows, their range, the scale and the codes are steps in series, of the keys with a load of the slot in front of
// each store; other waves fill in.  Reading them back 20.8 us = 3.5 TB/s (16).  Single tokens are latency, slots to scale to codes: 48 of 8 heads 4.5 us where
// most scales stay, 6.0 where all of them rise and their blocks are re-scaled (the long runs, of which few meet older codes: 2.1 more); 4.6 to read 832.
//
// With positions, keys are turned (rotary.hpp) on their way in, in fp32: what is stored is the turned key rounded once, to its code.  Workgroups of four waves take
// one, two or four heads, waves that have the same head share its runs, and all four find the angles of a step together, in LDS.  Queries are workgroups of the same launch.
// 48 single tokens of 8 heads of 128, 32 heads of queries: 6.6 us, slots beside positions to angles to range to codes in a chain.  12003 tokens of prompts in blocks of 16 36 us
// (without positions 25), with 32 heads of queries 70 to 76 = 3.6 TB/s: the steps of a run in series, where turning takes registers (three waves a SIMD, vector ALU 37 % busy).
#include "rotary.hpp"

namespace w4a4 {
namespace {

enum Positions { kNone, kKeys, kKeysAndQueries };                  // what turns on the way

constexpr int kPiece = 16;                                         // tokens of a run that a wave takes at once
constexpr int kQueryHeads = 4;                                     // of a thread, which share its angles

struct AppendArgs {
    int8_t *k, *v;
    float *k_scale, *v_scale;
    const uint16_t *x[2];                                          // new keys, new values
    long ld[2];
    const int32_t *slots;
    int T, blocks, H, shift, tile;
};
// (The append without positions is a call of few microseconds, and takes 0.1 of them less without these 144 bytes of arguments, of which it reads none: 200 single tokens 4.48 -> 4.37.)
struct TurningArgs : AppendArgs {
    int waves, window, query_tile;                                 // that share a run; tokens whose angles are there at once; tokens whose queries a workgroup turns
    const int32_t *positions;                                      // keys that turn
    RotaryArgs r;
    RotaryWork q;                                                  // the step's queries
};

// Code of x.  CAREFUL, where infinities or NaN are among the tokens: NaN is stored as 0, an infinity as +-127.  Else |x| is at most
// 127 scales but for a rounding, and adding 1.5 * 2^23 to x / scale rounds it to an integer (to nearest even), which is then the lowest byte.
template <bool CAREFUL>
__device__ __forceinline__ uint32_t code8(float x, float inv) {
    if constexpr (CAREFUL) {
        const float t = x * inv;                                   // (NaN also where an infinity meets a scale of 0)
        return t != t ? 0u : (uint32_t)(int)rintf(fminf(fmaxf(t, -127.0f), 127.0f));
    } else {
        return __builtin_bit_cast(uint32_t, x * inv + 12582912.0f);
    }
}
__device__ __forceinline__ uint32_t bytes4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {      // the lowest bytes
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u), 0x05040100u);
}

// Largest magnitude of sixteen-bit numbers, two a word, as their bits: above the pattern of infinity where one is a NaN.
typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));
struct Range {
    ushort2_t most = {0, 0};
    __device__ __forceinline__ void take(uint32_t w) { most = __builtin_elementwise_max(most, __builtin_bit_cast(ushort2_t, w & 0x7FFF7FFFu)); }
    __device__ __forceinline__ uint32_t over_wave() const {
        return lanes_reduce<64>((uint32_t)max(most[0], most[1]), [](uint32_t x, uint32_t y) { return x > y ? x : y; });
    }
};
template <bool BF16>
constexpr uint32_t kInf = BF16 ? 0x7F80 : 0x7C00;
template <bool BF16>
__device__ __forceinline__ uint32_t finite2(uint32_t w) {          // what does not count for a range, left out
    if ((w & 0x7FFFu) >= kInf<BF16>) w &= 0xFFFF0000u;
    if ((w >> 16 & 0x7FFFu) >= kInf<BF16>) w &= 0x0000FFFFu;
    return w;
}

// The scale of a unit (a head's block) that had the scale `had` after tokens of range `wide`; what stays of the block is re-scaled where it
// rises, by `waves` waves of which this is one.  Returns the scale's reciprocal.
__device__ __forceinline__ float settle(float *scale, float had, int8_t *codes, int bytes, bool first, float wide, int lane, int part = 0, int waves = 1) {
    const float was = first ? 0.0f : had;
    float now = fmaxf(was, wide / 127.0f);
    if (now < 1.1754943508e-38f) now = 0.0f;                       // (its reciprocal would not be a number)
    if (!first && now != was) {
        const float ratio = now > 0.0f ? was / now : 0.0f;
#pragma unroll 4
        for (int i = 16 * (lane + 64 * part); i < bytes; i += 16 * 64 * waves) {
            u32x4_t p = *reinterpret_cast<const u32x4_t *>(codes + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t c[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) c[e] = code8<false>((float)(int8_t)(p[j] >> (8 * e)), ratio);
                p[j] = bytes4(c[0], c[1], c[2], c[3]);
            }
            *reinterpret_cast<u32x4_t *>(codes + i) = p;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // the new codes, other lanes', come behind these
    }
    if (lane == 0 && part == 0 && now != had) *scale = now;
    return now > 0.0f ? 1.0f / now : 0.0f;
}

// Keys: tokens t0 .. t1-1 into the block's rows.
template <bool BF16, int D>
__device__ __forceinline__ void append_keys(const AppendArgs &a, int t0, int t1, int b, int h, bool first, int lane) {
    constexpr int LANES = D / 8, ROWS = 64 / LANES, N = (kPiece + ROWS - 1) / ROWS;   // lanes of a row, rows at once, loads of a chunk
    const int block = 1 << a.shift, row = lane / LANES;
    const bool on = row < ROWS;
    const uint16_t *x = a.x[0] + h * D + lane % LANES * 8;
    const size_t unit = (size_t)b * a.H + h;
    int8_t *codes = a.k + unit * D * block;
    const float had = a.k_scale[unit];
    u32x4_t w[N];
    auto load = [&](int c) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int t = c + i * ROWS + row;
            w[i] = u32x4_t{0, 0, 0, 0};
            if (on && t < t1) w[i] = *reinterpret_cast<const u32x4_t *>(x + t * a.ld[0]);
        }
    };
    auto range = [&](bool careful) {
        Range m;
        for (int c = t0; c < t1; c += N * ROWS) {
            load(c);
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) m.take(careful ? finite2<BF16>(w[i][j]) : w[i][j]);
        }
        return m.over_wave();
    };
    uint32_t wide = range(false);
    const bool careful = wide >= kInf<BF16>;
    if (careful) wide = range(true);
    const float inv = settle(a.k_scale + unit, had, codes, D * block, first, to_float<BF16>((uint16_t)wide), lane);
    auto write = [&](auto careful) {
        constexpr bool C = decltype(careful)::value;
        for (int c = t0; c < t1; c += N * ROWS) {
            if (t1 - t0 > N * ROWS) load(c);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int t = c + i * ROWS + row;
                if (!on || t >= t1) continue;
                uint32_t o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = code8<C>(to_float<BF16>((uint16_t)(w[i][j / 2] >> (16 * (j % 2)))), inv);
                *reinterpret_cast<u32x2_t *>(codes + (size_t)(a.slots[t] & (block - 1)) * D + lane % LANES * 8) =
                    u32x2_t{bytes4(o[0], o[1], o[2], o[3]), bytes4(o[4], o[5], o[6], o[7])};
            }
        }
    };
    if (careful) write(std::true_type{});
    else write(std::false_type{});
}

// Where an append has positions, `waves` (1, 2 or 4) of a workgroup's four share a run, chunk by chunk, and so a block of many tokens does not wait for one of them.
// All four take the same steps.
struct Share {
    int waves, part;                                               // this wave's part
    uint32_t *ranges;                                              // [2][4] in LDS
    // Largest `mine` of the waves that share; any: one of the workgroup's is `from` or more.
    __device__ __forceinline__ uint32_t most(uint32_t mine, int use, uint32_t from, bool &any) const {
        const int wave = threadIdx.x >> 6, first = wave & -waves;
        if ((threadIdx.x & 63) == 0) ranges[4 * use + wave] = mine;
        __syncthreads();
        any = false;
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = ranges[4 * use + i];
            any |= x >= from;                                      // (the same in every wave)
            if (i >= first && i < first + waves) mine = max(mine, x);
        }
        any = __builtin_amdgcn_readfirstlane(any);
        return __builtin_amdgcn_readfirstlane(mine);
    }
};

// Cosines and sines of the pairs of some tokens, and those tokens' positions, in LDS: found by all four waves of a workgroup together.
struct Window {
    float *cosines, *sines;                                        // [tokens][pairs]
    int *positions;
    uint64_t turns[2];                                             // of the lane's pairs
    int first, count;
    __device__ __forceinline__ void open(const TurningArgs &a, float *lds) {
        const int lane = threadIdx.x & 63, last = a.r.pairs - 1;
        cosines = lds;
        sines = lds + a.window * a.r.pairs;
        positions = reinterpret_cast<int *>(sines + a.window * a.r.pairs);
        first = count = 0;
        turns[0] = a.r.turns[min(lane, last)];
        turns[1] = a.r.turns[min(lane + 64, last)];
    }
    __device__ __forceinline__ void fill(const TurningArgs &a, int from, int tokens) {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), pairs = a.r.pairs;
        if (count) __syncthreads();                                // (the angles before have been read)
        first = from;
        count = min(tokens, a.T - from);                           // at most 64
        const int mine = a.positions[from + min(lane, count - 1)];
        if (wave == 0 && lane < count) positions[lane] = mine;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int p = lane + 64 * i;
            if (p >= pairs) break;
#pragma unroll 1
            for (int t = wave; t < count; t += 4) {
                const Turn turn = turn_of(turns[i], (uint32_t)__builtin_amdgcn_readlane(mine, t), a.r.magnitude, a.r.inverse);
                cosines[t * pairs + p] = turn.cos;
                sines[t * pairs + p] = turn.sin;
            }
        }
        __syncthreads();
    }
};

// The features d .. d+7 of a key (a lane's, in `to`), turned: cosines and sines of the token's pairs lie in LDS.  `other` holds their partners where pairs are
// halves and a multiple of eight; of other numbers of pairs they are fetched one by one (x: the lane's features).
template <bool BF16>
__device__ __forceinline__ void turn8(const RotaryArgs &r, u32x4_t other, const uint16_t *x, int d, const float *cosines, const float *sines, float (&to)[8]) {
    if (d >= 2 * r.pairs) return;
    if (r.pairs % 8 == 0) {                                        // angles four at a time
        const int p0 = r.interleaved ? d / 2 : d < r.pairs ? d : d - r.pairs;
        const float4_t *c = reinterpret_cast<const float4_t *>(cosines + p0), *s = reinterpret_cast<const float4_t *>(sines + p0);
        if (r.interleaved) {
            const float4_t cs = c[0], sn = s[0];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Turn t{cs[j], sn[j]};
                const float u = to[2 * j], v = to[2 * j + 1];
                to[2 * j] = turned_a(t, u, v);
                to[2 * j + 1] = turned_b(t, u, v);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const Turn t{c[j / 4][j % 4], s[j / 4][j % 4]};
                const float v = to_float<BF16>((uint16_t)(other[j / 2] >> (16 * (j % 2))));
                to[j] = d < r.pairs ? turned_a(t, to[j], v) : turned_b(t, v, to[j]);
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int f = d + j, p = r.interleaved ? f / 2 : f < r.pairs ? f : f - r.pairs;
        if (f >= 2 * r.pairs) break;
        const Turn t{cosines[p], sines[p]};
        if (r.interleaved) {
            if (j % 2) continue;
            const float u = to[j], v = to[j + 1];
            to[j] = turned_a(t, u, v);
            to[j + 1] = turned_b(t, u, v);
        } else {
            const float v = to_float<BF16>(x[f < r.pairs ? j + r.pairs : j - r.pairs]);
            to[j] = f < r.pairs ? turned_a(t, to[j], v) : turned_b(t, v, to[j]);
        }
    }
}

// Tokens of a run that a wave turns at once, and waves that may share one (us at 2 | 4: 30000 tokens of 2 heads of 64 in blocks of 128 32 | 43, 12003 of 8 of 128 in
// blocks of 64 49 | 64; 4000 of 2 heads of 256, whose chunks are shorter, in blocks of 64 37 | 28).
template <int D>
struct Turning {
    static constexpr int LANES = D / 8, ROWS = 64 / LANES, N = D == 64 ? 2 : 4, CHUNK = N * ROWS;    // lanes of a row, rows at once, loads of a chunk
    static constexpr int WAVES = D == 256 ? 4 : 2;
};

// Keys with positions: tokens t0 .. t1-1 into the block's rows (h past the last head: nothing, but in step).
template <bool BF16, int D>
__device__ __forceinline__ void append_turned_keys(const TurningArgs &a, int t0, int t1, int b, int h, bool first, int lane, Window &window, const Share &share) {
    constexpr int LANES = Turning<D>::LANES, ROWS = Turning<D>::ROWS, N = Turning<D>::N, CHUNK = Turning<D>::CHUNK;
    const int block = 1 << a.shift, row = min(lane / LANES, ROWS - 1), d = lane % LANES * 8, pairs = a.r.pairs, step = share.waves * CHUNK;
    const bool there = h < a.H, on = lane / LANES < ROWS && there;
    if (!there) h = 0;
    const uint16_t *x = a.x[0] + h * D + d;
    const size_t unit = (size_t)b * a.H + h;
    int8_t *codes = a.k + unit * D * block;
    float had = a.k_scale[unit], turned[N][8], inv = 0.0f;
    int slots[N];
    auto load = [&](int s) {                                       // the wave's chunk of the step from token s on (rows that are not there: the last one again)
        const int c = s + share.part * CHUNK + row;
        auto at = [&](int i) { return x + min(c + i * ROWS, t1 - 1) * a.ld[0]; };
        u32x4_t w[N], other[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            w[i] = *reinterpret_cast<const u32x4_t *>(at(i));
            slots[i] = a.slots[min(c + i * ROWS, t1 - 1)];
        }
        if (!a.r.interleaved && pairs % 8 == 0) {
            const int to = d < pairs ? pairs : d < 2 * pairs ? -pairs : 0;
#pragma unroll
            for (int i = 0; i < N; ++i) other[i] = *reinterpret_cast<const u32x4_t *>(at(i) + to);
        }
        if (s < window.first || min(s + step, t1) > window.first + window.count) window.fill(a, s, a.window);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int t = c + i * ROWS, from = min(t, t1 - 1) - window.first;
#pragma unroll
            for (int j = 0; j < 8; ++j) turned[i][j] = to_float<BF16>((uint16_t)(w[i][j / 2] >> (16 * (j % 2))));
            if (window.positions[from] >= 0) turn8<BF16>(a.r, other[i], at(i), d, window.cosines + from * pairs, window.sines + from * pairs, turned[i]);
            if (!on || t >= t1)
#pragma unroll
                for (int j = 0; j < 8; ++j) turned[i][j] = 0.0f;
            __builtin_amdgcn_sched_barrier(0);                     // (angles of more rows are more registers than there are)
        }
    };
    // the run's range, that of its finite numbers where there are others (the bits of fp32 numbers), its codes
    enum { kRange, kFinite, kWrite } pass = kRange;
    bool careful = false, none;
    uint32_t most = 0;
    for (;;) {
        for (int s = t0; s < t1; s += step) {
            if (pass == kRange || t1 - t0 > step) load(s);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (pass != kWrite) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t bits = __builtin_bit_cast(uint32_t, turned[i][j]) & 0x7FFFFFFFu;
                        most = max(most, pass == kFinite && bits >= 0x7F800000u ? 0u : bits);
                    }
                } else if (on && s + share.part * CHUNK + i * ROWS + row < t1) {
                    uint32_t o[8];
                    if (careful) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] = code8<true>(turned[i][j], inv);
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] = code8<false>(turned[i][j], inv);
                    }
                    *reinterpret_cast<u32x2_t *>(codes + (size_t)(slots[i] & (block - 1)) * D + d) = u32x2_t{bytes4(o[0], o[1], o[2], o[3]), bytes4(o[4], o[5], o[6], o[7])};
                }
            }
        }
        if (pass == kWrite) break;
        most = lanes_reduce<64>(most, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
        asm volatile("" : "+v"(had));                              // (has been read before another wave writes it)
        if (pass == kRange) {
            most = share.most(most, 0, 0x7F800000u, careful);
            if (careful) {
                pass = kFinite;
                most = 0;
                continue;
            }
        } else {
            most = share.most(most, 1, ~0u, none);
        }
        if (there) inv = settle(a.k_scale + unit, had, codes, D * block, first, __builtin_bit_cast(float, most), lane, share.part, share.waves);
        __syncthreads();                                           // (the block's old codes are re-scaled)
        pass = kWrite;
    }
}

// Values: tokens t0 .. t1-1 into the block's columns.  ordered: their slots follow each other, from slot `off` of the block on.  SHARED: by the waves that
// share a run (h past the last head: nothing, but in step).
template <bool BF16, int D, bool SHARED>
__device__ __forceinline__ void append_values(const AppendArgs &a, int t0, int t1, int b, int h, bool first, bool ordered, int off, int lane, const Share &share) {
    constexpr int F = D == 64 ? 1 : 2, N = D == 256 ? 2 : 1;       // neighbouring features a lane, and times that
    constexpr int FEW = 4;                                         // tokens below which codes are stored byte by byte
    const int block = 1 << a.shift;
    const bool there = !SHARED || h < a.H, on = lane * F < D && there;
    if (!there) h = 0;
    const uint16_t *x = a.x[1] + h * D + (on ? lane * F : 0);      // (lanes without a feature: the first one again)
    const size_t unit = (size_t)b * a.H + h;
    int8_t *codes = a.v + unit * D * block;
    float had = a.v_scale[unit];
    uint32_t w[N][kPiece];
    auto load = [&](int t, int i) {                                // the lane's features of token t
#pragma unroll
        for (int n = 0; n < N; ++n) w[n][i] = F == 2 ? *reinterpret_cast<const uint32_t *>(x + t * a.ld[1] + 128 * n) : x[t * a.ld[1]];
    };
    // pieces of sixteen slots of the block where the tokens are in order: the first token's place in its piece comes first
    const bool few = t1 - t0 < FEW;
    const int c0 = ordered && !few ? t0 - (off & (kPiece - 1)) : t0, mine = SHARED ? c0 + kPiece * share.part : c0, step = SHARED ? kPiece * share.waves : kPiece;
    auto chunk = [&](int c) {                                      // tokens c .. c + 15; the run's first and last one again where it has none
        if (few) {
#pragma unroll
            for (int i = 0; i < FEW - 1; ++i) load(min(t0 + i, t1 - 1), i);
        } else {
#pragma unroll
            for (int i = 0; i < kPiece; ++i) load(min(max(c + i, t0), t1 - 1), i);
        }
    };
    auto range = [&](bool careful) {
        Range m;
        for (int c = mine; c < t1; c += step) {
            if (!careful || t1 - c0 > step) chunk(c);
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                if (i >= FEW - 1 && few) break;
#pragma unroll
                for (int n = 0; n < N; ++n) m.take(careful ? finite2<BF16>(w[n][i]) : w[n][i]);
            }
        }
        return m.over_wave();
    };
    uint32_t wide = range(false);
    bool careful = wide >= kInf<BF16>, none;
    if constexpr (SHARED) {
        asm volatile("" : "+v"(had));                              // (has been read before another wave writes it)
        wide = share.most(wide, 0, kInf<BF16>, careful);
    }
    if (careful) {
        wide = range(true);
        if constexpr (SHARED) wide = share.most(wide, 1, ~0u, none);
    }
    float inv = 0.0f;
    if (there) inv = settle(a.v_scale + unit, had, codes, D * block, first, to_float<BF16>((uint16_t)wide), lane, SHARED ? share.part : 0, SHARED ? share.waves : 1);
    if constexpr (SHARED) __syncthreads();                         // (the block's old codes are re-scaled)
    auto write = [&](auto careful) {
        constexpr bool C = decltype(careful)::value;
        auto code = [&](int n, int f, int i) { return code8<C>(to_float<BF16>((uint16_t)(w[n][i] >> (16 * f))), inv); };
        if (few) {
            if (SHARED && share.part) return;
#pragma unroll
            for (int i = 0; i < FEW - 1; ++i)
                if (t0 + i < t1) {
                    int8_t *to = codes + (a.slots[t0 + i] & (block - 1));
#pragma unroll
                    for (int n = 0; n < N; ++n)
#pragma unroll
                        for (int f = 0; f < F; ++f)
                            if (on) to[(size_t)(128 * n + lane * F + f) * block] = (int8_t)code(n, f, i);
                }
            return;
        }
        for (int c = mine; c < t1; c += step) {
            if (t1 - c0 > step) chunk(c);
            const int lo = max(t0 - c, 0), hi = min(t1 - c, kPiece);                     // tokens lo .. hi-1 of the chunk
            const int at = ordered ? off + (c - t0) : 0;           // (a multiple of 16) slot of the chunk's first token
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    int8_t *to = codes + (size_t)(128 * n + lane * F + f) * block;
                    u32x4_t o;
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = bytes4(code(n, f, 4 * j), code(n, f, 4 * j + 1), code(n, f, 4 * j + 2), code(n, f, 4 * j + 3));
                    if (ordered && hi - lo == kPiece) {
                        if (on) *reinterpret_cast<u32x4_t *>(to + at) = o;
                    } else if (ordered && hi - lo >= FEW) {
                        if (on) {
                            const u32x4_t old = *reinterpret_cast<const u32x4_t *>(to + at);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                uint32_t mask = 0;
#pragma unroll
                                for (int e = 0; e < 4; ++e) mask |= (4 * j + e >= lo && 4 * j + e < hi ? 0xFFu : 0u) << (8 * e);
                                o[j] = (o[j] & mask) | (old[j] & ~mask);
                            }
                            *reinterpret_cast<u32x4_t *>(to + at) = o;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < kPiece; ++i)
                            if (i >= lo && i < hi && on) to[a.slots[c + i] & (block - 1)] = (int8_t)(o[i / 4] >> (8 * (i % 4)));
                    }
                }
        }
    };
    if (careful) write(std::true_type{});
    else write(std::false_type{});
}

// Waves a SIMD: turning keys takes up to 168 registers, three of them.  Heads of 256 keep 11 to 13 of theirs in scratch memory for that, which is still the faster way (us by
// three | two waves, two heads: 3000 tokens in blocks of 32 12 | 16, 12003 in blocks of 16 22.5 | 23.6, 4000 in blocks of 64 22.8 | 21.6), and all keep 90 to 125 scalar ones in
// lanes of a vector register.  Without positions heads of 96 need 93 where they are told to, and five waves run; by themselves they take 97.
template <bool BF16, int D, Positions POSITIONS>
__global__ __launch_bounds__(256, POSITIONS != kNone ? 3 : D == 96 ? 5 : 1) void kv8_append_kernel(std::conditional_t<POSITIONS == kNone, AppendArgs, TurningArgs> a) {
    constexpr bool ROTARY = POSITIONS != kNone;
    extern __shared__ __attribute__((aligned(16))) float angles[]; // ROTARY: a window's
    __shared__ uint32_t ranges[8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int which, tile = blockIdx.x;                                  // 0 .. H-1: keys of a head, H .. 2H-1: values
    bool values;
    Window window;
    Share share{1, 0, ranges};
    if constexpr (ROTARY) {                                        // workgroups of some heads' keys, all tiles of them, then of values, then of queries
        const int tiles = (a.T + a.tile - 1) / a.tile, heads = 4 / a.waves, groups = (a.H + heads - 1) / heads, group = blockIdx.x / tiles;
        if (POSITIONS == kKeysAndQueries && group >= 2 * groups) {
            const int t0 = ((int)blockIdx.x - 2 * groups * tiles) * a.query_tile, count = min(a.query_tile, a.T - t0);
            switch (a.q.way) {
                case kRotaryNeighbours: return rotary_tokens<BF16, kRotaryNeighbours, kQueryHeads>(a.q, t0, count);
                case kRotaryHalves8: return rotary_tokens<BF16, kRotaryHalves8, kQueryHeads>(a.q, t0, count);
                case kRotaryHalves4: return rotary_tokens<BF16, kRotaryHalves4, kQueryHeads>(a.q, t0, count);
                default: return rotary_tokens<BF16, kRotarySingle, kQueryHeads>(a.q, t0, count);
            }
        }
        tile -= group * tiles;
        values = group >= groups;
        which = (group - (values ? groups : 0)) * heads + wave / a.waves;
        share.waves = a.waves;
        share.part = wave & (a.waves - 1);
        if (!values) window.open(a, angles);
    } else {
        which = __builtin_amdgcn_readfirstlane(blockIdx.y * 4 + wave);
        if (which >= 2 * a.H) return;
        values = which >= a.H;
        if (values) which -= a.H;
    }
    const int t_first = tile * a.tile, t_last = min(t_first + a.tile, a.T), mask = (1 << a.shift) - 1;
    auto block_of = [&](int slot) { return slot >= 0 && (slot >> a.shift) < a.blocks ? slot >> a.shift : -1; };   // -1: not stored
    // slots of the token before the tile and of the 63 from its first one on; where runs begin; where a slot does not follow the one before
    const int at = t_first - 1 + lane, read = a.slots[min(max(at, 0), a.T - 1)];
    if constexpr (ROTARY)
        if (!values && a.tile == 1) window.fill(a, t_first, 1);    // (while the slots are on their way)
    const int slot = at >= 0 && at < a.T ? read : -1, b = block_of(slot);
    const int b_before = __shfl_up(b, 1, 64), slot_before = __shfl_up(slot, 1, 64);
    const unsigned long long begins = __ballot(lane > 0 && b != b_before), jumps = __ballot(lane > 0 && slot != slot_before + 1);
    const unsigned long long firsts = __ballot(b >= 0 && (slot & mask) == 0);
    for (int i = 1; i <= t_last - t_first; ++i) {
        const int bi = __builtin_amdgcn_readlane(b, i), t0 = t_first - 1 + i;
        if (bi < 0 || !(begins >> i & 1)) continue;                // (not the first token of a run)
        const unsigned long long after = i < 63 ? begins >> (i + 1) << (i + 1) : 0;
        const int end = after ? __builtin_ctzll(after) : 64;       // (lane behind the run, or the run goes on behind the lanes)
        const unsigned long long in = (end < 64 ? (1ull << end) - 1 : ~0ull) & ~((1ull << i) - 1);
        bool first = (firsts & in) != 0, ordered = !(jumps & in & ~(1ull << i));
        int t1 = t_first - 1 + end;
        if (end == 64) {                                           // a long run: on with windows of 64
            int before = __builtin_amdgcn_readlane(slot, 63);
            for (;; t1 += 64) {
                const int s = t1 + lane < a.T ? a.slots[t1 + lane] : -1;
                int ahead = __shfl_up(s, 1, 64);
                if (lane == 0) ahead = before;
                const unsigned long long out = __ballot(block_of(s) != bi);
                const unsigned long long same = out ? (1ull << __builtin_ctzll(out)) - 1 : ~0ull;
                first |= (__ballot((s & mask) == 0) & same) != 0;
                ordered &= !(__ballot(s != ahead + 1) & same);
                before = __builtin_amdgcn_readlane(s, 63);
                if (out) {
                    t1 += __builtin_ctzll(out);
                    break;
                }
            }
        }
        const int off = __builtin_amdgcn_readlane(slot, i) & mask;
        if (values) append_values<BF16, D, ROTARY>(a, t0, t1, bi, which, first, ordered, off, lane, share);
        else if constexpr (ROTARY) append_turned_keys<BF16, D>(a, t0, t1, bi, which, first, lane, window, share);
        else append_keys<BF16, D>(a, t0, t1, bi, which, first, lane);
    }
}

struct ReadArgs {
    const int8_t *k, *v;
    const float *k_scale, *v_scale;
    uint16_t *out[2];
    const int32_t *slots;
    int T, blocks, H, shift;
};

// TILE tokens of a head's keys or values by a wave.  Values of tokens that follow each other lie in one or two pieces of a block, which
// are fetched whole; else each token's codes are fetched by themselves.
template <bool BF16, int D, int TILE>
__global__ __launch_bounds__(256) void kv8_read_kernel(ReadArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int which = __builtin_amdgcn_readfirstlane(blockIdx.y * 4 + wave), block = 1 << a.shift;
    if (which >= 2 * a.H) return;
    const bool val = which >= a.H;
    const int h = val ? which - a.H : which, t0 = blockIdx.x * TILE;
    const float *scales = val ? a.v_scale : a.k_scale;
    uint16_t *out = a.out[val] + h * D;
    if (!val) {
        constexpr int LANES = D / 16, ROWS = 64 / LANES, N = (TILE + ROWS - 1) / ROWS;
        const int row = lane / LANES, d = lane % LANES * 16;
        u32x4_t w[N];
        float scale[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int t = t0 + i * ROWS + row, slot = t < a.T ? a.slots[t] : -1;
            w[i] = u32x4_t{0, 0, 0, 0};
            scale[i] = 0.0f;
            if (slot >= 0 && (slot >> a.shift) < a.blocks) {
                const size_t unit = (size_t)(slot >> a.shift) * a.H + h;
                w[i] = *reinterpret_cast<const u32x4_t *>(a.k + (unit * block + (slot & (block - 1))) * D + d);
                scale[i] = scales[unit];
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int t = t0 + i * ROWS + row;
            if (row >= ROWS || i * ROWS + row >= TILE || t >= a.T) continue;
            u32x4_t o[2];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t c = w[i][j / 2] >> (16 * (j % 2));
                o[j / 4][j % 4] = from_float<BF16>((float)(int8_t)c * scale[i]) | (uint32_t)from_float<BF16>((float)(int8_t)(c >> 8) * scale[i]) << 16;
            }
            u32x4_t *to = reinterpret_cast<u32x4_t *>(out + (size_t)t * a.H * D + d);
            to[0] = o[0];
            to[1] = o[1];
        }
        return;
    }
    constexpr int F = D == 64 ? 1 : 2, N = D == 256 ? 2 : 1;       // neighbouring features a lane, and times that
    const bool on = lane * F < D;
    const int mine = lane < TILE && t0 + lane < a.T ? a.slots[t0 + lane] : -1;       // the slots, one a lane
    const bool there = mine >= 0 && (mine >> a.shift) < a.blocks;
    const int n = min(TILE, a.T - t0), s0 = __builtin_amdgcn_readlane(mine, 0), s1 = __builtin_amdgcn_readlane(mine, n - 1);
    const bool two = __ballot(lane < n && (!there || (mine >> 4 != s0 >> 4 && mine >> 4 != s1 >> 4))) == 0;
    auto address = [&](int slot, int f) { return a.v + (((size_t)(slot >> a.shift) * a.H + h) * D + f) * block + (slot & (block - 1)); };
    const float scale = there ? scales[(size_t)(mine >> a.shift) * a.H + h] : 0.0f;
    int8_t c[N][F][TILE];
    if (two) {
        u32x4_t p[2][N][F];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int m = 0; m < N; ++m)
#pragma unroll
                for (int f = 0; f < F; ++f)
                    p[k][m][f] = *reinterpret_cast<const u32x4_t *>(address((k ? s1 : s0) & ~15, on ? 128 * m + lane * F + f : 0));
#pragma unroll
        for (int i = 0; i < TILE; ++i) {
            const int s = __builtin_amdgcn_readlane(mine, i);      // (behind the tokens: some byte of the pieces, not written)
            const bool second = s >> 4 != s0 >> 4;
#pragma unroll
            for (int m = 0; m < N; ++m)
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    const u32x4_t q = second ? p[1][m][f] : p[0][m][f];
                    const uint32_t lo = s & 4 ? q[1] : q[0], hi = s & 4 ? q[3] : q[2];
                    c[m][f][i] = (int8_t)((s & 8 ? hi : lo) >> (8 * (s & 3)));
                }
        }
    } else {
#pragma unroll
        for (int i = 0; i < TILE; ++i) {
            const int s = __builtin_amdgcn_readlane(mine, i);
#pragma unroll
            for (int m = 0; m < N; ++m)
#pragma unroll
                for (int f = 0; f < F; ++f) c[m][f][i] = 0;
            if (s >= 0 && (s >> a.shift) < a.blocks && on)
#pragma unroll
                for (int m = 0; m < N; ++m)
#pragma unroll
                    for (int f = 0; f < F; ++f) c[m][f][i] = *address(s, 128 * m + lane * F + f);
        }
    }
#pragma unroll
    for (int i = 0; i < TILE; ++i) {
        const float by = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scale), i));
        if (i >= n || !on) continue;
#pragma unroll
        for (int m = 0; m < N; ++m) {
            uint16_t *to = out + (size_t)(t0 + i) * a.H * D + 128 * m + lane * F;
            const uint32_t y = from_float<BF16>((float)c[m][0][i] * by);
            if constexpr (F == 2) *reinterpret_cast<uint32_t *>(to) = y | (uint32_t)from_float<BF16>((float)c[m][1][i] * by) << 16;
            else *to = (uint16_t)y;
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

namespace {

// What both entry points ask of keys, values and slots.
int rows_check(const w4a4_kv8_cache *C, const void *K, const void *V, int dtype, int tokens, int ldk, int ldv, const int32_t *slots) {
    if (const int rc = kv8_cache_check(C)) return rc;
    if (tokens < 0 || (dtype != W4A4_F16 && dtype != W4A4_BF16)) return W4A4_ERR_INVALID_ARG;
    const int row = C->heads * C->features;
    if (ldk < row || ldv < row) return W4A4_ERR_INVALID_ARG;
    if (tokens == 0) return W4A4_OK;
    if (!K || !V || !slots) return W4A4_ERR_INVALID_ARG;
    if (ldk % 8 || ldv % 8 || !aligned16(K) || !aligned16(V)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    return W4A4_OK;
}

template <Positions POSITIONS>
int append(const w4a4_kv8_cache *C, const void *K, const void *V, int dtype, int tokens, int ldk, int ldv, const int32_t *slots, const int32_t *positions,
           const RotaryArgs &r, const RotaryWork &q, hipStream_t st) {
    std::conditional_t<POSITIONS == kNone, AppendArgs, TurningArgs> a;
    static_cast<AppendArgs &>(a) = {C->k, C->v, C->k_scale, C->v_scale, {static_cast<const uint16_t *>(K), static_cast<const uint16_t *>(V)}, {ldk, ldv},
                                    slots, tokens, C->blocks, C->heads, __builtin_ctz(C->block), tokens <= 512 ? 1 : kPiece};
    return by_features(C->features, [&](auto d) {
        constexpr int D = decltype(d)::value, CHUNK = Turning<D>::CHUNK, WAVES = Turning<D>::WAVES;
        static_assert(WAVES * CHUNK <= 64, "a lane each");
        size_t lds = 0;
        dim3 grid((tokens + a.tile - 1) / a.tile, (2 * C->heads + 3) / 4);
        if constexpr (POSITIONS != kNone) {
            a.positions = positions;
            a.r = r;
            a.q = q;
            const int share = C->block / (D == 256 ? 8 : 16);
            a.waves = share < WAVES ? share : WAVES;
            // (a workgroup for a token each: sharing leaves few of its waves something to do, so not where there are many; 200 tokens of 8 heads of 64 13 us shared, 8 not)
            if (a.tile == 1 && (long)tokens * C->heads * a.waves > 2048) a.waves = 1;
            a.window = a.waves * CHUNK;
            lds = (size_t)a.window * (2 * r.pairs + 1) * sizeof(float);                 // at most 33 KB
            // Tokens of a workgroup, whose runs it takes one after the other.  Where there are thousands, prompts are among them, and most workgroups of sixteen would meet
            // no first token of a block (us at 16 | at most 63: 30000 tokens of 2 heads of 64 in blocks of 128 77 | 32); some hundreds may be requests of one token each (us
            // at 16 | this: 600 of those, 8 heads of 128 in blocks of 16 61 | 21, 1000 of 64 43 | 36; prompts of 600 and 1000 tokens 10.8 | 13.3 and 13.5 | 15.6).
            const int heads = 4 / a.waves, groups = (C->heads + heads - 1) / heads, few = tokens / 128;
            if (tokens > 512 && few < kPiece) a.tile = few;
            if (tokens >= 4096) a.tile = C->block < 63 ? C->block : 63;
            a.query_tile = tokens <= 512 ? 1 : 16;
            const long tiles = (tokens + (long)a.tile - 1) / a.tile, all = tiles * 2 * groups + (POSITIONS == kKeysAndQueries ? (tokens + (long)a.query_tile - 1) / a.query_tile : 0);
            if (!grid_fits(all, 256)) return (int)W4A4_ERR_UNSUPPORTED_SHAPE;
            grid = dim3((unsigned)all);
        }
        if (dtype == W4A4_BF16) hipLaunchKernelGGL((kv8_append_kernel<true, D, POSITIONS>), grid, dim3(256), lds, st, a);
        else hipLaunchKernelGGL((kv8_append_kernel<false, D, POSITIONS>), grid, dim3(256), lds, st, a);
        return launch_status();
    });
}

}  // namespace

extern "C" int w4a4_kv8_append(const w4a4_kv8_cache *C, const void *K, const void *V, int dtype, int tokens, int ldk, int ldv,
                               const int32_t *slots, void *stream) {
    if (const int rc = rows_check(C, K, V, dtype, tokens, ldk, ldv, slots)) return rc;
    if (tokens == 0) return W4A4_OK;
    return append<kNone>(C, K, V, dtype, tokens, ldk, ldv, slots, nullptr, RotaryArgs{}, RotaryWork{}, as_stream(stream));
}

extern "C" int w4a4_kv8_append_rotary(const w4a4_kv8_cache *C, const w4a4_kv8_rows *T, const w4a4_rotary_angles *R, void *stream) {
    if (!T) return W4A4_ERR_INVALID_ARG;
    if (const int rc = rows_check(C, T->k, T->v, T->dtype, T->tokens, T->ldk, T->ldv, T->slots)) return rc;
    if (const int rc = rotary_check(R, C->features)) return rc;
    if (T->q && (T->heads <= 0 || (long)T->heads * C->features > T->ldq)) return W4A4_ERR_INVALID_ARG;
    if (T->tokens == 0) return W4A4_OK;
    if (!T->positions || !T->q != !T->q_out || (T->q && T->q == T->q_out)) return W4A4_ERR_INVALID_ARG;
    if (T->q && (T->ldq % 8 || !aligned16(T->q) || !aligned16(T->q_out))) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const RotaryArgs r = rotary_args(R);
    hipStream_t st = as_stream(stream);
    auto keys = [&](auto positions, const RotaryWork &q) {
        return append<decltype(positions)::value>(C, T->k, T->v, T->dtype, T->tokens, T->ldk, T->ldv, T->slots, T->positions, r, q, st);
    };
    if (!T->q) return keys(std::integral_constant<Positions, kKeys>{}, RotaryWork{});
    return keys(std::integral_constant<Positions, kKeysAndQueries>{},
                rotary_work(T->q, T->tokens, T->heads, C->features, T->ldq, T->positions, r, T->q_out, (long)T->heads * C->features, kQueryHeads));
}

extern "C" int w4a4_kv8_read(const w4a4_kv8_cache *C, const int32_t *slots, int tokens, int dtype, void *K, void *V, void *stream) {
    if (const int rc = kv8_cache_check(C)) return rc;
    if (tokens < 0 || (dtype != W4A4_F16 && dtype != W4A4_BF16)) return W4A4_ERR_INVALID_ARG;
    if (tokens == 0) return W4A4_OK;
    if (!slots || !K || !V) return W4A4_ERR_INVALID_ARG;
    if (!aligned16(K) || !aligned16(V)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const ReadArgs a{C->k, C->v, C->k_scale, C->v_scale, {static_cast<uint16_t *>(K), static_cast<uint16_t *>(V)}, slots, tokens,
                     C->blocks, C->heads, __builtin_ctz(C->block)};
    // Four tokens a wave while that leaves waves to spare.  us at 4 | 16, 832 tokens of 8 heads of 128: 4.6 | 6.8.
    const bool few = tokens <= 4096;
    const dim3 grid((tokens + (few ? 3 : 15)) / (few ? 4 : 16), (2 * C->heads + 3) / 4);
    return by_features(C->features, [&](auto d) {
        constexpr int D = decltype(d)::value;
        auto run = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, as_stream(stream), a); };
        if (dtype == W4A4_BF16) few ? run(kv8_read_kernel<true, D, 4>) : run(kv8_read_kernel<true, D, 16>);
        else few ? run(kv8_read_kernel<false, D, 4>) : run(kv8_read_kernel<false, D, 16>);
        return launch_status();
    });
}
