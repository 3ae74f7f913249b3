// What the two kernels of attention over the 8-bit cache share (gfx950): arguments, rows and keys of a tile, codes as fp16 numbers.
#pragma once
#include "gen.hpp"

namespace w4a4 {

constexpr int kStep = 64;                                          // keys of a step
constexpr int kSlots = 512, kMostGroups = 4096;                    // pieces of few groups, and groups that are cut, at most
constexpr int kCounters = kSlots + kMostGroups;                    // in the workspace
// Rows of a request and head that kv8_attention.hip takes, in tiles that read the keys again.  us there | by kv8_prompt.hip, 8 key heads of 128: 36 or 64
// rows, 32 requests of 1000 keys 32 | 52, one of 20000 34 | 58, 200 of 1000 208 | 200; 96 rows, 32 of 1000 47 | 54, 8 of 5000 65 | 64, 200 of 1000 310 | 220.
constexpr int kFewRows = 64;
// Requests from which on a call whose bound allows more rows launches both kernels, each for its requests.  us both | only the one for many rows,
// 8 key heads of 128, groups of 4: 4 requests of 4000 keys, 100 queries and three single ones 50 | 58, all of 300 queries 157 | 152; 64 of
// 2000, 1500 queries and 63 single ones 160 | 220.  (With fewer requests a single token beside a prompt is one useful wave of eight; that was not measured
// over a long cache.)
constexpr int kMixed = 4;

// n / d for n * d < 2^32, one multiplication (a division by a number that the kernel gets costs some forty instructions).
struct Div {
    uint64_t by;
    int d;
    explicit Div(int d) : by(((1ull << 32) + d - 1) / d), d(d) {}
    __device__ __forceinline__ int of(int n) const { return (int)(((uint64_t)(uint32_t)n * by) >> 32); }
    __device__ __forceinline__ int rest(int n, int q) const { return n - q * d; }
};

struct AttnArgs {
    const uint16_t *q;
    const int8_t *k, *v;
    const float *k_scale, *v_scale;
    const int32_t *table, *lens, *start;
    uint16_t *out;
    float *lse, *po, *pml;                                         // pieces of groups: [workgroup][row][D] and [..][row][2]
    int *arrived;
    long ldq;
    int tokens, blocks, H, shift, width, window, queries, requests, slots;
    int least, most;                                               // rows of a request that this kernel takes; others are another's
    Div group, tiles, heads;                                       // queries of a head of the cache; tiles of a request; = H
    float scale;                                                   // in powers of two: scale / ln 2
};

// Queries (0 where another kernel takes them) and keys of a request.
struct Sizes { int n, len; };
__device__ __forceinline__ Sizes sizes_of(const AttnArgs &a, int r) {
    const int n = max(min(min(a.start[r + 1], a.tokens) - max(a.start[r], 0), a.queries), 0), rows = n * a.group.d;
    const long room = (long)a.width << a.shift;
    return Sizes{rows >= a.least && rows <= a.most ? n : 0, min(max(a.lens[r], 0), room < 0x7fffff00L ? (int)room : 0x7fffff00)};
}
// The rows of a group and the keys they see.
struct Tile {
    int first, n, len, rows, row0;                                 // first token, queries, keys of the request; rows of it; this tile's first
    int begin, end;                                                // keys that any row of the tile sees
    int steps;                                                     // 0: no rows; else one at least
};
__device__ __forceinline__ Tile tile_of(const AttnArgs &a, Sizes s, int row0, int tile) {
    Tile t;
    t.first = 0;
    t.n = s.n;
    t.len = s.len;
    t.rows = s.n * a.group.d;
    t.row0 = row0;
    t.begin = t.end = t.steps = 0;
    if (row0 < t.rows) {
        const int lo = t.len - t.n + a.group.of(row0), hi = t.len - t.n + a.group.of(min(row0 + tile, t.rows) - 1);
        t.end = max(hi + 1, 0);
        t.begin = a.window ? min(max(lo - a.window + 1, 0), t.end) : 0;
        t.steps = t.end > t.begin ? (t.end - (t.begin & ~(kStep - 1)) + kStep - 1) / kStep : 1;
    }
    return t;
}
__device__ __forceinline__ Tile tile_of(const AttnArgs &a, int r, int row0, int tile) {
    Tile t = tile_of(a, sizes_of(a, r), row0, tile);
    t.first = max(a.start[r], 0);
    return t;
}

template <typename Op>
__device__ __forceinline__ float over_groups(float x, Op op) {     // op over the lanes l % 16 + 16 g, in all of them
    auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    x = op(__builtin_bit_cast(float, (unsigned)s[0]), __builtin_bit_cast(float, (unsigned)s[1]));
    s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return op(__builtin_bit_cast(float, (unsigned)s[0]), __builtin_bit_cast(float, (unsigned)s[1]));
}
__device__ __forceinline__ float max2(float x, float y) { return fmaxf(x, y); }
__device__ __forceinline__ float add2(float x, float y) { return x + y; }

// four codes of a word as four halves
__device__ __forceinline__ u32x2_t codes4(uint32_t w) {
    w ^= 0x80808080u;
    const half2_t off = {(_Float16)1152.0f, (_Float16)1152.0f};
    const half2_t a = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) - off;
    const half2_t b = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) - off;
    return u32x2_t{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
}
__device__ __forceinline__ u32x4_t codes8(uint32_t w0, uint32_t w1) {
    const u32x2_t a = codes4(w0), b = codes4(w1);
    return u32x4_t{a[0], a[1], b[0], b[1]};
}
__device__ __forceinline__ uint32_t pack_halves(float a, float b) {
    return __builtin_bit_cast(uint32_t, half2_t{(_Float16)a, (_Float16)b});
}
__device__ __forceinline__ float power(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }   // 2^e, -126 <= e <= 127

// log(2^m * sum).  The exponent of the sum is added to m first, which rounds nothing: the two may be large and of different signs.
__device__ __forceinline__ float log_sum(float m, float sum) {
    const float whole = m + (float)__builtin_amdgcn_frexp_expf(sum);
    return sum != 0.0f ? (whole + log2f(__builtin_amdgcn_frexp_mantf(sum))) * 0.69314718056f : -INFINITY;
}

// Pieces of `piece` steps that `steps` < 2^26 make: at least enough (where steps are millions, one or two more, which are then empty), the same
// for all who ask.  By a reciprocal: an integer division is 40 instructions.
__device__ __forceinline__ int pieces_in(int steps, int piece) {
    const int n = (int)((float)steps * __builtin_amdgcn_rcpf((float)piece)), left = steps - n * piece;
    return n + (left > 0) + (left > piece) + (left > 2 * piece) + (left > 3 * piece);
}

// Many rows (kv8_prompt.hip).
bool kv8_prompt_wanted(const w4a4_kv8_cache &C, const w4a4_kv8_queries &Q);
int kv8_prompt_tiles(const w4a4_kv8_cache &C, const w4a4_kv8_queries &Q);                 // of a request
size_t kv8_prompt_workspace_bytes(const w4a4_kv8_cache &C, const w4a4_kv8_queries &Q);    // behind the counters
int kv8_prompt(AttnArgs a, const w4a4_kv8_cache &C, const w4a4_kv8_queries &Q, float *parts, hipStream_t st);

}  // namespace w4a4
