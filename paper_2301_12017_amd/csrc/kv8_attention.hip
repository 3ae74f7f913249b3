// Attention over the 8-bit cache.
//
//   s[t] = scale * k_scale[block of t] * sum_d q[d] ck[t,d]        for the keys t that the query sees
//   out = sum_t e^s[t] v_scale[block of t] cv[t] / sum_t e^s[t],   lse = log sum_t e^s[t]
//
// One pass over the keys with a running maximum.  A wave takes 64 keys at a time and sixteen rows (the queries of one request
// and key head: query j of head g is row j * group + g, so that the rows of a tile see nearly the same keys).  The scores are
// computed transposed, S^T = K Q^T, so that a lane holds sixteen scores of ONE row; they are then, converted in place, the
// operand P^T of O^T = V^T P^T.
//
// Codes go from memory straight into registers, sixteen bytes a lane, and become fp16 numbers by byte permutation and one
// subtraction: 0x6400 | u is 1024 + u, u = code + 128.  Nothing passes through LDS, because the order of keys in a tile of S^T
// is free: tile T, row r is key 16 * (r / 4) + 4 T + r % 4 of the 64, which makes the sixteen keys of a lane group of S^T
// exactly the sixteen bytes that it loads of a feature of V.  All of them lie in one block of the cache (blocks hold 16 tokens
// or a multiple): one pair of scales per lane and step.
//
// Queries are brought to fp16 by a power of two per row (largest magnitude in [2^14, 2^15)): exact for fp16 and, but for what is
// 2^28 below the row's largest, for bf16.  Scores and their sums are fp32.  The weights are rounded to fp16 (half a step of 2^-11
// each, of the size of the output's own rounding) with v_scale in them; they are held at c * v_scale, c a power of two per
// wave that keeps the largest product near 2^13, so that weights down to 2^-27 keep all their bits.
//
// Bound by the bytes of the cache for single tokens: keys are shared out over pieces (workgroups) and the waves of each; pieces
// leave their sum, maximum and unfinished output in the workspace, and a second kernel joins them in a fixed order.
#include "gen.hpp"

namespace w4a4 {

int kv8_cache_check(const w4a4_kv8_cache *C);

namespace {

constexpr int kWaves = 4, kStep = 64;                              // waves of a workgroup, keys of a step
constexpr float kUnset = 1.2676506e30f;                            // 2^100: c before a scale of values has been seen

struct AttnArgs {
    const uint16_t *q;
    const int8_t *k, *v;
    const float *k_scale, *v_scale;
    const int32_t *table, *lens, *start;
    uint16_t *out;
    float *lse, *po, *pml;                                         // joined later: [row][piece][D], [row][piece][2]
    long ldq;
    int tokens, blocks, H, group, shift, width, window, queries, pieces, piece;
    float scale;                                                   // in powers of two: scale / ln 2
};

// The rows of one workgroup and the keys they see.
struct Tile {
    int first, n, len, rows, row0;                                 // first token, queries, keys of the request; rows of it; this tile's first
    int begin, end;                                                // keys that any row of the tile sees
};
__device__ __forceinline__ Tile tile_of(const AttnArgs &a, int r, int row0, int tile) {
    Tile t;
    t.first = max(a.start[r], 0);
    t.n = min(min(a.start[r + 1], a.tokens) - t.first, a.queries);
    t.rows = t.n > 0 ? t.n * a.group : 0;
    t.len = min(max(a.lens[r], 0), (int)min((long)a.width << a.shift, 0x7fffff00L));
    t.row0 = row0;
    t.begin = t.end = 0;
    if (row0 < t.rows) {
        const int lo = t.len - t.n + row0 / a.group, hi = t.len - t.n + (min(row0 + tile, t.rows) - 1) / a.group;
        t.end = max(hi + 1, 0);
        t.begin = a.window ? min(max(lo - a.window + 1, 0), t.end) : 0;
    }
    return t;
}
__device__ __forceinline__ int pieces_of(const AttnArgs &a, const Tile &t) {   // pieces begin at a whole step
    const int keys = t.end - (t.begin & ~(kStep - 1));
    return t.end > t.begin ? min((keys + a.piece - 1) / a.piece, a.pieces) : 0;
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

// D features, NR tiles of sixteen rows.
template <bool BF16, int D, int NR>
__global__ __launch_bounds__(kWaves * 64, D * NR >= 256 ? 1 : 2) void kv8_attention_kernel(AttnArgs a) {
    constexpr int NT = D / 16, KW = D / 64, KT = D % 64 != 0;      // feature tiles; 64-feature loads of a key, and one of 32
    extern __shared__ __attribute__((aligned(16))) float smem[];   // [wave][NR * NT * 4][64], then m, l and c of [wave][NR * 16]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, kg = lane >> 4;
    const int r = blockIdx.z, h = blockIdx.y % a.H, tile = blockIdx.y / a.H, p = blockIdx.x;
    const Tile t = tile_of(a, r, tile * 16 * NR, 16 * NR);
    if (t.row0 >= t.rows) return;
    const int np = pieces_of(a, t);
    if (p >= max(np, 1)) return;
    const int base = (t.begin & ~(kStep - 1)) + p * a.piece, stop = p + 1 >= a.pieces ? t.end : min(base + a.piece, t.end);
    const int steps = stop > base ? (stop - base + kStep - 1) / kStep : 0;

    // the lane's rows
    int hi[NR], lo[NR];                                            // last and first key that each sees
    u32x4_t q[NR][2 * KW + KT];
    float back[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int row = min(t.row0 + 16 * i + col, t.rows - 1), j = row / a.group;
        hi[i] = t.len - t.n + j;
        lo[i] = a.window ? hi[i] - a.window + 1 : 0;
        const uint16_t *src = a.q + (long)(t.first + j) * a.ldq + (h * a.group + row % a.group) * D;
#pragma unroll
        for (int c = 0; c < KW; ++c)
#pragma unroll
            for (int s = 0; s < 2; ++s) q[i][2 * c + s] = *reinterpret_cast<const u32x4_t *>(src + 64 * c + 16 * kg + 8 * s);
        if (KT) q[i][2 * KW] = *reinterpret_cast<const u32x4_t *>(src + 64 * KW + 8 * kg);
        float most = 0.0f;
#pragma unroll
        for (int c = 0; c < 2 * KW + KT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                most = fmaxf(most, fmaxf(fabsf(to_float<BF16>((uint16_t)q[i][c][e])), fabsf(to_float<BF16>((uint16_t)(q[i][c][e] >> 16)))));
        most = over_groups(most, max2);
        const int e = most > 0.0f && most < INFINITY ? max((int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127, -100) : 14;
        const float up = power(14 - e);
        back[i] = power(e - 14) * a.scale;
#pragma unroll
        for (int c = 0; c < 2 * KW + KT; ++c)
#pragma unroll
            for (int w = 0; w < 4; ++w)
                q[i][c][w] = pack_halves(to_float<BF16>((uint16_t)q[i][c][w]) * up, to_float<BF16>((uint16_t)(q[i][c][w] >> 16)) * up);
    }
    // wave-uniform: keys that all rows of the tile see
    const int all_hi = t.len - t.n + t.row0 / a.group;
    const int all_lo = a.window ? t.len - t.n + (min(t.row0 + 16 * NR, t.rows) - 1) / a.group - a.window + 1 : 0;

    struct Ids { int k, v; bool ok; };                             // blocks of the lane's rows of K and of its lane group's keys
    const int32_t *ids_of = a.table + (size_t)r * a.width;
    const int kgroup = col >> 2, mask = (1 << a.shift) - 1;
    auto fetch_ids = [&](int s) {
        const int key0 = base + kStep * s, kk = key0 + 16 * kgroup, kv = key0 + 16 * kg;
        Ids d;
        d.k = kk < stop && kk + 15 >= t.begin ? ids_of[kk >> a.shift] : -1;
        d.v = kv < stop && kv + 15 >= t.begin ? ids_of[kv >> a.shift] : -1;
        d.ok = (unsigned)d.v < (unsigned)a.blocks;
        if ((unsigned)d.k >= (unsigned)a.blocks) d.k = 0;
        if (!d.ok) d.v = 0;
        return d;
    };
    u32x4_t kw[4][KW], vw[NT];
    u32x2_t kt[4];
    float ks, vs, ksn = 0, vsn = 0;
    auto fetch_k = [&](const Ids &d, int s) {
        const int key = base + kStep * s + 16 * kgroup + (col & 3);
        const int8_t *src = a.k + ((((size_t)d.k * a.H + h) << a.shift) + (key & mask)) * D;
#pragma unroll
        for (int T = 0; T < 4; ++T) {
#pragma unroll
            for (int c = 0; c < KW; ++c) kw[T][c] = *reinterpret_cast<const u32x4_t *>(src + 4 * T * D + 64 * c + 16 * kg);
            if (KT) kt[T] = *reinterpret_cast<const u32x2_t *>(src + 4 * T * D + 64 * KW + 8 * kg);
        }
        const size_t unit = (size_t)d.v * a.H + h;
        ksn = d.ok ? a.k_scale[unit] : 0.0f;
        vsn = d.ok ? a.v_scale[unit] : 0.0f;
    };
    auto fetch_v = [&](const Ids &d, int s) {
        const int key = base + kStep * s + 16 * kg;
        const int8_t *src = a.v + ((((size_t)d.v * a.H + h) * D + col) << a.shift) + (key & mask);
#pragma unroll
        for (int n = 0; n < NT; ++n) vw[n] = *reinterpret_cast<const u32x4_t *>(src + ((size_t)(16 * n) << a.shift));
    };

    float4_t o[NR][NT];
    float m[NR], l[NR], c = kUnset;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.0f;
#pragma unroll
        for (int n = 0; n < NT; ++n) o[i][n] = float4_t{0, 0, 0, 0};
    }

    Ids now = {0, 0, false}, next = {0, 0, false};
    if (wave < steps) {
        now = fetch_ids(wave);
        fetch_k(now, wave);
        fetch_v(now, wave);
        if (wave + kWaves < steps) next = fetch_ids(wave + kWaves);
    }
    for (int s = wave; s < steps; s += kWaves) {
        const int key0 = base + kStep * s;
        const bool more = s + kWaves < steps, ok = now.ok;
        ks = ksn;
        vs = vsn;
        float4_t sc[NR][4];
#pragma unroll
        for (int T = 0; T < 4; ++T) {
#pragma unroll
            for (int i = 0; i < NR; ++i) sc[i][T] = float4_t{0, 0, 0, 0};
#pragma unroll
            for (int cc = 0; cc < KW; ++cc)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const u32x4_t x = codes8(kw[T][cc][2 * half], kw[T][cc][2 * half + 1]);
#pragma unroll
                    for (int i = 0; i < NR; ++i) sc[i][T] = mfma16<false>(x, q[i][2 * cc + half], sc[i][T]);
                }
            if (KT) {
                const u32x4_t x = codes8(kt[T][0], kt[T][1]);
#pragma unroll
                for (int i = 0; i < NR; ++i) sc[i][T] = mfma16<false>(x, q[i][2 * KW], sc[i][T]);
            }
        }
        if (more) fetch_k(next, s + kWaves);

        // c follows the scales of values
        if (__any(vs * c > 32768.0f)) {
            float most = vs;
            most = over_groups(most, max2);
            const int e = most < INFINITY ? (int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127 : 0;
            const float to = power(min(max(12 - e, -100), 100));
            const float by = to / c;                               // (nothing has been summed yet where c is unset)
            c = to;
#pragma unroll
            for (int i = 0; i < NR; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e2 = 0; e2 < 4; ++e2) o[i][n][e2] *= by;
        }
        const bool plain = key0 + kStep - 1 <= all_hi && key0 >= all_lo && __all(ok);
        u32x4_t pw[NR][2];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const float kf = ks * back[i];
            float x[16];
#pragma unroll
            for (int T = 0; T < 4; ++T)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * T + e] = sc[i][T][e] * kf;
            if (!plain) {
                const int key = key0 + 16 * kg;                    // the lane's keys are key .. key + 15, in order
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!ok || key + e > hi[i] || key + e < lo[i]) x[e] = -INFINITY;
            }
            float mx = x[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
            mx = over_groups(mx, max2);
            if (__any(mx > m[i])) {
                const float to = fmaxf(mx, m[i]), by = m[i] > -INFINITY ? __builtin_amdgcn_exp2f(m[i] - to) : 0.0f;
                m[i] = to;
                l[i] *= by;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][n][e] *= by;
            }
            const float sub = m[i] > -INFINITY ? m[i] : 0.0f, vf = vs * c;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                x[e] = __builtin_amdgcn_exp2f(x[e] - sub);
                l[i] += x[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                pw[i][0][e] = pack_halves(x[2 * e] * vf, x[2 * e + 1] * vf);
                pw[i][1][e] = pack_halves(x[8 + 2 * e] * vf, x[8 + 2 * e + 1] * vf);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const u32x4_t x = codes8(vw[n][2 * half], vw[n][2 * half + 1]);
#pragma unroll
                for (int i = 0; i < NR; ++i) o[i][n] = mfma16<false>(x, pw[i][half], o[i][n]);
            }
        if (more) {
            fetch_v(next, s + kWaves);
            now = next;
            if (s + 2 * kWaves < steps) next = fetch_ids(s + 2 * kWaves);
        }
    }

    // the waves' parts of the same rows
    constexpr int REGS = NR * NT * 4;
    float *const ml = smem + kWaves * REGS * 64;                   // [m | l | 1 / c][wave][NR * 16]
    constexpr int ROWS = NR * 16, PART = kWaves * ROWS;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const float sum = over_groups(l[i], add2);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) smem[(wave * REGS + (i * NT + n) * 4 + e) * 64 + lane] = o[i][n][e];
        if (kg == 0) {
            ml[wave * ROWS + 16 * i + col] = m[i];
            ml[PART + wave * ROWS + 16 * i + col] = sum;
            ml[2 * PART + wave * ROWS + 16 * i + col] = 1.0f / c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int row = t.row0 + 16 * i + col;
        if (row >= t.rows) continue;
        float mx = -INFINITY, sum = 0.0f, by[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, ml[w * ROWS + 16 * i + col]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float mw = ml[w * ROWS + 16 * i + col], e = mw > -INFINITY ? __builtin_amdgcn_exp2f(mw - mx) : 0.0f;
            sum += e * ml[PART + w * ROWS + 16 * i + col];
            by[w] = e * ml[2 * PART + w * ROWS + 16 * i + col];
        }
        const bool whole = np <= 1;
        const float inv = whole ? (sum != 0.0f ? 1.0f / sum : 0.0f) : 1.0f;
        const size_t at = (size_t)(t.first + row / a.group) * (a.H * a.group) + h * a.group + row % a.group;
        for (int n = wave; n < NT; n += kWaves) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[e] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) y[e] += smem[(w * REGS + (i * NT + n) * 4 + e) * 64 + lane] * by[w];
                y[e] *= inv;
            }
            if (whole) {
                const uint32_t y0 = from_float<BF16>(y[0]) | (uint32_t)from_float<BF16>(y[1]) << 16;
                const uint32_t y1 = from_float<BF16>(y[2]) | (uint32_t)from_float<BF16>(y[3]) << 16;
                *reinterpret_cast<u32x2_t *>(a.out + at * D + 16 * n + 4 * kg) = u32x2_t{y0, y1};
            } else {
                *reinterpret_cast<float4_t *>(a.po + (at * a.pieces + p) * D + 16 * n + 4 * kg) = float4_t{y[0], y[1], y[2], y[3]};
            }
        }
        if (wave == 0 && kg == 0) {
            if (!whole) {
                a.pml[(at * a.pieces + p) * 2] = mx;
                a.pml[(at * a.pieces + p) * 2 + 1] = sum;
            } else if (a.lse) {
                a.lse[at] = sum != 0.0f ? (mx + log2f(sum)) * 0.69314718056f : -INFINITY;
            }
        }
    }
}

// A wave per row: the pieces of a tile's rows.
template <bool BF16, int D, int NR>
__global__ __launch_bounds__(256) void kv8_join_kernel(AttnArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = blockIdx.y, h = blockIdx.x % a.H, tile = blockIdx.x / a.H;
    const Tile t = tile_of(a, r, tile * 16 * NR, 16 * NR);
    if (t.row0 >= t.rows) return;
    const int np = pieces_of(a, t);
    if (np <= 1) return;
    constexpr int F = (D + 63) / 64;
    for (int row = t.row0 + wave; row < min(t.row0 + 16 * NR, t.rows); row += 4) {
        const size_t at = (size_t)(t.first + row / a.group) * (a.H * a.group) + h * a.group + row % a.group;
        const float *ml = a.pml + at * a.pieces * 2, *po = a.po + at * a.pieces * D;
        float mx = -INFINITY, sum = 0.0f, y[F] = {};
        for (int p = 0; p < np; ++p) mx = fmaxf(mx, ml[2 * p]);
        for (int p = 0; p < np; ++p) {
            const float e = ml[2 * p] > -INFINITY ? __builtin_amdgcn_exp2f(ml[2 * p] - mx) : 0.0f;
            sum += e * ml[2 * p + 1];
#pragma unroll
            for (int f = 0; f < F; ++f)
                if (64 * f + lane < D) y[f] += e * po[(size_t)p * D + 64 * f + lane];
        }
        const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
        for (int f = 0; f < F; ++f)
            if (64 * f + lane < D) a.out[at * D + 64 * f + lane] = from_float<BF16>(y[f] * inv);
        if (lane == 0 && a.lse) a.lse[at] = sum != 0.0f ? (mx + log2f(sum)) * 0.69314718056f : -INFINITY;
    }
}

// How a call is shared out: tiles of rows, pieces of keys.
struct Split { int nr, tiles, pieces, piece; };
Split split_of(const w4a4_kv8_cache &C, const w4a4_kv8_queries &Q) {
    Split s;
    const int group = Q.heads / C.heads;
    const long rows = (long)Q.queries * group;
    s.nr = rows > 16 ? 2 : 1;
    s.tiles = (int)((rows + 16 * s.nr - 1) / (16 * s.nr));
    const long keys = Q.window ? min((long)Q.context, (long)Q.window + 16 * s.nr + kStep) : Q.context;
    const long groups = (long)s.tiles * C.heads * Q.requests;      // workgroups without pieces
    long piece = (keys * groups + 1023) / 1024;
    piece = (max(piece, 256L) + 255) / 256 * 256;
    s.pieces = (int)max(1L, (keys + piece - 1) / piece);
    s.piece = (int)piece;
    return s;
}

template <bool BF16, int D, int NR>
int launch(AttnArgs &a, const Split &s, int requests, hipStream_t st) {
    auto kern = kv8_attention_kernel<BF16, D, NR>;
    constexpr size_t lds = ((size_t)kWaves * NR * (D / 16) * 4 * 64 + 3 * kWaves * NR * 16) * sizeof(float);
    static KernelState ks;
    if (prepare_kernel(reinterpret_cast<const void *>(kern), lds, ks) < 0) return W4A4_ERR_HIP;
    hipLaunchKernelGGL(kern, dim3(s.pieces, a.H * s.tiles, requests), dim3(kWaves * 64), lds, st, a);
    if (s.pieces > 1) hipLaunchKernelGGL((kv8_join_kernel<BF16, D, NR>), dim3(a.H * s.tiles, requests), dim3(256), 0, st, a);
    return launch_status();
}

int check(const w4a4_kv8_cache *C, const w4a4_kv8_queries *Q) {
    if (const int rc = kv8_cache_check(C)) return rc;
    if (!Q || Q->tokens < 0 || Q->requests < 0 || Q->heads <= 0 || Q->queries < 0 || Q->context < 0 || Q->window < 0 || Q->width < 0) return W4A4_ERR_INVALID_ARG;
    if (Q->dtype != W4A4_F16 && Q->dtype != W4A4_BF16) return W4A4_ERR_INVALID_ARG;
    if (Q->heads % C->heads || Q->ldq < Q->heads * C->features || !(Q->scale > 0.0f && Q->scale < INFINITY)) return W4A4_ERR_INVALID_ARG;
    if (Q->ldq % 8 || Q->heads > 8192) return W4A4_ERR_UNSUPPORTED_SHAPE;
    return W4A4_OK;
}

}  // namespace
}  // namespace w4a4

using namespace w4a4;

extern "C" size_t w4a4_kv8_attention_workspace_bytes(const w4a4_kv8_cache *C, const w4a4_kv8_queries *Q) {
    if (check(C, Q) || !Q->tokens || !Q->requests || !Q->queries) return 0;
    const Split s = split_of(*C, *Q);
    return s.pieces > 1 ? (size_t)Q->tokens * Q->heads * s.pieces * (C->features + 2) * sizeof(float) : 0;
}

extern "C" int w4a4_kv8_attention(const w4a4_kv8_cache *C, const w4a4_kv8_queries *Q, void *out, float *lse, void *workspace,
                                  size_t workspace_bytes, void *stream) {
    if (const int rc = check(C, Q)) return rc;
    if (!Q->tokens || !Q->requests || !Q->queries) return W4A4_OK;
    if (!Q->q || !Q->lens || !Q->start || !out || (Q->width && !Q->table)) return W4A4_ERR_INVALID_ARG;
    if (!aligned16(Q->q) || !aligned16(out)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const Split s = split_of(*C, *Q);
    if (Q->requests > 65535 || (long)C->heads * s.tiles > 65535) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const size_t need = w4a4_kv8_attention_workspace_bytes(C, Q);
    if (need && (!workspace || workspace_bytes < need)) return W4A4_ERR_WORKSPACE;
    if (need && !aligned16(workspace)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    float *po = static_cast<float *>(workspace);
    AttnArgs a{static_cast<const uint16_t *>(Q->q), C->k, C->v, C->k_scale, C->v_scale, Q->table, Q->lens, Q->start,
               static_cast<uint16_t *>(out), lse, po, po + (size_t)Q->tokens * Q->heads * s.pieces * C->features, Q->ldq, Q->tokens, C->blocks, C->heads,
               Q->heads / C->heads, __builtin_ctz(C->block), C->blocks ? Q->width : 0, Q->window, Q->queries, s.pieces, s.piece, Q->scale * 1.44269504f};
    hipStream_t st = as_stream(stream);
    auto run = [&](auto bf16, auto d) {
        constexpr bool BF = decltype(bf16)::value;
        constexpr int D = decltype(d)::value;
        return s.nr == 2 ? launch<BF, D, 2>(a, s, Q->requests, st) : launch<BF, D, 1>(a, s, Q->requests, st);
    };
    auto typed = [&](auto d) { return Q->dtype == W4A4_BF16 ? run(std::true_type{}, d) : run(std::false_type{}, d); };
    switch (C->features) {
        case 64: return typed(std::integral_constant<int, 64>{});
        case 96: return typed(std::integral_constant<int, 96>{});
        case 128: return typed(std::integral_constant<int, 128>{});
        default: return typed(std::integral_constant<int, 256>{});
    }
}
