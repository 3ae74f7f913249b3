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
// each, of the size of the output's own rounding) with v_scale in them, v_scale = f 2^e, 1/2 <= f < 1:  e is added to the score (in powers of
// two), so that the row's maximum is that of the products e^s v_scale, and f comes in at the rounding.  The largest product of a row so
// becomes 2^13 to 2^14, whatever scales the blocks have that it does not see or gives no weight, and products down to 2^-27 of it keep all
// their bits.  Sums of weights leave e out again, exactly, sixteen keys at a time.
//
// Bound by the bytes of the cache for single tokens.  A (request, tile of rows, key head) is a group; a workgroup takes a group or,
// where requests are long, a piece of one: every workgroup finds from the lengths by itself how long a piece is and
// which one is its own.  The pieces of a group leave sum, maximum and unfinished output in the workspace, and the one that
// comes last joins them, in their order (a counter says who that is, not in which order sums are taken).
//
// Measured (kernel trace, median): one request of 150001 keys, 8 heads of 128, 62.4 us = 4.9 TB/s, the rate of a large copy; 32 requests of
// 160 to 5000 keys (168 MB), 43.5 us = 3.9 TB/s, of which the lengths, the pieces and the join are 4; one request of 777 keys, 7.1 us, which is
// launch, the table's words, two steps of a wave one after the other and the sum over its eight waves.
#include "kv8_attention.hpp"

#include <algorithm>

namespace w4a4 {

int kv8_cache_check(const w4a4_kv8_cache *C);

namespace {

constexpr float kTop = 14.0f;                                      // log2 of a row's largest weight times 2^e
constexpr int kLeast = -80;                                        // least e: 2^(kTop - e) times 2^31 keys stays an fp32 number

// Two floats at the coherence point, past the L2s (each XCD has its own): what workgroups leave for one another.  Release and
// acquire fences at device scope would write back and invalidate a whole L2 each time (a call of 512 workgroups 208 us instead of 49).
__device__ __forceinline__ void leave2(float *p, float x, float y) {
    const unsigned long long v = __builtin_bit_cast(uint32_t, x) | (unsigned long long)__builtin_bit_cast(uint32_t, y) << 32;
    __hip_atomic_store(reinterpret_cast<unsigned long long *>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
struct Two { float x, y; };
__device__ __forceinline__ Two take2(const float *p) {
    const unsigned long long v = __hip_atomic_load(reinterpret_cast<const unsigned long long *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return Two{__builtin_bit_cast(float, (uint32_t)v), __builtin_bit_cast(float, (uint32_t)(v >> 32))};
}

// How the groups are cut, and which piece is this workgroup's.  Each wave works it out by itself.
struct Cut { int entry, head, piece, at; };                        // piece: steps of one; at: which one of the group (entry < 0: none)
template <typename Entry>
__device__ __forceinline__ Cut cut_of(const AttnArgs &a, int entries, int least, Entry entry) {
    const int lane = threadIdx.x & 63, per = (entries + 63) / 64, e0 = min(lane * per, entries), e1 = min(e0 + per, entries);
    auto plus = [](int x, int y) { return x + y; };
    // equal shares of all steps, and larger pieces until there are no more of them than places for workgroups (where groups are
    // more than the places, a piece more for each place).  Up to as many groups as places, that leaves few pieces for what is long: of 512
    // places, with 8 heads, 32 requests of up to 5000 keys are cut at 1.3 times the fair share, 64 at 2, and where one of them has 100000 keys and the others 300, at 2
    // (32 requests), 3.5 (48) or not at all (52 to 64); 65 requests have pieces of the fair share again.
    int mine = 0, only = 0;
    for (int i = e0; i < e1; ++i) mine += only = entry(i).steps;
    const float fair = (float)lanes_reduce<64>(mine, plus) * (float)a.H / (float)a.slots;
    const int most = entries * a.H <= a.slots ? a.slots : entries * a.H + a.slots;
    constexpr float kMore[8] = {1.0f, 1.1f, 1.2f, 1.3f, 1.45f, 1.7f, 2.2f, 3.5f};
    int piece = 0x2000000, count[8] = {};
    auto size = [&](int j) { return max((int)__builtin_ceilf(fair * kMore[j]), least); };
    for (int i = e0; i < e1; ++i) {
        const int steps = per == 1 ? only : entry(i).steps;
#pragma unroll
        for (int j = 0; j < 8; ++j) count[j] += pieces_in(steps, size(j));
    }
#pragma unroll
    for (int j = 7; j >= 0; --j)
        if (lanes_reduce<64>(count[j], plus) * a.H <= most) piece = size(j);
    mine = 0;
    for (int i = e0; i < e1; ++i) mine += pieces_in(per == 1 ? only : entry(i).steps, piece);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(upto, o, 64);
        if (lane >= o) upto += u;
    }
    const unsigned long long in = __ballot((int)blockIdx.x < upto * a.H);
    Cut c{-1, 0, piece, 0};
    if (!in) return c;
    const int owner = __builtin_ctzll(in);
    int before = __builtin_amdgcn_readlane(upto - mine, owner), e = min(owner * per, entries - 1);
    for (;; ++e) {                                                 // (one round where a lane has one entry)
        const int n = per == 1 ? __builtin_amdgcn_readlane(mine, owner) : pieces_in(entry(e).steps, piece);
        if ((int)blockIdx.x < (before + n) * a.H || e + 1 >= entries) break;
        before += n;
    }
    const int in_entry = blockIdx.x - before * a.H;
    c.entry = e;
    c.at = a.heads.of(in_entry);                                   // (the heads of a request side by side: they read neighbouring memory)
    c.head = a.heads.rest(in_entry, c.at);
    return c;
}

// D features, NR tiles of sixteen rows, NW waves.  CUT: groups may be cut; else a workgroup per group.
template <bool BF16, int D, int NR, int NW, bool CUT>
__global__ __launch_bounds__(NW * 64, D <= 128 ? 2 : 1) void kv8_attention_kernel(AttnArgs a) {
    constexpr int NT = D / 16, KW = D / 64, KT = D % 64 != 0;      // feature tiles; 64-feature loads of a key, and one of 32
    constexpr int ROWS = NR * 16, REGS = NR * NT * 4, PART = NW * ROWS;
    constexpr bool AHEAD = D * NR <= 128 || D == 256;              // keys AND values of the next step are fetched during this one
    extern __shared__ __attribute__((aligned(16))) float smem[];   // [wave][REGS][64], then m and l of [wave][ROWS]
    const int tid = threadIdx.x, wave = tid >> 6;
    const int entries = a.requests * a.tiles.d;
    auto entry = [&](int e) {
        const int r = a.tiles.of(e);
        return tile_of(a, r, a.tiles.rest(e, r) * ROWS, ROWS);
    };
    Cut cut;
    if constexpr (CUT) {
        cut = cut_of(a, entries, NW, entry);
        if (cut.entry < 0) return;
    } else {
        cut.entry = a.heads.of(blockIdx.x);
        cut.head = a.heads.rest(blockIdx.x, cut.entry);
        cut.piece = cut.at = 0;
    }
    const int r = a.tiles.of(cut.entry), h = cut.head;
    const int lane = tid & 63, col = lane & 15, kg = lane >> 4, kgroup = col >> 2;
    // Blocks of the lane's rows of K and of its lane group's keys.  What lies behind a request's last block may be anything, but
    // the row of the table is there: the first ones are asked for before the request's length is known.
    struct Ids { int k, v; };
    const int32_t *ids_of = a.table + (size_t)r * a.width;
    auto fetch_ids = [&](int key0) { return Ids{ids_of[min((key0 + 16 * kgroup) >> a.shift, a.width - 1)], ids_of[min((key0 + 16 * kg) >> a.shift, a.width - 1)]}; };
    Ids next = {0, 0};
    if (!CUT && a.width && !a.window) next = fetch_ids(wave * kStep);
    const Tile t = entry(cut.entry);
    if (!t.steps) return;
    // (the pieces of a group are equally long: no short one at its end)
    const int np = CUT ? pieces_in(t.steps, cut.piece) : 1, piece = CUT ? pieces_in(t.steps, np) : t.steps, first_step = cut.at * piece;
    const int steps = min(piece, t.steps - first_step);
    if (CUT && a.width && !a.window) next = fetch_ids((first_step + wave) * kStep);
    const int base = (t.begin & ~(kStep - 1)) + first_step * kStep, stop = min(base + steps * kStep, t.end);
    const int todo = stop > base ? steps : 0;
    if (a.window && wave < todo) next = fetch_ids(base + wave * kStep);

    // the lane's rows
    int hi[NR], lo[NR];                                            // last and first key that each sees
    u32x4_t q[NR][2 * KW + KT];
    float back[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int row = min(t.row0 + 16 * i + col, t.rows - 1), j = a.group.of(row);
        hi[i] = t.len - t.n + j;
        lo[i] = a.window ? hi[i] - a.window + 1 : 0;
        const uint16_t *src = a.q + (long)(t.first + j) * a.ldq + (h * a.group.d + a.group.rest(row, j)) * D;
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
    const int all_hi = t.len - t.n + a.group.of(t.row0);
    const int all_lo = a.window ? t.len - t.n + a.group.of(min(t.row0 + 16 * NR, t.rows) - 1) - a.window + 1 : 0;

    const int mask = (1 << a.shift) - 1;
    struct Blocks { int k, v; bool ok; };                          // ok: the lane group's keys are there
    auto settle = [&](const Ids &d, int s) {
        const int kv = base + kStep * s + 16 * kg;
        Blocks b;
        b.ok = (kv < stop) & (kv + 15 >= t.begin) & ((unsigned)d.v < (unsigned)a.blocks);
        b.k = (unsigned)d.k < (unsigned)a.blocks ? d.k : 0;
        b.v = (unsigned)d.v < (unsigned)a.blocks ? d.v : 0;
        return b;
    };
    u32x4_t kw[4][KW], vw[NT];
    u32x2_t kt[4];
    float ks, vs, ksn = 0, vsn = 0;
    auto fetch_k = [&](const Blocks &d, int s) {
        const int key = base + kStep * s + 16 * kgroup + (col & 3);
        const int8_t *src = a.k + ((((size_t)d.k * a.H + h) << a.shift) + (key & mask)) * D;
#pragma unroll
        for (int T = 0; T < 4; ++T) {
#pragma unroll
            for (int c = 0; c < KW; ++c) kw[T][c] = *reinterpret_cast<const u32x4_t *>(src + 4 * T * D + 64 * c + 16 * kg);
            if (KT) kt[T] = *reinterpret_cast<const u32x2_t *>(src + 4 * T * D + 64 * KW + 8 * kg);
        }
        const size_t unit = (size_t)d.v * a.H + h;
        const float kx = a.k_scale[unit], vx = a.v_scale[unit];    // (of keys that are not there: whatever they hold)
        // (a scale that is no finite number makes NaN of the scores, which the mask keeps from rows that do not see them)
        const bool finite = fabsf(vx) < INFINITY && fabsf(kx) < INFINITY;
        ksn = d.ok ? finite ? kx : NAN : 0.0f;
        vsn = d.ok && finite ? vx : 0.0f;
    };
    auto fetch_v = [&](const Blocks &d, int s) {
        const int key = base + kStep * s + 16 * kg;
        const int8_t *src = a.v + ((((size_t)d.v * a.H + h) * D + col) << a.shift) + (key & mask);
#pragma unroll
        for (int n = 0; n < NT; ++n) vw[n] = *reinterpret_cast<const u32x4_t *>(src + ((size_t)(16 * n) << a.shift));
    };

    float4_t o[NR][NT];
    float m[NR], l[NR];                                            // m: where the largest product is 2^kTop
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.0f;
#pragma unroll
        for (int n = 0; n < NT; ++n) o[i][n] = float4_t{0, 0, 0, 0};
    }

    Blocks now = {0, 0, false}, then = now;                        // of this step, and of the wave's next
    if (wave < todo) {
        now = settle(next, wave);
        fetch_k(now, wave);
        if (AHEAD) fetch_v(now, wave);
        if (wave + NW < todo) next = fetch_ids(base + (wave + NW) * kStep);
    }
    for (int s = wave; s < todo; s += NW) {
        const int key0 = base + kStep * s;
        const bool more = s + NW < todo, ok = now.ok;
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
        if (more) then = settle(next, s + NW);
        if (AHEAD && more) fetch_k(then, s + NW);
        if (!AHEAD) fetch_v(now, s);

        // v_scale = f 2^e (0, and what is below 2^-81: e as it would be there, f smaller)
        const int e0 = max((int)(__builtin_bit_cast(uint32_t, vs) >> 23) - 126, kLeast);
        const float level = (float)e0, f = __builtin_amdgcn_ldexpf(vs, -e0);
        const bool plain = key0 + kStep - 1 <= all_hi && key0 >= all_lo && __all(ok);
        u32x4_t pw[NR][2];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const float kf = ks * back[i];
            float x[16];
#pragma unroll
            for (int T = 0; T < 4; ++T)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * T + e] = __builtin_fmaf(sc[i][T][e], kf, level);
            if (!plain) {
                const int key = key0 + 16 * kg;                    // the lane's keys are key .. key + 15, in order
                const int first = lo[i] - key;
                const unsigned many = ok && hi[i] >= lo[i] ? hi[i] - lo[i] : 0, none = ok && hi[i] >= lo[i] ? 0 : 0x40000000;
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = (unsigned)(e - first) + none <= many ? x[e] : -INFINITY;
            }
            float mx = x[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
            mx = over_groups(mx, max2) - kTop;
            if (__any(mx > m[i])) {
                const float to = fmaxf(mx, m[i]), by = m[i] > -INFINITY ? __builtin_amdgcn_exp2f(m[i] - to) : 0.0f;
                m[i] = to;
                l[i] *= by;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][n][e] *= by;
            }
            const float sub = m[i] > -INFINITY ? m[i] : 0.0f;
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                x[e] = __builtin_amdgcn_exp2f(x[e] - sub);
                sum += x[e];
            }
            l[i] += __builtin_amdgcn_ldexpf(sum, -e0);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                pw[i][0][e] = pack_halves(x[2 * e] * f, x[2 * e + 1] * f);
                pw[i][1][e] = pack_halves(x[8 + 2 * e] * f, x[8 + 2 * e + 1] * f);
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
            if (AHEAD) fetch_v(then, s + NW);
            else fetch_k(then, s + NW);
            now = then;
            if (s + 2 * NW < todo) next = fetch_ids(base + (s + 2 * NW) * kStep);
        }
    }

    // the waves' parts of the same rows
    float *const ml = smem + NW * REGS * 64;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const float sum = over_groups(l[i], add2);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int f = 0; f < 4; ++f) smem[(wave * REGS + (i * NT + n) * 4 + f) * 64 + lane] = o[i][n][f];
        if (kg == 0) {
            ml[wave * ROWS + 16 * i + col] = m[i];
            ml[PART + wave * ROWS + 16 * i + col] = sum;
        }
    }
    __syncthreads();
    const bool whole = np <= 1;
    for (int n = wave; n < NT; n += NW) {                          // sixteen features
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int row = t.row0 + 16 * i + col;
            if (row >= t.rows) continue;
            float mx = -INFINITY, sum = 0.0f, by[NW], y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                by[w] = ml[w * ROWS + 16 * i + col];
                mx = fmaxf(mx, by[w]);
            }
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float f = by[w] > -INFINITY ? __builtin_amdgcn_exp2f(by[w] - mx) : 0.0f;
                sum += f * ml[PART + w * ROWS + 16 * i + col];
                by[w] = f;
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] += smem[(w * REGS + (i * NT + n) * 4 + k) * 64 + lane] * by[w];
            }
            const int j = a.group.of(row);
            const size_t at = ((size_t)(t.first + j) * a.H + h) * a.group.d + a.group.rest(row, j);
            if (whole) {
                const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
                const uint32_t y0 = from_float<BF16>(y[0] * inv) | (uint32_t)from_float<BF16>(y[1] * inv) << 16;
                const uint32_t y1 = from_float<BF16>(y[2] * inv) | (uint32_t)from_float<BF16>(y[3] * inv) << 16;
                *reinterpret_cast<u32x2_t *>(a.out + at * D + 16 * n + 4 * kg) = u32x2_t{y0, y1};
                if (n == 0 && kg == 0 && a.lse) a.lse[at] = log_sum(mx, sum);
            } else {
                float *to = a.po + ((size_t)blockIdx.x * ROWS + 16 * i + col) * D + 16 * n + 4 * kg;
                leave2(to, y[0], y[1]);
                leave2(to + 2, y[2], y[3]);
                if (n == 0 && kg == 0) leave2(a.pml + ((size_t)blockIdx.x * ROWS + 16 * i + col) * 2, mx, sum);
            }
        }
    }
    if (whole) return;

    // the pieces of the group are those of workgroups w0, w0 + H, ...
    if constexpr (CUT) {
    __shared__ int s_last;
    const int w0 = blockIdx.x - cut.at * a.H;
    __builtin_amdgcn_s_waitcnt(0);                                 // what this wave left is there before the workgroup's arrival is
    __syncthreads();
    if (tid == 0) {
        s_last = __hip_atomic_fetch_add(a.arrived + w0, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == np - 1;
        if (s_last) __hip_atomic_store(a.arrived + w0, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next call
    }
    __syncthreads();
    if (!s_last) return;
    // maximum and sum of each row over the parts: THREADS / ROWS lanes a row
    constexpr int THREADS = NW * 64, LANES = THREADS / ROWS, QUADS = D / 4;
    const int rows = min(ROWS, t.rows - t.row0), parts = np;
    auto part = [&](int w) { return (size_t)(w0 + w * a.H) * ROWS; };
    {
        const int row = tid / LANES;
        float mx = -INFINITY, sum = 0.0f;
        if (row < rows)
            for (int w = tid % LANES; w < parts; w += LANES) {
                const Two x = take2(a.pml + (part(w) + row) * 2);
                if (x.x > -INFINITY || x.y != 0.0f) {              // (NaN, which is no maximum)
                    const float to = fmaxf(mx, x.x);
                    sum = sum * __builtin_amdgcn_exp2f(mx - to) + x.y * __builtin_amdgcn_exp2f(x.x - to);
                    mx = to;
                }
            }
        const float most = lanes_reduce<LANES>(mx, max2);
        sum = lanes_reduce<LANES>(mx > -INFINITY ? sum * __builtin_amdgcn_exp2f(mx - most) : sum, add2);
        if (tid % LANES == 0) {
            ml[row] = most;
            ml[ROWS + row] = sum != 0.0f ? 1.0f / sum : 0.0f;
            if (row < rows && a.lse) {
                const int j = a.group.of(t.row0 + row);
                a.lse[((size_t)(t.first + j) * a.H + h) * a.group.d + a.group.rest(t.row0 + row, j)] = log_sum(most, sum);
            }
        }
    }
    __syncthreads();
    // the outputs: four features of a row a thread; where rows are few, several threads share the parts
    const int items = rows * QUADS, ways = max(THREADS / items, 1);
    for (int i0 = 0; i0 < items; i0 += THREADS) {
        const int i = ways > 1 ? tid % items : i0 + tid, way = ways > 1 ? tid / items : 0, row = i / QUADS, f = i % QUADS * 4;
        const bool in = way < ways && i < items;
        float4_t y = {0, 0, 0, 0};
        if (in) {
            const float most = ml[row];
#pragma unroll 8
            for (int w = way; w < parts; w += ways) {
                const Two x = take2(a.pml + (part(w) + row) * 2), v0 = take2(a.po + (part(w) + row) * D + f), v1 = take2(a.po + (part(w) + row) * D + f + 2);
                const float by = x.x > -INFINITY ? __builtin_amdgcn_exp2f(x.x - most) : 0.0f;
                y[0] += by * v0.x;
                y[1] += by * v0.y;
                y[2] += by * v1.x;
                y[3] += by * v1.y;
            }
        }
        if (ways > 1) {
            if (in) *reinterpret_cast<float4_t *>(smem + 4 * (way * items + i)) = y;
            __syncthreads();
            if (in && way == 0)
                for (int k = 1; k < ways; ++k) {
                    const float4_t v = *reinterpret_cast<const float4_t *>(smem + 4 * (k * items + i));
#pragma unroll
                    for (int g = 0; g < 4; ++g) y[g] += v[g];
                }
        }
        if (in && way == 0) {
            const int j = a.group.of(t.row0 + row);
            const float inv = ml[ROWS + row];
            const size_t at = ((size_t)(t.first + j) * a.H + h) * a.group.d + a.group.rest(t.row0 + row, j);
            const uint32_t y0 = from_float<BF16>(y[0] * inv) | (uint32_t)from_float<BF16>(y[1] * inv) << 16;
            const uint32_t y1 = from_float<BF16>(y[2] * inv) | (uint32_t)from_float<BF16>(y[3] * inv) << 16;
            *reinterpret_cast<u32x2_t *>(a.out + at * D + f) = u32x2_t{y0, y1};
        }
    }
    }
}

// How the requests of few rows are shared out, and whether there may be requests of many (kv8_prompt.hip).
struct Split {
    bool some, many;                                               // launched: this kernel; the one for many rows
    int most;                                                      // rows of a request that this one takes
    int nr, tiles;
    bool cut;                                                      // groups are cut where they are long
    int places;                                                    // for pieces in the workspace
};
Split split_of(const w4a4_kv8_cache &C, const w4a4_kv8_queries &Q) {
    Split s;
    s.many = kv8_prompt_wanted(C, Q);
    s.some = !s.many || Q.requests >= kMixed;
    // Where requests of many rows may be among others, single tokens are most of the others: one tile of sixteen rows where a token fits.
    const int group = Q.heads / C.heads;
    s.most = !s.many ? kFewRows : group <= 16 ? 16 : group <= 32 ? 32 : kFewRows;
    const long rows = std::min((long)Q.queries * group, (long)s.most);
    s.nr = rows > 16 && C.features <= 128 ? 2 : 1;
    s.tiles = (int)((rows + 16 * s.nr - 1) / (16 * s.nr));
    const long keys = Q.window ? std::min((long)Q.context, (long)Q.window + 16 * s.nr + kStep) : Q.context;
    const long groups = (long)s.tiles * C.heads * Q.requests;
    // Finding the pieces and joining them costs 4 us, a round of eight steps of a group 2 us.  us whole | cut, 8 key heads of 128: one
    // request of 1024 keys 11.2 | 13.0, 1280 12.6 | 13.0, 2048 16.4 | 13.0; eight of 1280 13.5 | 15.2, 2048 18.0 | 17.2; forty of 1280 30.5 | 29.3.
    s.cut = s.some && keys > 20 * kStep && groups <= kMostGroups;
    s.places = s.cut ? (int)groups + kSlots : 0;
    return s;
}

template <bool BF16, int D, int NR, int NW, bool CUT>
int launch_waves(AttnArgs &a, const Split &s, hipStream_t st) {
    auto kern = kv8_attention_kernel<BF16, D, NR, NW, CUT>;
    constexpr size_t lds = ((size_t)NW * NR * (D / 16) * 4 * 64 + 2 * NW * NR * 16) * sizeof(float);
    static KernelState ks;
    const void *fn = reinterpret_cast<const void *>(kern);
    const int cus = prepare_kernel(fn, lds, ks);
    if (cus < 0) return W4A4_ERR_HIP;
    int grid = a.H * a.tiles.d * a.requests;
    if (CUT) {
        const int at_once = resident_per_cu(fn, NW * 64, lds, ks);
        if (at_once <= 0) return W4A4_ERR_HIP;
        a.slots = min(kSlots, cus * at_once);
        grid = grid <= a.slots ? a.slots : grid + a.slots;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(NW * 64), lds, st, a);
    return launch_status();
}

template <bool BF16, int D, int NR>
int launch(AttnArgs &a, const Split &s, hipStream_t st) {
    constexpr int NW = D <= 128 ? 8 : 4;
    if (!s.cut) return launch_waves<BF16, D, NR, NW, false>(a, s, st);
    // Few groups: eight waves a workgroup, half as many pieces to join; more: four waves, two workgroups a CU, which hide each other's
    // beginning and end.  us at 8 | 4 waves, 128 features: 8 groups of 150001 keys 63 | 68, 48 of 30000 and less 16.1 | 20.0; 256 groups, one request of 8000
    // keys and 31 of 300, 51 | 18, 64 x 8 of 1280 45 | 36; 248 of 160 to 5000 keys 46 | 45.
    if (a.H * a.tiles.d * a.requests <= 32) return launch_waves<BF16, D, NR, NW, true>(a, s, st);
    return launch_waves<BF16, D, NR, 4, true>(a, s, st);
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
    // (the two kernels come one after the other, and leave their parts in the same place)
    const size_t few = s.cut ? (size_t)s.places * 16 * s.nr * (C->features + 2) * sizeof(float) : 0;
    const size_t parts = std::max(few, s.many ? kv8_prompt_workspace_bytes(*C, *Q) : 0);
    return parts ? kCounters * sizeof(int) + parts : 0;
}

extern "C" int w4a4_kv8_attention(const w4a4_kv8_cache *C, const w4a4_kv8_queries *Q, void *out, float *lse, void *workspace,
                                  size_t workspace_bytes, void *stream) {
    if (const int rc = check(C, Q)) return rc;
    if (!Q->tokens || !Q->requests || !Q->queries) return W4A4_OK;
    if (!Q->q || !Q->lens || !Q->start || !out || (Q->width && !Q->table)) return W4A4_ERR_INVALID_ARG;
    if (!aligned16(Q->q) || !aligned16(out)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const Split s = split_of(*C, *Q);
    // steps are counted in 32 bits, and divisions (Div) are exact below 2^32
    const int group = Q->heads / C->heads, tiles = max(s.tiles, s.many ? kv8_prompt_tiles(*C, *Q) : 0);
    if (Q->requests > 65535 || (double)Q->queries * group * group > 4e9 || (double)Q->requests * tiles * max(tiles, C->heads * C->heads) > 4e9 ||
        ((double)Q->width * C->block / kStep + 2) * C->heads * tiles * Q->requests > 2e9) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const size_t need = w4a4_kv8_attention_workspace_bytes(C, Q);
    if (need && (!workspace || workspace_bytes < need)) return W4A4_ERR_WORKSPACE;
    if (need && !aligned16(workspace)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    const int window = Q->window > 1 << 30 ? 0 : Q->window;        // (positions minus a window stay above -2^31)
    int *arrived = static_cast<int *>(workspace);
    float *po = reinterpret_cast<float *>(arrived + (need ? kCounters : 0));
    AttnArgs a{static_cast<const uint16_t *>(Q->q), C->k, C->v, C->k_scale, C->v_scale, Q->table, Q->lens, Q->start,
               static_cast<uint16_t *>(out), lse, po, po + (size_t)s.places * 16 * s.nr * C->features, arrived, Q->ldq, Q->tokens, C->blocks, C->heads,
               __builtin_ctz(C->block), C->blocks ? Q->width : 0, window, Q->queries, Q->requests, 0, 0, s.most,
               Div(group), Div(s.tiles), Div(C->heads), Q->scale * 1.44269504f};
    hipStream_t st = as_stream(stream);
    auto run = [&](auto bf16, auto d) {
        constexpr bool BF = decltype(bf16)::value;
        constexpr int D = decltype(d)::value;
        if constexpr (D <= 128)
            if (s.nr == 2) return launch<BF, D, 2>(a, s, st);
        return launch<BF, D, 1>(a, s, st);
    };
    auto typed = [&](auto d) { return Q->dtype == W4A4_BF16 ? run(std::true_type{}, d) : run(std::false_type{}, d); };
    auto few = [&] {
        switch (C->features) {
            case 64: return typed(std::integral_constant<int, 64>{});
            case 96: return typed(std::integral_constant<int, 96>{});
            case 128: return typed(std::integral_constant<int, 128>{});
            default: return typed(std::integral_constant<int, 256>{});
        }
    };
    if (s.some)
        if (const int rc = few()) return rc;
    if (!s.many) return W4A4_OK;
    a.least = s.some ? s.most + 1 : 0;
    a.most = 0x7fffffff;
    a.tiles = Div(kv8_prompt_tiles(*C, *Q));
    return kv8_prompt(a, *C, *Q, po, st);
}
