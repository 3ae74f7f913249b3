// Attention over the 8-bit cache for many rows: prompts, or what follows an earlier part of one.
//
// The mathematics is kv8_attention.hip's (scores transposed, codes as fp16 numbers, queries brought to fp16 by a power of two per
// row, weights rounded to fp16 with the values' scales in them); the shape is another one.  NW waves of 32 rows share the keys:
// 64 of them at a time are fetched as codes by all threads, become fp16 numbers ONCE and go to LDS, two buffers in turn,
// and the 32 x 32 matrix instruction reads them from there.  A lane holds sixteen scores of one row out of 32 keys, the keys
// 8 (i / 4) + 4 (lane / 32) + i % 4; values are stored in LDS in the order in which that makes the weights the operand of the
// second product.
//
// A weight times its block's scale is one exponential: exp2(raw * k + log2(v_scale) - m); the row's sum is taken from the same numbers,
// divided by the scale again, once per sixteen keys.  The maximum m is that of the row's own products e^s v_scale, so that blocks that a row does
// not see, or gives no weight, take no bits from it: the largest product becomes 2^6, products down to 2^-20 of it keep all their bits as
// fp16 numbers.  m is let fall behind by up to 2^8 before what has been summed is re-scaled: weights stay below 2^15.  (To look for weights
// that are too large among the packed ones, and for a maximum only then, took 207 us where this takes 190.)  Scales are taken relative to
// z, a power of two near the wave's first one that is not 0 (it follows one that is 2^96 above); a block 2^80 below z, or of scale 0, counts as one
// 2^80 below, and outputs that such blocks alone can make, less than 2^-73 of 2^z, are zeros.
//
// Bound by the vector ALU between the products: per score an FMA, an exponential at a quarter of the rate, a sum, half a
// maximum and half a conversion, and 1.25 instructions per code and workgroup, beside 16 matrix instructions of 32 cycles for 32 x 32
// scores (128 features).  Measured: 1500 queries of a request of 4100 keys and 751 of one of 3726, 32 heads on 8 of 128 features (124 GFLOP), 172 us
// for the call among others = 720 TFLOP/s (kernel trace: 178 to 188, and 13.4 for the join); matrix pipe 29 %, vector ALU 46 % of the cycles (counters), hardly
// at the same time with two waves in a SIMD, and more do not fit its registers.
//
// A group is 32 NW rows of a request and key head.  Groups beyond whole rounds of the device's workgroups are cut into pieces,
// whose outputs a second kernel joins by their sums, each of its workgroups a slice of a group.
#include "kv8_attention.hpp"

namespace w4a4 {
namespace {

constexpr int kMostPieces = 768;                                   // of groups that are cut
constexpr float kTop = 6.0f;                                       // log2 of a row's largest weight when its maximum is up to date
constexpr float kLag = 8.0f;                                       // how far a maximum may fall behind, in powers of two
constexpr float kNone = -300.0f;                                   // log2 of a scale of 0
// Least log2 of a scale relative to z, and the largest before z follows: 2^(kTop + kLag - kBelow) times 2^31 keys stays an fp32 number, and behind
// a weight of 2^(kTop - kAbove) in the sum others down to 2^-36 of it count.
constexpr float kBelow = -80.0f, kAbove = 96.0f;
typedef float float16_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ float16_t mfma32(u32x4_t a, u32x4_t b, float16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}
template <typename Op>
__device__ __forceinline__ float both_halves(float x, Op op) {     // op over the two lanes l, l + 32, in both of them
    const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return op(__builtin_bit_cast(float, (unsigned)s[0]), __builtin_bit_cast(float, (unsigned)s[1]));
}

__device__ __forceinline__ int upto_lane(int x) {                  // sum over the lanes up to this one
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(x, o, 64);
        if (lane >= o) x += u;
    }
    return x;
}

// The work of a call: groups 0 .. whole-1 as they are, then the pieces of the others.  Each wave works it out by itself (in the join one for all).
struct Plan {
    int per, whole, piece, items;                                  // entries a lane; whole groups; steps of a piece; groups and pieces in all
    int before, rank;                                              // pieces (or groups) and entries with rows in front of this lane's entries
    int mine;                                                      // its own
};
// f(steps) for the tiles of `tile` rows with rows among entries e0 .. e1-1, in order.
template <typename Of, typename F>
__device__ __forceinline__ void each_tile(const AttnArgs &a, int tile, int e0, int e1, Of sizes, F f) {
    for (int e = e0; e < e1;) {
        const int r = a.tiles.of(e), next = min((r + 1) * a.tiles.d, e1);
        const Sizes z = sizes(r);
        const int rows = z.n * a.group.d, last = min(next, r * a.tiles.d + (rows + tile - 1) / tile);
        for (; e < last; ++e) f(tile_of(a, z, (e - r * a.tiles.d) * tile, tile).steps);
        e = next;
    }
}
template <typename Of>
__device__ __forceinline__ Plan plan_of(const AttnArgs &a, int tile, int entries, Of sizes) {
    const int lane = threadIdx.x & 63;
    auto plus = [](int x, int y) { return x + y; };
    Plan p;
    p.per = (entries + 63) / 64;
    const int e0 = min(lane * p.per, entries), e1 = min(e0 + p.per, entries);
    int some = 0, most = 0, rest = 0;
    each_tile(a, tile, e0, e1, sizes, [&](int s) {
        ++some;
        most = max(most, s);
        rest += s;
    });
    p.rank = upto_lane(some) - some;
    const int groups = lanes_reduce<64>(some, plus) * a.H, whole_entries = groups / a.slots * a.slots / a.H;
    most = lanes_reduce<64>(most, [](int x, int y) { return max(x, y); });
    p.whole = whole_entries * a.H;
    int r = p.rank;
    if (whole_entries) {                                           // (wave-uniform)
        rest = 0;
        each_tile(a, tile, e0, e1, sizes, [&](int s) { rest += r++ >= whole_entries ? s : 0; });
    }
    const float fair = (float)lanes_reduce<64>(rest, plus) * (float)a.H / (float)a.slots;
    // the size that gets through soonest: rounds of pieces, each of which costs about four steps more, and a hundredth of one to join (not
    // cut: one round of the longest)
    p.piece = 0x2000000;                                           // (more than the steps of 2^31 keys)
    int size[3], n[3] = {};
#pragma unroll
    for (int k = 0; k < 3; ++k) size[k] = max((int)__builtin_ceilf(fair / (float)(k + 1)), 4);
    r = p.rank;
    each_tile(a, tile, e0, e1, sizes, [&](int s) {
        const bool is_whole = r++ < whole_entries;
#pragma unroll
        for (int k = 0; k < 3; ++k) n[k] += is_whole ? 1 : pieces_in(s, size[k]);
    });
    p.mine = some;
    float best = (float)most;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const int all = (lanes_reduce<64>(n[k], plus) - whole_entries) * a.H;
        const float cost = (float)((all + a.slots - 1) / a.slots * (size[k] + 4)) + 1.0f + 0.01f * (float)all;
        if (all <= kMostPieces && cost < best) {
            best = cost;
            p.piece = size[k];
            p.mine = n[k];
        }
    }
    p.before = upto_lane(p.mine) - p.mine;
    p.items = lanes_reduce<64>(p.mine, plus) * a.H;
    return p;
}
struct Item { int entry, head, at, pieces; };
template <typename Of>
__device__ __forceinline__ Item item_of(const AttnArgs &a, const Plan &p, int tile, int entries, int item, Of sizes) {
    const int lane = threadIdx.x & 63, owner = __builtin_ctzll(__ballot(item < (p.before + p.mine) * a.H));
    int before = __builtin_amdgcn_readlane(p.before, owner), rank = __builtin_amdgcn_readlane(p.rank, owner);
    const int end = min((owner + 1) * p.per, entries);
    for (int e0 = owner * p.per;; e0 += 64) {                      // an entry a lane
        const int e = e0 + lane, r = a.tiles.of(min(e, end - 1));
        const int steps = e < end ? tile_of(a, sizes(r), a.tiles.rest(e, r) * tile, tile).steps : 0;
        const unsigned long long some = __ballot(steps > 0);
        const int nth = rank + __builtin_popcountll(some & ((1ull << lane) - 1));
        const int n = steps == 0 ? 0 : nth * a.H >= p.whole ? pieces_in(steps, p.piece) : 1, upto = upto_lane(n);
        const unsigned long long in = __ballot(item < (before + upto) * a.H);
        if (in || e0 + 64 >= end) {
            const int at = in ? __builtin_ctzll(in) : 0;
            Item i;
            i.entry = e0 + at;
            i.pieces = __builtin_amdgcn_readlane(n, at);
            const int rest = item - (before + __builtin_amdgcn_readlane(upto, at) - i.pieces) * a.H;
            i.at = a.heads.of(rest);                               // (the heads of a request side by side)
            i.head = a.heads.rest(rest, i.at);
            return i;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
        rank += __builtin_popcountll(some);
    }
}

// Sizes of the first requests, which the plan and every item go through, kept in LDS.
constexpr int kKept = 512;
__device__ __forceinline__ void keep_sizes(const AttnArgs &a, Sizes *kept) {
    for (int r = threadIdx.x; r < min(a.requests, kKept); r += blockDim.x) kept[r] = sizes_of(a, r);
    __syncthreads();
}

// The arguments of the kernel, read again: what is kept of them in scalar registers from one end of the kernel to the other does not
// fit and would be moved to and fro in the inner loop.
__device__ __forceinline__ AttnArgs again() {
    auto p = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const AttnArgs *)p;
}

template <int D> constexpr int kPitchK = D + 8;                     // halves of a row in LDS
template <int D> constexpr int kPitchV = kStep + 8;
template <int D> constexpr size_t kBuffer = (size_t)(kStep * kPitchK<D> + D * kPitchV<D>) * 2;

template <bool BF16, int D, int NW>
__global__ __launch_bounds__(NW * 64, D <= 128 ? 2 : 1) void kv8_prompt_kernel(AttnArgs args) {
    constexpr int ROWS = 32 * NW, THREADS = 64 * NW, FT = D / 32, QS = D / 16, N = (4 * D + THREADS - 1) / THREADS, NH = D <= 128 ? 2 : 1;
    extern __shared__ __attribute__((aligned(16))) uint16_t lds[]; // two buffers of [64][keys' row], [D][values' row]
    __shared__ float s_scale[2][2][4];                             // [buffer][of keys, log2 of values][sixteen keys]; of keys: -infinity for none
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, hl = lane >> 5, mask = (1 << args.shift) - 1;
    const int entries = args.requests * args.tiles.d;
    __shared__ Sizes kept[kKept];
    keep_sizes(args, kept);
    const Plan plan = plan_of(args, ROWS, entries, [&](int r) { return r < kKept ? kept[r] : sizes_of(args, r); });
    for (int item = blockIdx.x; item < plan.items; item += gridDim.x) {
        const AttnArgs a = again();
        const Item it = item_of(a, plan, ROWS, entries, item, [&](int r) { return r < kKept ? kept[r] : sizes_of(a, r); });
        const int r = a.tiles.of(it.entry), h = it.head;
        const Tile t = tile_of(a, r, a.tiles.rest(it.entry, r) * ROWS, ROWS);
        const int first_step = it.pieces > 1 ? it.at * plan.piece : 0, steps_in = it.pieces > 1 ? min(plan.piece, t.steps - first_step) : t.steps;
        const int base = (t.begin & ~(kStep - 1)) + first_step * kStep, stop = min(base + steps_in * kStep, t.end);
        const int steps = stop > base ? (stop - base + kStep - 1) / kStep : 0;
        const int32_t *ids_of = a.table + (size_t)r * a.width;
        // the lane's chunks in a block: codes of a head lie at head * features * tokens of a block, for keys and for values
        const uint32_t unit = (uint32_t)(a.H * D) << a.shift;
        const int8_t *kbase[N], *vbase[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = min(tid + i * THREADS, 4 * D - 1);
            kbase[i] = a.k + ((size_t)h * D << a.shift) + ((c / (D / 16)) & mask) * D + c % (D / 16) * 16;
            vbase[i] = a.v + (((size_t)h * D + (c >> 2)) << a.shift) + ((16 * (c & 3)) & mask);
        }

        // codes of a step: keys in sixteens of a row, values in sixteens of a feature
        u32x4_t kreg[N], vreg[N];
        int kid[N], vid[N];
        float ks = 0.0f, vs = 0.0f;
        bool there = false;
        auto id_of = [&](int key) {                                // (a 32-bit offset from a uniform address)
            return *reinterpret_cast<const int32_t *>(reinterpret_cast<const char *>(ids_of) + 4u * (uint32_t)min(key >> a.shift, a.width - 1));
        };
        auto fetch_ids = [&](int s) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = min(tid + i * THREADS, 4 * D - 1), key0 = base + s * kStep;
                kid[i] = id_of(key0 + c / (D / 16));
                vid[i] = id_of(key0 + 16 * (c & 3));
            }
        };
        auto fetch = [&](int s) {
            const int key0 = base + s * kStep;
            if (tid < 4) {
                const int key = key0 + 16 * tid;
                there = (key < stop) & (key + 15 >= t.begin) & ((unsigned)vid[0] < (unsigned)a.blocks);
                const size_t at = (size_t)(there ? vid[0] : 0) * a.H + h;
                ks = a.k_scale[at];
                vs = a.v_scale[at];
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t kb = (unsigned)kid[i] < (unsigned)a.blocks ? kid[i] : 0, vb = (unsigned)vid[i] < (unsigned)a.blocks ? vid[i] : 0;
                kreg[i] = *reinterpret_cast<const u32x4_t *>(kbase[i] + (uint64_t)kb * unit + (key0 & mask) * D);
                vreg[i] = *reinterpret_cast<const u32x4_t *>(vbase[i] + (uint64_t)vb * unit + (key0 & mask));
            }
        };
        auto put = [&](int buf) {
            uint16_t *kd = lds + buf * (kBuffer<D> / 2), *vd = kd + kStep * kPitchK<D>;
            if (tid < 4) {
                // (a scale that is no finite number makes NaN of the scores, which the mask keeps from rows that do not see them)
                s_scale[buf][0][tid] = !there ? -INFINITY : fabsf(vs) < INFINITY && fabsf(ks) < INFINITY ? ks : NAN;
                s_scale[buf][1][tid] = there && vs > 0.0f && vs < INFINITY ? fmaxf(__builtin_amdgcn_logf(vs), -140.0f) : kNone;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = tid + i * THREADS;
                if (4 * D % THREADS != 0 && c >= 4 * D) break;
                u32x4_t *k = reinterpret_cast<u32x4_t *>(kd + c / (D / 16) * kPitchK<D> + c % (D / 16) * 16);
                k[0] = codes8(kreg[i][0], kreg[i][1]);
                k[1] = codes8(kreg[i][2], kreg[i][3]);
                // keys 0..3, 8..11 for the lower half of a wave, 4..7, 12..15 for the upper one
                u32x4_t *v = reinterpret_cast<u32x4_t *>(vd + (c >> 2) * kPitchV<D> + 16 * (c & 3));
                v[0] = codes8(vreg[i][0], vreg[i][2]);
                v[1] = codes8(vreg[i][1], vreg[i][3]);
            }
        };

        if (steps > 0) {
            fetch_ids(0);
            fetch(0);
            if (steps > 1) fetch_ids(1);
        }
        // the lane's row
        const int wrow = t.row0 + 32 * wave, row = min(wrow + col, t.rows - 1), j = a.group.of(row);
        const bool any = wrow < t.rows;
        const int hi = t.len - t.n + j, lo = a.window ? hi - a.window + 1 : 0;
        const int hi0 = __builtin_amdgcn_readfirstlane(t.len - t.n + a.group.of(min(wrow, t.rows - 1)));
        const int hi1 = __builtin_amdgcn_readfirstlane(t.len - t.n + a.group.of(min(wrow + 31, t.rows - 1)));
        const int lo0 = a.window ? hi0 - a.window + 1 : 0, lo1 = a.window ? hi1 - a.window + 1 : 0;
        u32x4_t q[QS];
        float back;
        {
            const uint16_t *src = a.q + (long)(t.first + j) * a.ldq + (h * a.group.d + a.group.rest(row, j)) * D + 8 * hl;
#pragma unroll
            for (int s = 0; s < QS; ++s) q[s] = *reinterpret_cast<const u32x4_t *>(src + 16 * s);
            float most = 0.0f;
#pragma unroll
            for (int s = 0; s < QS; ++s)
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    most = fmaxf(most, fmaxf(fabsf(to_float<BF16>((uint16_t)q[s][w])), fabsf(to_float<BF16>((uint16_t)(q[s][w] >> 16)))));
            most = both_halves(most, max2);
            const int e = most > 0.0f && most < INFINITY ? max((int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127, -100) : 14;
            const float up = power(14 - e);
            back = power(e - 14) * a.scale;
#pragma unroll
            for (int s = 0; s < QS; ++s)
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    q[s][w] = pack_halves(to_float<BF16>((uint16_t)q[s][w]) * up, to_float<BF16>((uint16_t)(q[s][w] >> 16)) * up);
        }
        float16_t o[FT];
#pragma unroll
        for (int f = 0; f < FT; ++f) o[f] = float16_t{};
        float m = -INFINITY, l = 0.0f, z = kNone;                  // (z is the same in all lanes)

        __syncthreads();                                           // (the last item's keys have been read)
        if (steps > 0) put(0);
        if (steps > 1) {
            fetch(1);
            if (steps > 2) fetch_ids(2);
        }
        __syncthreads();
        for (int s = 0; s < steps; ++s) {
            const int buf = s & 1;
            const uint16_t *kd = lds + buf * (kBuffer<D> / 2) + col * kPitchK<D> + 8 * hl;
            const uint16_t *vd = lds + buf * (kBuffer<D> / 2) + kStep * kPitchK<D> + col * kPitchV<D> + 8 * hl;
            float kf[4], ex[4], rv[4];                             // of sixteen keys: their scale, log2 of the values' scale over 2^z, 1 / that
            bool shown = true;
            float top = kNone;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                kf[g] = s_scale[buf][0][g];
                ex[g] = s_scale[buf][1][g];
                shown &= kf[g] != -INFINITY;
                top = fmaxf(top, ex[g]);
            }
            if (__builtin_amdgcn_readfirstlane(top > z + kAbove)) {            // wave-uniform, seldom more than once
                const float to = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, __builtin_floorf(top)))), by = fminf(to - z, -kBelow);
                z = to;
                m -= by;
                l *= __builtin_amdgcn_exp2f(by);
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                ex[g] = fmaxf(ex[g] - z, kBelow);
                rv[g] = __builtin_amdgcn_exp2f(-ex[g]);
            }
            if (s + 1 < steps) {                                   // (the other buffer's step is over for every wave)
                put(buf ^ 1);
                if (s + 2 < steps) {
                    fetch(s + 2);
                    if (s + 3 < steps) fetch_ids(s + 3);
                }
            }
#pragma unroll
            for (int part = 0; part < 2; part += NH) {
                const int key0 = base + s * kStep + 32 * part;
                if (!any || key0 > hi1 || key0 + 32 * NH - 1 < lo0) continue;           // wave-uniform
                const bool plain = __builtin_amdgcn_readfirstlane(shown) && key0 + 32 * NH - 1 <= hi0 && key0 >= lo1;
                // Operands are read from LDS four at a time, while the products of the four before are under way (the compiler by itself reads
                // each one directly in front of its product and waits for it: a third slower).
                constexpr int SETS = NH * QS / 4;
                float16_t x[NH];
#pragma unroll
                for (int n = 0; n < NH; ++n) x[n] = float16_t{};
                u32x4_t kk[2][4];
                auto key_set = [&](int k) {                        // of each sixteen features: the 32 keys of both halves, or two sixteens
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        kk[k & 1][u] = *reinterpret_cast<const u32x4_t *>(kd + 32 * (part + u % NH) * kPitchK<D> + 16 * (k * (4 / NH) + u / NH));
                };
                key_set(0);
#pragma unroll
                for (int k = 0; k < SETS; ++k) {
                    if (k + 1 < SETS) key_set(k + 1);
                    __builtin_amdgcn_sched_barrier(0x16);
#pragma unroll
                    for (int u = 0; u < 4; ++u) x[u % NH] = mfma32(kk[k & 1][u], q[k * (4 / NH) + u / NH], x[u % NH]);
                }
                u32x4_t vv[2][FT];
                auto value_set = [&](int g) {
#pragma unroll
                    for (int f = 0; f < FT; ++f) vv[g & 1][f] = *reinterpret_cast<const u32x4_t *>(vd + 32 * f * kPitchV<D> + 16 * (2 * part + g));
                };
                value_set(0);
                u32x4_t pw[2 * NH];
                auto weigh = [&](auto is_plain) {
                    constexpr bool PLAIN = decltype(is_plain)::value;
                    if constexpr (!PLAIN) {
#pragma unroll
                        for (int n = 0; n < NH; ++n)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const int key = key0 + 32 * n + 8 * (i / 4) + 4 * hl + i % 4;
                                x[n][i] = (key <= hi) & (key >= lo) & (kf[2 * (part + n) + i / 8] != -INFINITY) ? x[n][i] : -INFINITY;
                            }
                    }
                    float by[2 * NH], mx = -INFINITY;
#pragma unroll
                    for (int g = 0; g < 2 * NH; ++g) {
                        by[g] = kf[2 * part + g] * back;
                        float e = x[g / 2][8 * (g % 2)];
#pragma unroll
                        for (int i = 1; i < 8; ++i) e = fmaxf(e, x[g / 2][8 * (g % 2) + i]);
                        mx = fmaxf(mx, PLAIN || e > -INFINITY ? __builtin_fmaf(e, by[g], ex[2 * part + g]) : -INFINITY);
                    }
                    mx = both_halves(mx, max2) - kTop;
                    if (__any(mx > m + kLag)) {                    // the first steps, seldom later; rows that need it
                        const float to = mx > m + kLag ? mx : m, a0 = m > -INFINITY ? __builtin_amdgcn_exp2f(m - to) : 0.0f;
                        m = to;
                        l *= a0;
#pragma unroll
                        for (int f = 0; f < FT; ++f)
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[f][i] *= a0;
                    }
                    const float sub = m > -INFINITY ? m : 0.0f;
#pragma unroll
                    for (int g = 0; g < 2 * NH; ++g) {
                        const float sh = ex[2 * part + g] - sub;
                        float p[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float raw = x[g / 2][8 * (g % 2) + i];
                            float e = __builtin_fmaf(raw, by[g], sh);
                            if (!PLAIN) e = raw == -INFINITY ? raw : e;     // (what the mask took; a NaN stays one)
                            p[i] = __builtin_amdgcn_exp2f(e);
                        }
                        l = __builtin_fmaf(((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])), rv[2 * part + g], l);
                        pw[g] = u32x4_t{pack_halves(p[0], p[1]), pack_halves(p[2], p[3]), pack_halves(p[4], p[5]), pack_halves(p[6], p[7])};
                    }
                };
                if (plain) weigh(std::true_type{});
                else weigh(std::false_type{});
#pragma unroll
                for (int g = 0; g < 2 * NH; ++g) {
                    if (g + 1 < 2 * NH) value_set(g + 1);
                    __builtin_amdgcn_sched_barrier(0x16);
#pragma unroll
                    for (int f = 0; f < FT; ++f) o[f] = mfma32(vv[g & 1][f], pw[g], o[f]);
                }
            }
            if (s + 1 < steps) __syncthreads();
        }

        l = both_halves(l, add2);
        const AttnArgs b = again();
        const float inv = l != 0.0f ? __builtin_amdgcn_exp2f(z) / l : 0.0f, least = __builtin_amdgcn_exp2f(z + (kBelow + 7.0f));
#pragma unroll
        for (int f = 0; f < FT; ++f)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                o[f][i] *= inv;
                o[f][i] = fabsf(o[f][i]) < least ? 0.0f : o[f][i];
            }
        const bool mine = wrow + col < t.rows;
        const size_t at = ((size_t)(t.first + j) * b.H + h) * b.group.d + b.group.rest(row, j);
        if (it.pieces > 1) {                                       // [item][wave][four features][lane]: joined later
            const size_t slot = item - plan.whole;
            if (any) {
                float4_t *po = reinterpret_cast<float4_t *>(b.po + slot * ROWS * D) + wave * (D / 2) * 16 + lane;
#pragma unroll
                for (int f = 0; f < FT; ++f)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        po[(4 * f + i) * 64] = float4_t{o[f][4 * i], o[f][4 * i + 1], o[f][4 * i + 2], o[f][4 * i + 3]};
                if (hl == 0) *reinterpret_cast<float2 *>(b.pml + (slot * ROWS + 32 * wave + col) * 2) = float2{m, l};
            }
            continue;
        }
        uint16_t *dst = b.out + at * D;
#pragma unroll
        for (int f = 0; f < FT; ++f)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                auto two = [&](int k) { return (uint32_t)from_float<BF16>(o[f][k]) | (uint32_t)from_float<BF16>(o[f][k + 1]) << 16; };
                const auto s0 = __builtin_amdgcn_permlane32_swap(two(4 * i), two(4 * i + 4), false, false);
                const auto s1 = __builtin_amdgcn_permlane32_swap(two(4 * i + 2), two(4 * i + 6), false, false);
                if (any && mine) *reinterpret_cast<u32x4_t *>(dst + 32 * f + 8 * (i + hl)) = u32x4_t{(uint32_t)s0[0], (uint32_t)s1[0], (uint32_t)s0[1], (uint32_t)s1[1]};
            }
        if (any && mine && hl == 0 && b.lse) b.lse[at] = log_sum(m, l);
    }
}

// The pieces of the groups that are cut: the workgroup of piece i of n takes the i-th of n slices of the group.
template <bool BF16, int D, int NW>
__global__ __launch_bounds__(1024) void kv8_prompt_join_kernel(AttnArgs a) {
    constexpr int ROWS = 32 * NW, QUADS = NW * (D / 8) * 64;       // fours of features of a row
    const int entries = a.requests * a.tiles.d;
    __shared__ Sizes kept[kKept];
    keep_sizes(a, kept);
    auto sizes = [&](int r) { return r < kKept ? kept[r] : sizes_of(a, r); };
    __shared__ Plan plans[64];                                     // (its sixteen waves would wait for one another at the same long sums)
    if (threadIdx.x < 64) plans[threadIdx.x] = plan_of(a, ROWS, entries, sizes);
    __syncthreads();
    Plan plan = plans[threadIdx.x & 63];
    plan.per = __builtin_amdgcn_readfirstlane(plan.per);
    plan.whole = __builtin_amdgcn_readfirstlane(plan.whole);
    plan.piece = __builtin_amdgcn_readfirstlane(plan.piece);
    plan.items = __builtin_amdgcn_readfirstlane(plan.items);
    for (int item = plan.whole + blockIdx.x; item < plan.items; item += gridDim.x) {
        const Item it = item_of(a, plan, ROWS, entries, item, sizes);
        if (it.pieces <= 1) continue;
        const int r = a.tiles.of(it.entry);
        const Tile t = tile_of(a, r, a.tiles.rest(it.entry, r) * ROWS, ROWS);
        const size_t slot0 = item - plan.whole - it.at * a.H;      // of the group's first piece; the others are H further each
        const int share = ((QUADS + it.pieces - 1) / it.pieces + 63) / 64 * 64;
        for (int i = it.at * share + threadIdx.x; i < min((it.at + 1) * share, QUADS); i += 1024) {
            const int lane = i & 63, k = i / 64 % (D / 8), wave = i / 64 / (D / 8), in = 32 * wave + (lane & 31), row = t.row0 + in;
            if (row >= t.rows) continue;
            float m = -INFINITY, l = 0.0f;
            float4_t y = {0, 0, 0, 0};
            for (int w = 0; w < it.pieces; ++w) m = fmaxf(m, a.pml[((slot0 + (size_t)w * a.H) * ROWS + in) * 2]);
#pragma unroll 4
            for (int w = 0; w < it.pieces; ++w) {
                const size_t slot = slot0 + (size_t)w * a.H;
                const float2 ml = *reinterpret_cast<const float2 *>(a.pml + (slot * ROWS + in) * 2);
                const float4_t v = reinterpret_cast<const float4_t *>(a.po + slot * ROWS * D)[i];
                const float by = ml.x > -INFINITY ? __builtin_amdgcn_exp2f(ml.x - m) : 0.0f;
                const float weight = by * ml.y;                    // (of what the piece has for itself: its output is finished)
                l += weight;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] += weight * v[e];
            }
            const float inv = l != 0.0f ? 1.0f / l : 0.0f;
            const int j = a.group.of(row), d = 32 * (k / 4) + 8 * (k % 4) + 4 * (lane >> 5);
            const size_t at = ((size_t)(t.first + j) * a.H + it.head) * a.group.d + a.group.rest(row, j);
            const uint32_t y0 = from_float<BF16>(y[0] * inv) | (uint32_t)from_float<BF16>(y[1] * inv) << 16;
            const uint32_t y1 = from_float<BF16>(y[2] * inv) | (uint32_t)from_float<BF16>(y[3] * inv) << 16;
            *reinterpret_cast<u32x2_t *>(a.out + at * D + d) = u32x2_t{y0, y1};
            if (d == 0 && a.lse) a.lse[at] = log_sum(m, l);
        }
    }
}

int waves_of(const w4a4_kv8_cache &C, const w4a4_kv8_queries &Q) {
    const long rows = (long)Q.queries * (Q.heads / C.heads);
    return rows <= 128 || C.features == 256 ? 4 : 8;              // (256 features: a wave's registers leave room for one on a SIMD)
}

template <bool BF16, int D, int NW>
int launch(AttnArgs &a, hipStream_t st) {
    auto kern = kv8_prompt_kernel<BF16, D, NW>;
    constexpr size_t lds = 2 * kBuffer<D>;
    static KernelState ks;
    const void *fn = reinterpret_cast<const void *>(kern);
    const int cus = prepare_kernel(fn, lds, ks);
    if (cus < 0) return W4A4_ERR_HIP;
    const int at_once = resident_per_cu(fn, NW * 64, lds, ks);
    if (at_once <= 0) return W4A4_ERR_HIP;
    a.slots = min(kMostPieces, cus * at_once);
    hipLaunchKernelGGL(kern, dim3((unsigned)a.slots), dim3(NW * 64), lds, st, a);
    hipLaunchKernelGGL((kv8_prompt_join_kernel<BF16, D, NW>), dim3((unsigned)cus), dim3(1024), 0, st, a);
    return launch_status();
}

}  // namespace

bool kv8_prompt_wanted(const w4a4_kv8_cache &C, const w4a4_kv8_queries &Q) { return (long)Q.queries * (Q.heads / C.heads) > kFewRows; }

int kv8_prompt_tiles(const w4a4_kv8_cache &C, const w4a4_kv8_queries &Q) {
    const int rows = 32 * waves_of(C, Q);
    return (int)(((long)Q.queries * (Q.heads / C.heads) + rows - 1) / rows);
}

size_t kv8_prompt_workspace_bytes(const w4a4_kv8_cache &C, const w4a4_kv8_queries &Q) {
    return (size_t)kMostPieces * 32 * waves_of(C, Q) * (C.features + 2) * sizeof(float);
}

int kv8_prompt(AttnArgs a, const w4a4_kv8_cache &C, const w4a4_kv8_queries &Q, float *parts, hipStream_t st) {
    const int nw = waves_of(C, Q);
    a.po = parts;
    a.pml = parts + (size_t)kMostPieces * 32 * nw * C.features;
    auto run = [&](auto bf16, auto d) {
        constexpr bool BF = decltype(bf16)::value;
        constexpr int D = decltype(d)::value;
        if constexpr (D <= 128)
            if (nw == 8) return launch<BF, D, 8>(a, st);
        return launch<BF, D, 4>(a, st);
    };
    auto typed = [&](auto d) { return Q.dtype == W4A4_BF16 ? run(std::true_type{}, d) : run(std::false_type{}, d); };
    switch (C.features) {
        case 64: return typed(std::integral_constant<int, 64>{});
        case 96: return typed(std::integral_constant<int, 96>{});
        case 128: return typed(std::integral_constant<int, 128>{});
        default: return typed(std::integral_constant<int, 256>{});
    }
}

}  // namespace w4a4
