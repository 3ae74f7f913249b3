// Linear layers of many tokens whose operands are both microscaled 4-bit floating point: tiles in LDS.
//
// The arithmetic is that of mx4_linear.hip, on the 32 x 32 form of the matrix instruction, two of which take a plane of 128 numbers.
//   * A stage of the ring in LDS is one plane of the tile's BM token rows and BN channel rows, 64 bytes of codes and a word of exponents each.  In
//     memory the rows of a plane follow each other, so every DMA instruction moves sixteen whole rows, a kilobyte; a descriptor for each plane
//     ends at the matrix's last row, behind which rows read as zeros.
//   * Sixteen lanes that read operands together read sixteen rows, 64 bytes apart or FN times that: the four pieces of a row
//     change places with the row (XOR), and a block's channel rows are put in the order in which lanes want them, so that the
//     sixteen reads fall into sixteen different groups of four banks.  A lane's channels are FN neighbours, which it stores together.
//   * A lane of half h has pieces 2h and 2h + 1 of a plane, so one shift brings both bytes of exponents to where the instruction selects them.
//   * While a plane is multiplied, the next one's operands are read and NS - 1 others are on their way; one barrier a plane, behind a matrix instruction.
//
// What bounds it: 8192 x 8192 x 8192 263 us = 4.2 PFLOP/s by tiles of 256 x 256, of 6.1 that registers full of such operands reach (8.9 where they are zeros: it is the
// power that is short); without its DMA 214, without its stores 247, on zeros 204; matrix pipe 58 % of the cycles, no conflict in LDS.  Small K is bound by the
// results: 16384 x 16384 x 1024 195 us = 2.8 TB/s of results by 128 x 256, and 229 with fp16's GELU, whose eleven instructions a number are 50 us of every SIMD's time and
// (bf16's has fifteen: 13 us more) run beside other workgroups' products only in part.  Few tokens are bound by what a CU takes in: 301 tokens 4096 x 1056 5.0 us by 64 x 128.
#include "gemm_common.hpp"
#include "mx4.hpp"
#include "mx4_linear.hpp"

namespace w4a4 {
namespace {

typedef __attribute__((address_space(3))) void *lds_t;

constexpr int vm_and_lds(int n) { return (n & 0xF) | (0x7 << 4) | (0x0 << 8) | (((n >> 4) & 0x3) << 14); }   // vmcnt <= n, lgkmcnt == 0

// Where in a block of sixteen rows (64 pieces of 16 bytes) row r's piece k lies, when lanes read every F-th row: the block's number b
// tells apart those of one read.
template <int F>
__device__ __forceinline__ int place_row(int r) { return r / F + 16 / F * (r % F); }
template <int F>
__device__ __forceinline__ int row_at(int place) { return place % (16 / F) * F + place / (16 / F); }
template <int F>
__device__ __forceinline__ int turn_of_row(int r, int b) { return F == 4 ? b & 3 : F == 2 ? ((r / 2) >> 2) + 2 * (b & 1) : r >> 2; }

// One tile from (m0, n0) on: WM x WN waves of FM x FN fragments, KS times that with every KS-th plane each; a ring of NS steps.
template <int FM, int FN, int WM, int WN, int KS, int NS, bool BF16>
__device__ __forceinline__ void tile(const MX4LinearArgs &g, uint8_t *smem, int m0, int n0) {
    constexpr int BM = WM * FM * 32, BN = WN * FN * 32, NW = WM * WN, ROWS = BM + BN;
    constexpr int CODES = ROWS / 16, SCALES = ROWS / 64;           // DMA instructions of a plane
    constexpr int CPW = CODES / NW, SPW = (SCALES + NW - 1) / NW, LD = CPW + SPW;               // of a wave
    constexpr int PLANE = ROWS * 68, STAGE = KS * PLANE, NM = FM * FN, NF = FM + FN, RPS = (NF + NM - 2) / (NM - 1);   // operand reads behind a product
    static_assert((FN == 2 || FN == 4) && BM % 64 == 0 && BN % 64 == 0 && CODES % NW == 0, "whole DMA instructions, the same number for every wave");
    static_assert((NS - 1) * LD <= 63, "ring depth");
    uint8_t *dummy = smem + NS * STAGE;                            // of waves that have no exponents to fetch
    const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ks = all / NW, wave = all % NW, wm = wave / WN, wn = wave % WN;
    const int h = lane >> 5, cc = lane & 31;
    const int a_row = wm * FM * 32 + cc, w_row = wn * FN * 32 + cc * FN, n = n0 + w_row;  // of the lane's first fragments, in the tile; its first channel
    // the lane's biases (zeros past the last channel), requested in front of the tile's DMA: loads return in order
    const __amdgpu_buffer_rsrc_t bias_rsrc = make_rsrc(g.bias, g.bias && ks == 0 ? (uint32_t)g.N * 2 : 0);
    u32x2 bias = {0, 0};
    if constexpr (FN == 4) bias = __builtin_amdgcn_raw_buffer_load_b64(bias_rsrc, n * 2, 0, 0);
    else bias[0] = __builtin_amdgcn_raw_buffer_load_b32(bias_rsrc, n * 2, 0, 0);

    // ---- what this wave fetches of a stage ----
    int voff[CPW];
#pragma unroll
    for (int i = 0; i < CPW; ++i) {
        const int b = wave + i * NW, place = lane >> 2;            // block of sixteen rows of [tokens | channels]
        const bool chan = b >= BM / 16;
        const int bb = chan ? b - BM / 16 : b, r = chan ? row_at<FN>(place) : place;
        voff[i] = bb * 1024 + r * 64 + ((lane & 3) ^ (chan ? turn_of_row<FN>(r, bb) : turn_of_row<1>(r, bb))) * 16;
    }
    const uint32_t a_rows = (uint32_t)min(BM, g.M - m0), w_rows = (uint32_t)min(BN, g.N - n0);
    auto fetch = [&](int i, int stage, int step) {                 // instruction i of this wave's plane of a step
        const int c = step * KS + ks;
#if defined(__HIP_DEVICE_COMPILE__)   // (the host pass rejects the cast to an address in LDS)
        const bool there = c < g.planes;
        const size_t at_a = (size_t)c * g.M + m0, at_w = (size_t)c * g.N + n0;
        if (i < CPW) {
            const int b = wave + i * NW;
            const bool chan = b >= BM / 16;
            const __amdgpu_buffer_rsrc_t rs = make_rsrc(chan ? g.w + at_w * kPlaneBytes : g.a + at_a * kPlaneBytes, there ? (chan ? w_rows : a_rows) * kPlaneBytes : 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_t)(smem + stage * STAGE + ks * PLANE + b * 1024), 16, voff[i], 0, 0, 0);
        } else {
            const int b = wave + (i - CPW) * NW;                   // 64 rows
            const bool chan = b >= BM / 64;
            const int bb = chan ? b - BM / 64 : b;
            const __amdgpu_buffer_rsrc_t rs = make_rsrc(chan ? g.sw + at_w : g.sa + at_a, there && b < SCALES ? (chan ? w_rows : a_rows) * 4 : 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_t)(b < SCALES ? smem + stage * STAGE + ks * PLANE + ROWS * 64 + b * 256 : dummy), 4, (bb * 64 + lane) * 4, 0, 0, 0);
        }
#else
        (void)i, (void)stage, (void)c, (void)a_rows, (void)dummy, (void)w_rows;
#endif
    };

    // ---- operands ----
    const int a_at = (a_row >> 4) * 1024 + (a_row & 15) * 64 + ((2 * h) ^ turn_of_row<1>(a_row & 15, 0)) * 16;
    const int w_at = BM * 64 + (w_row >> 4) * 1024 + place_row<FN>(w_row & 15) * 64 + ((2 * h) ^ turn_of_row<FN>(w_row & 15, w_row >> 4)) * 16;
    auto read = [&](int f, int stage, int s) {                     // fragment f (tokens first), piece 2h + s
        const int at = f < FM ? a_at + f * 2048 : w_at + (f - FM) * (16 / FN * 64);
        return *reinterpret_cast<const u32x4_t *>(smem + stage * STAGE + ks * PLANE + (at ^ (16 * s)));
    };
    struct Scales { uint32_t a[FM], w[FN]; } sc, sn;
    auto read_scales = [&](int stage) {
        const uint8_t *p = smem + stage * STAGE + ks * PLANE + ROWS * 64;
#pragma unroll
        for (int i = 0; i < FM; ++i) sn.a[i] = *reinterpret_cast<const uint32_t *>(p + (a_row + 32 * i) * 4);
        const uint32_t *w = reinterpret_cast<const uint32_t *>(p + (BM + w_row) * 4);
#pragma unroll
        for (int j = 0; j < FN; ++j) sn.w[j] = w[j];
    };
    auto next_scales = [&]() {
#pragma unroll
        for (int i = 0; i < FM; ++i) sc.a[i] = sn.a[i] >> (16 * h);
#pragma unroll
        for (int j = 0; j < FN; ++j) sc.w[j] = sn.w[j] >> (16 * h);
    };
    auto in_order = [](int k) { return k == 0 ? 0 : k <= FN ? FM + k - 1 : k - FN; };      // A0, W0 .. , A1 ..: as the products want them

#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < LD; ++i) fetch(i, s, s);
    __builtin_amdgcn_s_waitcnt(vm_and_lds((NS - 1) * LD));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    v16f acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = to_float<BF16>((uint16_t)(bias[j / 2] >> (16 * (j % 2))));
    u32x4_t P[2][NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) P[0][f] = read(f, 0, 0);
    read_scales(0);
    next_scales();
    auto multiply = [&](int k, auto sub) {
        constexpr int S = decltype(sub)::value;
        const int i = k / FN, j = k % FN;
        const u32x4_t x = P[S][i], w = P[S][FM + j];
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v8i_t{(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0},
                                                                    v8i_t{(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0}, acc[i][j], 4, 4, S, (int)sc.a[i], S, (int)sc.w[j]);
    };
    int cur = 0;
    for (int c = 0, steps = (g.planes + KS - 1) / KS; c < steps; ++c) {
        const int nxt = cur == NS - 1 ? 0 : cur + 1;
#pragma unroll
        for (int k = 0; k < NM; ++k) {
            multiply(k, std::integral_constant<int, 0>{});
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = RPS * k; x < RPS * (k + 1) && x < NF; ++x) P[1][in_order(x)] = read(in_order(x), cur, 1);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int k = 0; k < NM; ++k) {
            multiply(k, std::integral_constant<int, 1>{});
            __builtin_amdgcn_sched_barrier(0);
            if (k == 0) {
                // the next plane has landed, and nobody reads this one any more
                __builtin_amdgcn_s_waitcnt(vm_and_lds((NS - 2) * LD));
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
            } else {
                if (k == 1) read_scales(nxt);
#pragma unroll
                for (int x = RPS * (k - 1); x < RPS * k && x < NF; ++x) P[0][in_order(x)] = read(in_order(x), nxt, 0);
#pragma unroll
                for (int i = (k - 1) * LD / (NM - 1); i < k * LD / (NM - 1); ++i) fetch(i, cur, c + NS);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        next_scales();
        cur = nxt;
    }
    __builtin_amdgcn_s_waitcnt(vm_and_lds(0));                     // no DMA may outlive the workgroup's LDS

    // ---- results: the lane's FN neighbouring channels of a token at a time ----
    const __amdgpu_buffer_rsrc_t out = make_rsrc(g.out + (size_t)m0 * g.N, a_rows * (uint32_t)g.N * 2);
    const uint32_t col = n < g.N ? (uint32_t)n * 2 : kPoison;      // (a lane's channels are all there or none)
    if constexpr (KS > 1) {                                        // the waves of a tile take a share of its registers each, in the order of K
        __syncthreads();
        float *sums = reinterpret_cast<float *>(smem);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e)
#pragma unroll
                for (int j = 0; j < FN; ++j) sums[((all * FM + i) * 16 + e) * (FN * 64) + j * 64 + lane] = acc[i][j][e];
        __syncthreads();
    }
    auto results = [&](auto f) {                                   // f(byte in the tile's rows, the lane's sums)
        if constexpr (KS == 1) {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float y[FN];
#pragma unroll
                    for (int j = 0; j < FN; ++j) y[j] = acc[i][j][e];
                    f((uint32_t)(wm * FM * 32 + i * 32 + 8 * (e >> 2) + 4 * h + (e & 3)) * (uint32_t)g.N * 2 + col, y);
                    if (e % 2) __builtin_amdgcn_sched_barrier(0);  // (or more of it is begun at once than there are registers for)
                }
        } else {
            const float *sums = reinterpret_cast<const float *>(smem) + wave * (NM * 16 * 64) + lane;
            for (int r = ks; r < FM * 16; r += KS) {
                float y[FN];
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    y[j] = 0.0f;
#pragma unroll
                    for (int k = 0; k < KS; ++k) y[j] += sums[k * (NW * NM * 16 * 64) + (r * FN + j) * 64];
                }
                f((uint32_t)(wm * FM * 32 + (r >> 4) * 32 + 8 * (r >> 2 & 3) + 4 * h + (r & 3)) * (uint32_t)g.N * 2 + col, y);
            }
        }
    };
    uint32_t w[FN / 2];
    if (g.act != W4A4_ACT_GELU) {
        results([&](uint32_t at, float (&y)[FN]) {
#pragma unroll
            for (int j = 0; j < FN; j += 2) w[j / 2] = from_float<BF16>(y[j]) | (uint32_t)from_float<BF16>(y[j + 1]) << 16;
            store_words<FN / 2, kStreamed>(out, at, w);
        });
        return;
    }
    results([&](uint32_t at, float (&y)[FN]) {
        float finite = 0.0f;                                       // NaN where a sum is none or infinite: those are done again, with care
#pragma unroll
        for (int j = 0; j < FN; j += 2) {
            finite = __fmaf_rn(y[j], 0.0f, __fmaf_rn(y[j + 1], 0.0f, finite));
            w[j / 2] = mx4_gelu2<BF16>(y[j], y[j + 1]);
        }
        if (__builtin_expect(finite != 0.0f, 0))
#pragma unroll
            for (int j = 0; j < FN; j += 2) {
                if (!(fabsf(y[j]) < INFINITY)) w[j / 2] = (w[j / 2] & 0xFFFF0000u) | from_float<BF16>(mx4_gelu_limit(y[j]));
                if (!(fabsf(y[j + 1]) < INFINITY)) w[j / 2] = (w[j / 2] & 0xFFFFu) | (uint32_t)from_float<BF16>(mx4_gelu_limit(y[j + 1])) << 16;
            }
        store_words<FN / 2, kStreamed>(out, at, w);
    });
}

// Tiles of an XCD follow each other, eight rows of tiles a column at a time.  The tiles behind `whole`, too few for another round of workgroups, are
// taken in quarters (TAIL).
template <int FM, int FN, int WM, int WN, int KS, int NS, int OCC, bool TAIL, bool BF16>
__global__ __attribute__((amdgpu_flat_work_group_size(WM *WN *KS * 64, WM *WN *KS * 64), amdgpu_waves_per_eu(OCC, OCC)))
void mx4_tiles_kernel(MX4LinearArgs g) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    constexpr int BM = WM * FM * 32, BN = WN * FN * 32;
    const bool part = TAIL && (int)blockIdx.x >= g.whole;
    const int u = TAIL && part ? xcd_tile(blockIdx.x - g.whole, gridDim.x - g.whole) : 0;
    const int t = TAIL && part ? g.whole + u / 4 : xcd_tile(blockIdx.x, TAIL ? g.whole : (int)gridDim.x);
    const int first = t / (8 * g.tiles_n) * 8, deep = min(8, g.tiles_m - first), rest = t - first * g.tiles_n;
    int m0 = (first + rest % deep) * BM, n0 = rest / deep * BN;
    if constexpr (TAIL) {
        if (part) {
            m0 += u / 2 % 2 * (BM / 2);
            n0 += u % 2 * (BN / 2);
            if (m0 < g.M && n0 < g.N) tile<FM / 2, FN / 2, WM, WN, KS, NS, BF16>(g, smem, m0, n0);
            return;
        }
    }
    tile<FM, FN, WM, WN, KS, NS, BF16>(g, smem, m0, n0);
}

template <int FM, int FN, int WM, int WN, int KS, int NS, int OCC, bool TAIL, bool BF16>
int launch(MX4LinearArgs g, hipStream_t st) {
    auto kern = mx4_tiles_kernel<FM, FN, WM, WN, KS, NS, OCC, TAIL, BF16>;
    constexpr int BM = WM * FM * 32, BN = WN * FN * 32;
    constexpr size_t ring = (size_t)NS * KS * (BM + BN) * 68 + 256, sums = KS > 1 ? (size_t)KS * BM * BN * 4 : 0, lds = ring > sums ? ring : sums;
    static_assert(lds <= 160 * 1024, "a CU's LDS");
    g.tiles_m = (int)(((long)g.M + BM - 1) / BM);
    g.tiles_n = (int)(((long)g.N + BN - 1) / BN);
    const long tiles = (long)g.tiles_m * g.tiles_n;                // (mx4_way has asked whether they are a launch)
    static KernelState ks;
    const int cus = prepare_kernel(reinterpret_cast<const void *>(kern), lds, ks);
    if (cus < 0) return W4A4_ERR_HIP;
    g.whole = (int)tiles;
    if (TAIL) {
        const int slots = cus, left = (int)(tiles % slots);
        if (tiles > slots && 4 * left <= slots && grid_fits(tiles + 3 * left, WM * WN * KS * 64)) g.whole = (int)tiles - left;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.whole + 4 * (tiles - g.whole))), dim3(WM * WN * KS * 64), lds, st, g);
    return launch_status();
}

template <int FM, int FN, int WM, int WN, int KS, int NS, int OCC, bool TAIL = false>
int typed(const MX4LinearArgs &g, int dtype, hipStream_t st) {
    return dtype == W4A4_BF16 ? launch<FM, FN, WM, WN, KS, NS, OCC, TAIL, true>(g, st) : launch<FM, FN, WM, WN, KS, NS, OCC, TAIL, false>(g, st);
}

}  // namespace

int mx4_tiles(const MX4LinearArgs &g, int dtype, MX4Tile tile, hipStream_t st) {
    switch (tile) {
        case kMX4Tile64x64: return typed<1, 2, 2, 1, 4, 4, 2>(g, dtype, st);              // K in four parts, two waves each
        case kMX4Tile64x128: return typed<1, 2, 2, 2, 1, 3, 4>(g, dtype, st);             // four waves; four workgroups a CU
        case kMX4Tile128x128: return typed<2, 2, 2, 2, 1, 3, 3>(g, dtype, st);            // three
        case kMX4Tile128x256: return typed<2, 4, 2, 2, 1, 3, 2>(g, dtype, st);            // two
        default: return typed<2, 4, 4, 2, 1, 4, 2, true>(g, dtype, st);                   // eight waves, one workgroup a CU
    }
}

}  // namespace w4a4
