// Block bookkeeping of one step of token generation, in one launch.
//
// For every request the number of blocks that its new tokens need, the running sums of those, of the tokens and of the blocks
// that ended requests give back; then each request takes its blocks from the ring of free ones at its own offset, every new token
// gets its slot and position, and the blocks given back go behind the free ones.  The sums are what all of it
// waits for and cost little (two words per request), so every workgroup computes them over all requests by itself, and no
// workgroup waits for another.  A workgroup then serves up to kChunk requests; where tokens are many, several
// workgroups share them (blockIdx.y).
//
// Nothing is read that another workgroup writes: the slot of a token in a new block is taken from the ring, not from
// the table, and the free part of the ring does not overlap what is given back.
//
// Bound by latency: the requests' words, the sums, the ring's and the table's words, one after the other.  Sums run over lanes
// (data-parallel primitives) and then over waves, three at a time; 64 requests take 256 threads, thousands 1024.
// Measured: 64 requests of one token each 4.5 us; 2999 requests, prompts, single tokens and ended ones mixed, 7.2 us (sums by shuffles
// and ended requests served by sixteen lanes each: 9.9).
#include "gen.hpp"

namespace w4a4 {
namespace {

constexpr int kChunk = 64;

struct PlanArgs {
    const int32_t *lens, *fresh, *state;
    int32_t *table, *ring, *state_out, *lens_out, *start, *slots, *positions;
    int requests, width, capacity, shift, tokens, chunk;           // (blocks of 1 << shift tokens; requests of a workgroup)
};

struct Request {                       // what one request asks for
    int len, have, back;
    unsigned add, need;
    bool fits, give;
};

__device__ __forceinline__ Request request_of(const PlanArgs &a, int len, int n) {
    Request q;
    q.len = len;
    const long room = (long)a.width << a.shift, round_up = (1 << a.shift) - 1;
    const bool bad = len < 0 || len > room;
    q.add = max(n, 0);
    q.fits = !bad && n >= 0 && (long)len + q.add <= room;
    q.give = !bad && n < 0;
    q.have = bad ? 0 : (int)((len + round_up) >> a.shift);
    q.need = q.fits ? (unsigned)(((long)len + q.add + round_up) >> a.shift) - q.have : 0;
    q.back = q.give ? q.have : 0;
    return q;
}

__device__ __forceinline__ int wrap(unsigned at, int capacity) {
    if (at < (unsigned)capacity) return (int)at;
    at -= capacity;
    return at < (unsigned)capacity ? (int)at : (int)(at % (unsigned)capacity);
}

// (sums of tokens stop at the largest number instead of beginning again: nothing that is wrong with a request's words moves a place backwards)
__device__ __forceinline__ unsigned plus(unsigned x, unsigned y) { return __builtin_elementwise_add_sat(x, y); }

template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned shifted(unsigned x) { return __builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false); }
__device__ __forceinline__ unsigned upto16(unsigned x) {           // sums of the lanes of a row up to each
    x = plus(x, shifted<0x111, 0xF>(x));
    x = plus(x, shifted<0x112, 0xF>(x));
    x = plus(x, shifted<0x114, 0xF>(x));
    return plus(x, shifted<0x118, 0xF>(x));
}
__device__ __forceinline__ unsigned upto64(unsigned x) {           // of the lanes of a wave
    x = upto16(x);
    x = plus(x, shifted<0x142, 0xA>(x));
    return plus(x, shifted<0x143, 0xC>(x));
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void kv8_plan_kernel(PlanArgs a) {
    __shared__ unsigned part[3][16];
    __shared__ unsigned c_start[kChunk + 1], c_take[kChunk], c_back[kChunk], c_need[kChunk];
    __shared__ int c_served[kChunk], c_len[kChunk], c_have[kChunk], c_give[kChunk];
    __shared__ unsigned s_taken;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (a.requests + THREADS - 1) / THREADS;
    const int r0 = min(tid * per, a.requests), r1 = min(r0 + per, a.requests);
    const int c0 = blockIdx.x * a.chunk, cn = min(a.chunk, a.requests - c0);
    const int state0 = a.state[0], state1 = a.state[1];
    if (tid == 0) {
        s_taken = 0;
        c_start[0] = 0;                                            // (no requests at all)
    }
    if (tid < 16) part[0][tid] = part[1][tid] = part[2][tid] = 0;
    __syncthreads();

    // sums of new tokens, of blocks wanted, of blocks given back: of this thread's requests, then of all before them
    unsigned sum[3] = {0, 0, 0};
    int len = 0, n = 0;
#pragma unroll 4
    for (int r = r0; r < r1; ++r) {
        len = a.lens[r];
        n = a.fresh[r];
        const Request q = request_of(a, len, n);
        sum[0] = plus(sum[0], q.add);
        sum[1] = plus(sum[1], q.need);
        sum[2] = plus(sum[2], q.back);
    }
    unsigned before[3], total[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const unsigned upto = upto64(sum[k]), ahead = __builtin_amdgcn_update_dpp(0, (int)upto, 0x138, 0xF, 0xF, false);   // the lane before
        before[k] = ahead;
        if (lane == 63) part[k][wave] = upto;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const unsigned upto = upto16(part[k][lane & 15]);
        total[k] = __builtin_amdgcn_readlane(upto, 15);
        if (wave) before[k] = plus(before[k], __builtin_amdgcn_readlane(upto, wave - 1));
    }
    const unsigned free = max(state1, 0);
    const int head = wrap(max(state0, 0), a.capacity);
    const bool last = blockIdx.x == gridDim.x - 1;
    unsigned taken = 0;
    for (int r = r0; r < r1; ++r) {
        if (per > 1) {
            len = a.lens[r];
            n = a.fresh[r];
        }
        const Request q = request_of(a, len, n);
        const unsigned upto = plus(before[1], q.need);
        const bool served = q.fits && (q.need == 0 || upto <= free);
        if (served && q.need) taken = upto;                        // (what is served is a prefix of what is wanted)
        if (r >= c0 && r < c0 + cn) {
            const int i = r - c0;
            c_start[i] = before[0];
            c_take[i] = before[1];
            c_back[i] = before[2];
            c_need[i] = served ? q.need : 0;
            c_served[i] = served;
            c_give[i] = q.back;
            c_len[i] = q.len;
            c_have[i] = q.have;
            if (i == cn - 1) c_start[cn] = plus(before[0], q.add);
            if (blockIdx.y == 0) {
                a.start[r] = (int)min(before[0], 0x7fffffffu);
                a.lens_out[r] = q.give ? 0 : served ? q.len + (int)q.add : q.len;
            }
        }
        before[0] = plus(before[0], q.add);
        before[1] = upto;
        before[2] = plus(before[2], q.back);
    }
    if (last && blockIdx.y == 0) {
        taken = lanes_reduce<64>(taken, [](unsigned x, unsigned y) { return x > y ? x : y; });
        if (lane == 0 && taken) atomicMax(&s_taken, taken);
    }
    __syncthreads();
    if (last && blockIdx.y == 0 && tid == 0) {
        a.start[a.requests] = (int)min(total[0], 0x7fffffffu);
        a.state_out[0] = wrap(head + s_taken, a.capacity);
        a.state_out[1] = (int)(state1 - s_taken + total[2]);
    }

    // slots and positions: a thread per token
    const unsigned t1 = min(c_start[max(cn, 0)], (unsigned)a.tokens);
    for (unsigned long t = c_start[0] + (unsigned long)blockIdx.y * THREADS + tid; t < t1; t += (unsigned long)gridDim.y * THREADS) {
        int lo = 0, hi = cn;                                       // the last request that starts at t or before, among those with tokens
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (c_start[mid] <= t) lo = mid;
            else hi = mid;
        }
        int slot = -1, pos = -1;
        if (c_served[lo]) {
            pos = c_len[lo] + (int)(t - c_start[lo]);
            const int b = pos >> a.shift, have = c_have[lo];
            const int id = b < have ? a.table[(size_t)(c0 + lo) * a.width + b] : a.ring[wrap(head + c_take[lo] + (b - have), a.capacity)];
            // (what cannot be a block's number makes no slot: shifted out of its word it would be another block's)
            if ((unsigned)id < 0x80000000u >> a.shift) slot = (id << a.shift) + (pos & ((1 << a.shift) - 1));
        }
        a.slots[t] = slot;
        a.positions[t] = pos;
    }
    if (last)                                                      // what no request owns
        for (unsigned long t = total[0] + (unsigned long)blockIdx.y * THREADS + tid; t < (unsigned long)a.tokens; t += (unsigned long)gridDim.y * THREADS)
            a.slots[t] = a.positions[t] = -1;
    // tables and ring: sixteen lanes per request that takes blocks; a wave per ended one, which may give back hundreds (four of its
    // words a lane are under way at once)
    if (blockIdx.y == 0) {
        for (int i = tid >> 4; i < cn; i += THREADS / 16) {
            int32_t *row = a.table + (size_t)(c0 + i) * a.width + c_have[i];
            const unsigned need = c_need[i];
            for (unsigned j = tid & 15; j < need; j += 16) row[j] = a.ring[wrap(head + c_take[i] + j, a.capacity)];
        }
        int turn = 0;
        for (unsigned long long ended = __ballot(lane < cn && c_give[lane] > 0); ended; ended &= ended - 1, ++turn) {
            if (turn % (THREADS / 64) != wave) continue;
            const int i = __builtin_ctzll(ended);
            const int32_t *row = a.table + (size_t)(c0 + i) * a.width;
            const unsigned back = c_give[i];
            for (unsigned j0 = lane; j0 < back; j0 += 256) {
                int id[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) id[k] = j0 + 64 * k < back ? row[j0 + 64 * k] : 0;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (j0 + 64 * k < back) a.ring[wrap(head + free + c_back[i] + j0 + 64 * k, a.capacity)] = id[k];
            }
        }
    }
}

}  // namespace
}  // namespace w4a4

using namespace w4a4;

extern "C" int w4a4_kv8_plan(const int32_t *lens, const int32_t *new_tokens, int requests, int32_t *table, int width, int32_t *ring,
                             int capacity, const int32_t *state, int block, int tokens, int32_t *state_out, int32_t *lens_out,
                             int32_t *start, int32_t *slots, int32_t *positions, void *stream) {
    if (requests < 0 || width < 0 || capacity <= 0 || block <= 0 || tokens < 0) return W4A4_ERR_INVALID_ARG;
    if (!ring || !state || !state_out || !start || (tokens && (!slots || !positions))) return W4A4_ERR_INVALID_ARG;
    if (requests && (!lens || !new_tokens || !lens_out || (width && !table))) return W4A4_ERR_INVALID_ARG;
    if (state == state_out || (requests && lens == lens_out)) return W4A4_ERR_INVALID_ARG;
    if (!kv8_block_ok(block) || (long)capacity * block > 0x7fffffffL) return W4A4_ERR_UNSUPPORTED_SHAPE;
    if ((long)requests * width > 0x7fffffffL) return W4A4_ERR_UNSUPPORTED_SHAPE;           // (blocks are counted in 32 bits)
    // Requests of a workgroup: sixteen, more where the device would have no CU for the workgroups; a batch of single tokens in few ones.
    const int chunk = requests <= 256 ? kChunk : min(kChunk, max(16, (requests + 255) / 256));
    const PlanArgs a{lens, new_tokens, state, table, ring, state_out, lens_out, start, slots, positions, requests, width, capacity, __builtin_ctz(block), tokens, chunk};
    const int chunks = requests ? (requests + chunk - 1) / chunk : 1;
    const int shares = max(1, min(16, tokens / (chunks * 4096)));
    const dim3 grid(chunks, shares);
    // us: 64 requests of one token 4.5, 2999 of up to 300 tokens 7.2 (with sixteen lanes for each ended request 9.9)
    if (requests <= 256) hipLaunchKernelGGL(kv8_plan_kernel<256>, grid, dim3(256), 0, as_stream(stream), a);
    else hipLaunchKernelGGL(kv8_plan_kernel<1024>, grid, dim3(1024), 0, as_stream(stream), a);
    return launch_status();
}
