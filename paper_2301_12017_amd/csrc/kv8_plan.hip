// Block bookkeeping of one step of token generation, in one launch.
//
// For every request the number of blocks that its new tokens need, the running sums of those, of the tokens and of the blocks
// that ended requests give back; then each request takes its blocks from the ring of free ones at its own offset, every new token
// gets its slot and position, and the blocks given back go behind the free ones.  The sums are what all of it
// waits for and cost little (three words per request), so every workgroup computes them over all requests by itself, and no
// workgroup waits for another.  A workgroup then serves kChunk requests; where tokens are many, several
// workgroups share them (blockIdx.y).
//
// Nothing is read that another workgroup writes: the slot of a token in a new block is taken from the ring, not from
// the table, and the free part of the ring does not overlap what is given back.
#include "gen.hpp"

namespace w4a4 {
namespace {

constexpr int kPlanThreads = 1024, kChunk = 64;

struct PlanArgs {
    const int32_t *lens, *fresh, *state;
    int32_t *table, *ring, *state_out, *lens_out, *start, *slots, *positions;
    int requests, width, capacity, shift, tokens;              // (blocks of 1 << shift tokens)
};

struct Request {                       // what one request asks for
    int len, add, have, need, back;
    bool fits, give;
};

__device__ __forceinline__ Request request_of(const PlanArgs &a, int r) {
    Request q;
    q.len = a.lens[r];
    const int n = a.fresh[r];
    const long room = (long)a.width << a.shift, round_up = (1 << a.shift) - 1;
    const bool bad = q.len < 0 || q.len > room;
    q.add = max(n, 0);
    q.fits = !bad && n >= 0 && (long)q.len + q.add <= room;
    q.give = !bad && n < 0;
    q.have = bad ? 0 : (int)((q.len + round_up) >> a.shift);
    q.need = q.fits ? (int)(((long)q.len + q.add + round_up) >> a.shift) - q.have : 0;
    q.back = q.give ? q.have : 0;
    return q;
}

__device__ __forceinline__ int wrap(long at, int capacity) {       // at >= 0
    if (at < capacity) return (int)at;
    if (at < 2L * capacity) return (int)(at - capacity);
    return (int)((unsigned long)at % (unsigned)capacity);
}

__global__ __launch_bounds__(kPlanThreads) void kv8_plan_kernel(PlanArgs a) {
    __shared__ long part[3][kPlanThreads / 64];
    __shared__ long c_start[kChunk + 1], c_take[kChunk], c_back[kChunk];
    __shared__ int c_served[kChunk];
    __shared__ long s_taken;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (a.requests + kPlanThreads - 1) / kPlanThreads;
    const int r0 = min(tid * per, a.requests), r1 = min(r0 + per, a.requests);
    const int c0 = blockIdx.x * kChunk, cn = min(kChunk, a.requests - c0);
    const long free = max(a.state[1], 0);
    const int head = wrap(max(a.state[0], 0), a.capacity);
    if (tid == 0) {
        s_taken = 0;
        c_start[0] = 0;                                            // (no requests at all)
    }

    // sums of new tokens, of blocks wanted, of blocks given back: of this thread's requests, then of all before them
    long sum[3] = {0, 0, 0};
    for (int r = r0; r < r1; ++r) {
        const Request q = request_of(a, r);
        sum[0] += q.add;
        sum[1] += q.need;
        sum[2] += q.back;
    }
    long before[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        long v = sum[k];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long u = __shfl_up(v, o, 64);
            if (lane >= o) v += u;
        }
        before[k] = v - sum[k];
        if (lane == 63) part[k][wave] = v;
    }
    __syncthreads();
    long total[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        long v = 0, all = 0;
        for (int w = 0; w < kPlanThreads / 64; ++w) {
            if (w == wave) v = all;
            all += part[k][w];
        }
        before[k] += v;
        total[k] = all;
    }
    long taken = 0;
    for (int r = r0; r < r1; ++r) {
        const Request q = request_of(a, r);
        const long upto = before[1] + q.need;
        const bool served = q.fits && (q.need == 0 || upto <= free);
        if (served && q.need) taken = upto;                        // (what is served is a prefix of what is wanted)
        if (r >= c0 && r < c0 + cn) {
            c_start[r - c0] = before[0];
            c_take[r - c0] = before[1];
            c_back[r - c0] = before[2];
            c_served[r - c0] = served;
            if (r == c0 + cn - 1) c_start[cn] = before[0] + q.add;
            if (blockIdx.y == 0) {
                a.start[r] = (int)before[0];
                a.lens_out[r] = q.give ? 0 : served ? q.len + q.add : q.len;
            }
        }
        before[0] += q.add;
        before[1] = upto;
        before[2] += q.back;
    }
    const bool last = blockIdx.x == gridDim.x - 1;
    if (last && blockIdx.y == 0 && taken) atomicMax((unsigned long long *)&s_taken, (unsigned long long)taken);
    __syncthreads();
    if (last && blockIdx.y == 0 && tid == 0) {
        a.start[a.requests] = (int)total[0];
        a.state_out[0] = wrap(head + s_taken, a.capacity);
        a.state_out[1] = (int)(a.state[1] - s_taken + total[2]);
    }

    // tables and ring: a wave per request
    if (blockIdx.y == 0)
        for (int i = wave; i < cn; i += kPlanThreads / 64) {
            const Request q = request_of(a, c0 + i);
            int32_t *row = a.table + (size_t)(c0 + i) * a.width;
            if (c_served[i])
                for (int j = lane; j < q.need; j += 64) row[q.have + j] = a.ring[wrap(head + c_take[i] + j, a.capacity)];
            for (int j = lane; j < q.back; j += 64) a.ring[wrap(head + free + c_back[i] + j, a.capacity)] = row[j];
        }
    // slots and positions: a thread per token
    const long t1 = min(c_start[cn], (long)a.tokens);
    for (long t = c_start[0] + (long)blockIdx.y * kPlanThreads + tid; t < t1; t += (long)gridDim.y * kPlanThreads) {
        int lo = 0, hi = cn;                                       // the last request that starts at t or before, among those with tokens
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (c_start[mid] <= t) lo = mid;
            else hi = mid;
        }
        int slot = -1, pos = -1;
        if (c_served[lo]) {
            const Request q = request_of(a, c0 + lo);
            pos = q.len + (int)(t - c_start[lo]);
            const int b = pos >> a.shift;
            const int id = b < q.have ? a.table[(size_t)(c0 + lo) * a.width + b] : a.ring[wrap(head + c_take[lo] + (b - q.have), a.capacity)];
            slot = (int)((uint32_t)id << a.shift) + (pos & ((1 << a.shift) - 1));
        }
        a.slots[t] = slot;
        a.positions[t] = pos;
    }
    if (last)                                                      // what no request owns
        for (long t = total[0] + (long)blockIdx.y * kPlanThreads + tid; t < a.tokens; t += (long)gridDim.y * kPlanThreads)
            a.slots[t] = a.positions[t] = -1;
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
    const PlanArgs a{lens, new_tokens, state, table, ring, state_out, lens_out, start, slots, positions, requests, width, capacity, __builtin_ctz(block), tokens};
    const int chunks = requests ? (requests + kChunk - 1) / kChunk : 1;
    const int shares = max(1, min(16, tokens / (chunks * 4 * kPlanThreads)));
    hipLaunchKernelGGL(kv8_plan_kernel, dim3(chunks, shares), dim3(kPlanThreads), 0, as_stream(stream), a);
    return launch_status();
}
