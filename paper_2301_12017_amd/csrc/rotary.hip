// Heads of features turned by their tokens' positions (rotary.hpp).
//
//   a' = m (a cos(p f) - b sin(p f)),  b' = m (b cos(p f) + a sin(p f))    for each pair (a, b) of features, p the position, f the pair's frequency
//
// Features behind the turned part are copied.
//
// Memory bounds it: 8191 tokens of 32 heads of 128, 26.4 us = 5.1 TB/s read and written, what a copy of them takes (halves of a head as pairs: 28).
// Few tokens are a launch and the latency of their loads: 16 of 12 heads of 64 3.1 us.
#include "rotary.hpp"

namespace w4a4 {
namespace {

template <bool BF16, int WAY, int B>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryWork a) {
    const long t0 = (long)blockIdx.x * a.share;
    rotary_tokens<BF16, WAY, B>(a, t0, (int)min((long)a.share, a.tokens - t0));
}

template <bool BF16, int B>
void launch(const RotaryWork &a, hipStream_t st) {
    const dim3 grid((unsigned)(((long)a.tokens + a.share - 1) / a.share));
    auto run = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a); };
    switch (a.way) {
        case kRotaryNeighbours: return run(rotary_kernel<BF16, kRotaryNeighbours, B>);
        case kRotaryHalves8: return run(rotary_kernel<BF16, kRotaryHalves8, B>);
        case kRotaryHalves4: return run(rotary_kernel<BF16, kRotaryHalves4, B>);
        default: return run(rotary_kernel<BF16, kRotarySingle, B>);
    }
}

}  // namespace

int rotary_launch(const RotaryWork &a, int dtype, int heads, hipStream_t st) {
    if (dtype == W4A4_BF16) heads == 1 ? launch<true, 1>(a, st) : launch<true, 4>(a, st);
    else heads == 1 ? launch<false, 1>(a, st) : launch<false, 4>(a, st);
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
    // Four heads of a thread share its angles, where there are tokens enough for all CUs.  us by one | four: 16 tokens of 12 heads of 64 3.1 | 3.5, 400 of 32 of 128 4.2 | 4.3,
    // 600 5.0 | 4.5, 8191 33 | 28.
    const int at_once = (long)tokens * heads * features < 256L * 256 * 8 * 4 ? 1 : 4;
    const RotaryWork work = rotary_work(X, tokens, heads, features, ldx, positions, rotary_args(R), out, ldo, at_once);
    if (!grid_fits(((long)tokens + work.share - 1) / work.share, 256)) return W4A4_ERR_UNSUPPORTED_SHAPE;
    return rotary_launch(work, dtype, at_once, as_stream(stream));
}
