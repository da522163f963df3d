// Rotary positions of packed tokens (tm_rope_apply).
//
// Bound by memory: 8192 tokens, 32 heads of 128, 64 of them turned: 29.5 us with nothing in the caches, 134 MB at 4.6 TB/s (22 us from the last-level cache); 16 tokens 4 us, an
// empty launch and two round trips.  Requesting two or four rounds of a wave's vectors ahead changed nothing.
#include "tm_rope_device.h"
#include "tm_paged_host.h"

#include <algorithm>

namespace tmw4 {

namespace {

// A wave takes `per_wave` heads of one token: it works out the token's sines and cosines once (a lane a pair) and reads them back from LDS for every head.  X and Y may be the same.
__global__ __launch_bounds__(256) void rope_kernel(const uint16_t* X, long x_stride, const int32_t* __restrict__ positions, RopePlan r,
                                                   uint16_t* Y, long y_stride, int tokens, int heads, int dim, int per_wave)
{
    __shared__ CosSin cs[4][kRopeMaxPairs];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int parts = (heads + per_wave - 1) / per_wave;
    const long job = (long)blockIdx.x * 4 + wave;
    const long token = job / parts;
    const int h0 = (int)(job - token * parts) * per_wave;
    if (token < tokens) rope_angles(cs[wave], r, positions[token], lane);
    __syncthreads();
    if (token >= tokens) return;
    rope_heads(X + token * x_stride, Y + token * y_stride, h0, min(h0 + per_wave, heads), dim, r, cs[wave], lane);
}

}  // namespace

hipError_t launch_rope(const uint16_t* X, long x_stride, const int32_t* positions, const RopePlan& r, uint16_t* Y, long y_stride, int tokens, int heads,
                       int dim, hipStream_t stream)
{
    // one round of a wave's lanes at a time where tokens are few
    const int round = 64 / ((dim + 15) / 16);
    const int per_wave = (long)tokens * heads >= 16384L * round ? heads : round;
    const long parts = (heads + per_wave - 1) / per_wave, most = 4 * most_ctas(256) / parts;       // tokens of a launch
    for (long t = 0; t < tokens; t += most) {
        const int n = (int)std::min(most, tokens - t);
        hipLaunchKernelGGL(rope_kernel, dim3((unsigned)((n * parts + 3) / 4)), dim3(256), 0, stream, X + t * x_stride, x_stride, positions + t, r, Y + t * y_stride, y_stride, n, heads,
                           dim, per_wave);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tmw4
