// Norms of queries and keys head by head with their rotation in the same pass (tm_heads_apply).
//
// Bound by memory where tokens are many: 8192 tokens of 32 / 8 heads of 128, nothing in the caches: 34.5 us, 168 MB at 4.9 TB/s (a large copy reaches 5.2; without norms 33.6 us); the arithmetic, 240 vector
// instructions for a lane's sixteen values, each of which takes its four cycles in 64 bits as in 32, and a wave's chain of load, sums over lanes, root and store bound the middle (1024 tokens 7.1 us, 21 MB), a
// launch the small (16 tokens 3.5 us).  Waiting for the stores of a round before the next one cost 3 % (3000 tokens: 13.6 us, so 13.0; 12.2 with what else was saved since).  Weights multiplied into the sines
// and cosines once a token, which saves a third of the arithmetic, took registers and with them waves: 38 us.  Keeping the cosines in registers 35.1, but 8.6 for 1024.  Five waves a SIMD forced: 35.6.
#include "tm_heads_device.h"
#include "tm_paged_host.h"

#include <algorithm>

namespace tmw4 {

namespace {

// A wave takes `rounds` times 64 / LANES heads of one token, queries first; LANES lanes hold a head, sixteen dimensions each.  Weights that all
// heads of a side share stay in registers.  X and Y of a side may be the same.
template <int LANES, int MODE, bool INTERLEAVED>
__global__ __launch_bounds__(256) void heads_kernel(HeadRows q, HeadRows k, const int32_t* __restrict__ positions, RopePlan r, int tokens, int dim, int rounds)
{
    constexpr int AT_ONCE = 64 / LANES;
    __shared__ CosSin cs[4][turns_of(8 * LANES)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), u = lane & (LANES - 1), slot = lane / LANES;
    const int q_rounds = (q.heads + AT_ONCE - 1) / AT_ONCE, all = q_rounds + (k.heads + AT_ONCE - 1) / AT_ONCE;
    const uint32_t parts = (uint32_t)(all + rounds - 1) / (uint32_t)rounds, job = blockIdx.x * 4 + wave;       // (a launch has fewer than 2^32 threads)
    const long token = job / parts;
    if (token >= tokens) return;
    const int first = (int)(job % parts) * rounds, last = min(first + rounds, all);
    const HeadPart<LANES, INTERLEAVED> part(u, dim, r);
    f16x8 a, b, wa, wb;
    Sixteen weights;
    auto request = [&](int round) {
        const bool keys = round >= q_rounds;
        const HeadRows& s = keys ? k : q;
        const int h = (round - (keys ? q_rounds : 0)) * AT_ONCE + slot, there = min(h, s.heads - 1);
        if (MODE != kNoNorm && (s.norm.stride || round == first || round == q_rounds)) wa = head_weights(s.norm, there, part.d0), wb = head_weights(s.norm, there, part.d1);
        const __amdgpu_buffer_rsrc_t x = make_rsrc(s.x + token * s.x_stride, (uint32_t)s.heads * (uint32_t)dim * 2u);
        a = load8(x, h * dim + part.d0);
        b = load8(x, h * dim + part.d1);
    };
    request(first);
    if (r.rot) {
        rope_angles_of<true>(cs[wave], r, positions + token * r.axes, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    wait_for_loads();                                        // (they were requested before the positions)
    for (int round = first; round < last; ++round) {
        const bool keys = round >= q_rounds;
        const HeadRows& s = keys ? k : q;
        f16x8 y0, y1;
        Sixteen from;
        if constexpr (MODE == kNoNorm) {
            y0 = a, y1 = b;
            if (round + 1 < last) request(round + 1);
            from.of(y0, y1);
        } else {
            from.of(a, b);
            if (s.norm.stride || round == first || round == q_rounds) weights.of(wa, wb);
            if (round + 1 < last) request(round + 1);
        }
        const int h = (round - (keys ? q_rounds : 0)) * AT_ONCE + slot;
        head_turn<LANES, MODE, INTERLEAVED>(y0, y1, from, weights, part, s.norm, cs[wave]);
        // no branch: heads that there are not lie behind the buffer's end, and what lies there is not stored
        const __amdgpu_buffer_rsrc_t y = make_rsrc(s.y + token * s.y_stride, (uint32_t)s.heads * (uint32_t)dim * 2u);
        store8(y, y0, part.any ? h * dim + part.d0 : kBehind);
        store8(y, y1, part.whole ? h * dim + part.d1 : kBehind);
    }
}

template <int LANES>
auto pick(int mode, bool interleaved)
{
    if (mode == kNoNorm) return interleaved ? heads_kernel<LANES, kNoNorm, true> : heads_kernel<LANES, kNoNorm, false>;
    if (mode == kPlainNorm) return interleaved ? heads_kernel<LANES, kPlainNorm, true> : heads_kernel<LANES, kPlainNorm, false>;
    return interleaved ? heads_kernel<LANES, kAnyNorm, true> : heads_kernel<LANES, kAnyNorm, false>;
}

}  // namespace

hipError_t launch_heads(const HeadRows& q, const HeadRows& k, const int32_t* positions, const RopePlan& r, int tokens, int dim, int num_cu, hipStream_t stream)
{
    const int lanes = dim <= 16 ? 1 : dim <= 32 ? 2 : dim <= 64 ? 4 : dim <= 128 ? 8 : 16, at_once = 64 / lanes;
    const int all = (q.heads + at_once - 1) / at_once + (k.heads + at_once - 1) / at_once;
    // Rounds a wave takes, which work out the token's angles once but follow one another: by the waves a compute unit would have of one each.  Measured with 1, 2, 3 and 5 (us; heads of 128): 32 / 8 heads, 5 rounds a token: 512 tokens 4.8, 5.3, 5.3,
    // 6.7; 1024 7.1, 7.2, 7.2, 7.7; 1500 9.9, 9.6, 8.8, 9.6; 2048 11.8, 11.1, 10.2, 10.1; 3000 15.4, 14.6, 13.3, 12.2; 8192 41.8, 36.3, 34.2, 34.6.  64 / 4 heads, 9 rounds: 1024 10.7, 9.6, 9.1,
    // 9.6, 2048 18.2, 15.9, 14.4, 13.8, and 15.4 with all nine.
    const long total = (long)tokens * all, least_parts = total < 24L * num_cu ? all : total < 48L * num_cu ? (all + 2) / 3 : (all + 4) / 5;
    const int rounds = (int)((all + least_parts - 1) / least_parts);
    const long parts = (all + rounds - 1) / rounds, most = 4 * most_ctas(256) / parts;       // tokens of a launch
    const auto of = lanes == 1 ? pick<1> : lanes == 2 ? pick<2> : lanes == 4 ? pick<4> : lanes == 8 ? pick<8> : pick<16>;
    const auto kernel = of(!q.norm.on && !k.norm.on ? kNoNorm : !q.norm.centred && !k.norm.centred ? kPlainNorm : kAnyNorm, r.interleaved || r.rot == 0);
    for (long t = 0; t < tokens; t += most) {
        const int n = (int)std::min(most, tokens - t);
        auto from = [&](HeadRows s) {
            s.x += t * s.x_stride;
            s.y += t * s.y_stride;
            return s;
        };
        hipLaunchKernelGGL(kernel, dim3((unsigned)((n * parts + 3) / 4)), dim3(256), 0, stream, from(q), from(k), positions ? positions + t * r.axes : nullptr, r, n, dim, rounds);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tmw4
