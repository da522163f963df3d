// Norms of queries and keys head by head with their rotation in the same pass (tm_heads_apply).
#include "tm_heads_device.h"
#include "tm_paged_host.h"

#include <algorithm>

namespace tmw4 {

namespace {

// Heads 0 .. q.heads - 1 are queries, those behind them keys.  A wave takes `rounds` times 64 / LANES heads of one token; LANES lanes hold a head, sixteen dimensions each.  A lane's dimensions
// are the same in every round, so the cosines and sines of its pairs stay in registers.  X and Y of a side may be the same.
template <int LANES>
__global__ __launch_bounds__(256) void heads_kernel(HeadRows q, HeadRows k, const int32_t* __restrict__ positions, RopePlan r, int tokens, int dim, int rounds)
{
    constexpr int AT_ONCE = 64 / LANES;
    __shared__ CosSin cs[4][kRopeMaxPairs];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), u = lane & (LANES - 1);
    const int heads = q.heads + k.heads, parts = (heads + AT_ONCE * rounds - 1) / (AT_ONCE * rounds);
    const long job = (long)blockIdx.x * 4 + wave;
    const long token = job / parts;
    if (token >= tokens) return;
    const int h0 = (int)(job - token * parts) * AT_ONCE * rounds, h1 = min(h0 + AT_ONCE * rounds, heads);
    const HeadPart part(u, dim, r);
    f16x8 a, b, wa, wb;
    auto side = [&](int h) -> const HeadRows& { return h < q.heads ? q : k; };
    auto request = [&](int h) {
        h = min(h, heads - 1);                               // (a head that exists)
        const HeadRows& s = side(h);
        if (h >= q.heads) h -= q.heads;
        const uint16_t* const x = s.x + token * s.x_stride + (long)h * dim;
        a = *(const f16x8*)(x + part.d0);
        b = *(const f16x8*)(x + part.d1);
        wa = head_weights(s.norm, h, part.d0);
        wb = head_weights(s.norm, h, part.d1);
    };
    request(h0 + lane / LANES);
    CosSin c[8] = {};
    if (r.rot) {
        rope_angles_of(cs[wave], r, positions + token * r.axes, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (part.turned) {
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = cs[wave][8 * u + i];
        }
    }
    for (int h = h0 + lane / LANES; h < h1 + lane / LANES; h += AT_ONCE) {       // (the same number of rounds in every lane)
        f16x8 y0 = a, y1 = b;
        const f16x8 w0 = wa, w1 = wb;
        if (h + AT_ONCE < h1 + lane / LANES) request(h + AT_ONCE);
        const HeadRows& s = side(min(h, heads - 1));
        head_turn<LANES>(y0, y1, w0, w1, part, s.norm, dim, r, c);
        if (h >= h1 || !part.any) continue;
        uint16_t* const y = s.y + token * s.y_stride + (long)(h < q.heads ? h : h - q.heads) * dim;
        *(f16x8*)(y + part.d0) = y0;
        if (part.whole) *(f16x8*)(y + part.d1) = y1;
    }
}

}  // namespace

hipError_t launch_heads(const HeadRows& q, const HeadRows& k, const int32_t* positions, const RopePlan& r, int tokens, int dim, hipStream_t stream)
{
    const int lanes = dim <= 16 ? 1 : dim <= 32 ? 2 : dim <= 64 ? 4 : dim <= 128 ? 8 : 16, at_once = 64 / lanes, heads = q.heads + k.heads;
    // one round of a wave's lanes at a time where tokens are few
    const int all = (heads + at_once - 1) / at_once, rounds = (long)tokens * all >= 16384L ? all : 1;
    const long parts = (heads + at_once * rounds - 1) / (at_once * rounds), most = 4 * most_ctas(256) / parts;       // tokens of a launch
    const auto kernel = lanes == 1 ? heads_kernel<1> : lanes == 2 ? heads_kernel<2> : lanes == 4 ? heads_kernel<4> : lanes == 8 ? heads_kernel<8> : heads_kernel<16>;
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
