// Reading keys and values back from the pages of a quantised cache (tm_paged_read): a run of 32 tokens of one KV head a CTA, numbered as for writing (tm_paged_append_impl.h).
//
// Bound by memory: 2 x 30000 tokens, 8 heads, 8-bit: 58 us, 279 MB at 4.8 TB/s.
#include "tm_attn_device.h"
#include "tm_paged_host.h"

namespace tmw4 {

namespace {

// Reading back: 256 threads turn a run's 4 KiB (2 KiB) of key codes and as many of value codes into fp16 rows in LDS, [32 tokens][128] with rows 16 bytes apart
// in the banks, and write whole 256-byte rows.  x = (q - z) * s: the product is exact in fp32 (8 + 11 bits), so there is one rounding.
constexpr int kReadRow = kHeadDim + 8;   // fp16 values of an LDS row

template <int BITS>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedPool pool, PagedSeqs seqs, uint16_t* __restrict__ K, uint16_t* __restrict__ V)
{
    __shared__ __align__(16) uint16_t rows[2][kRun * kReadRow];
    const int tid = threadIdx.x, lane = tid & 63, h = (int)(blockIdx.x % (unsigned)pool.heads);
    const RunJob job = run_job(pool, seqs, blockIdx.x / (unsigned)pool.heads, lane);
    if (!job.live) return;
    if (job.page >= 0) {
        const size_t run = paged_run(pool, job.page, h, job.run);
        const uint32_t* const words = pool.pairs + run * kRun * 2;
        auto value = [](float q, uint32_t pair) {
            const f16x2 p = as_f16x2(pair);
            return f32_to_f16_bits((q - (float)p.y) * (float)p.x);
        };
        if constexpr (BITS == 8) {
            const u32x4 kc = reinterpret_cast<const u32x4*>(pool.k + run * 4096)[tid], vc = reinterpret_cast<const u32x4*>(pool.v + run * 4096)[tid];
            const int c = tid & 15, hh = (tid >> 4) & 3, hi = tid >> 6;
            const int u = 16 * (hi >> 1) + c, d = 32 * hh + 16 * (hi & 1);
            const uint32_t kp = words[2 * u];
            u32x4 out[2];
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                const uint32_t two = kc[n >> 1] >> (16 * (n & 1));
                out[n >> 2][n & 3] = value((float)(two & 255u), kp) | ((uint32_t)value((float)(two >> 8 & 255u), kp) << 16);
            }
            *reinterpret_cast<u32x4*>(&rows[0][u * kReadRow + d]) = out[0];
            *reinterpret_cast<u32x4*>(&rows[0][u * kReadRow + d + 8]) = out[1];
#pragma unroll
            for (int n = 0; n < 16; ++n) {
                const int il = n >> 3, e = n & 7, t = (e & 3) + 4 * hh + 16 * (e >> 2);
                rows[1][t * kReadRow + 16 * (2 * hi + il) + c] = value((float)(vc[n >> 2] >> (8 * (n & 3)) & 255u), words[2 * t + 1]);
            }
        } else if (tid < 128) {
            const u32x4 kc = reinterpret_cast<const u32x4*>(pool.k + run * 2048)[tid];
            const int c = tid & 15, hh = (tid >> 4) & 3, u = 16 * (tid >> 6) + c;
            const uint32_t kp = words[2 * u];
#pragma unroll
            for (int tt = 0; tt < 4; ++tt) {
                u32x4 out;
#pragma unroll
                for (int n = 0; n < 4; ++n)                            // elements 2n and 2n + 1 sit at nibbles n and n + 4
                    out[n] = value((float)(kc[tt] >> (4 * n) & 15u), kp) | ((uint32_t)value((float)(kc[tt] >> (4 * n + 16) & 15u), kp) << 16);
                *reinterpret_cast<u32x4*>(&rows[0][u * kReadRow + 32 * hh + 8 * tt]) = out;
            }
        } else {
            const int id = tid - 128, c = id & 15, hh = (id >> 4) & 3, ii = id >> 6;
            const u32x4 vc = reinterpret_cast<const u32x4*>(pool.v + run * 2048)[id];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int t = (e & 3) + 4 * hh + 16 * (e >> 2), sh = 4 * ((e >> 1) + 4 * (e & 1));
                const uint32_t vp = words[2 * t + 1];
#pragma unroll
                for (int w = 0; w < 4; ++w) rows[1][t * kReadRow + 16 * (4 * ii + w) + c] = value((float)(vc[w] >> sh & 15u), vp);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int which = it >> 1, u = (tid >> 4) + 16 * (it & 1), d = 8 * (tid & 15);
        if (u < job.u0 || u >= job.u1) continue;
        u32x4 w = {0u, 0u, 0u, 0u};                                    // a page that the pool does not have reads as zeros
        if (job.page >= 0) w = *reinterpret_cast<const u32x4*>(&rows[which][u * kReadRow + d]);
        *reinterpret_cast<u32x4*>((which ? V : K) + ((size_t)(job.row + u) * pool.heads + h) * kHeadDim + d) = w;
    }
}

}  // namespace

hipError_t launch_paged_read(const PagedPool& pool, const PagedSeqs& seqs, uint16_t* K, uint16_t* V, hipStream_t stream)
{
    const long blocks = most_runs(seqs) * pool.heads;
    if (blocks <= 0 || blocks > most_ctas(256)) return hipErrorInvalidConfiguration;
    const auto kernel = pool.bits == 8 ? paged_read_kernel<8> : paged_read_kernel<4>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, stream, pool, seqs, K, V);
    return hipGetLastError();
}

}  // namespace tmw4
