// The kernel of few rows per sequence over pages and its launch; tm_paged_attn.hip and tm_paged_window.hip build it.
#pragma once
#include "tm_paged_columns_impl.h"

namespace tmw4 {

namespace {

template <int BITS, bool PACK, int PARTS, int TILES, bool ALONE, bool WINDOW>
__global__ __launch_bounds__(256 * TILES) __attribute__((amdgpu_waves_per_eu(BITS == 4 && PACK ? 1 : 2, 2))) void paged_columns_kernel(
    PagedPool pool, PagedSeqs seqs, const uint16_t* __restrict__ Q, long q_stride, uint16_t* __restrict__ O, int q_heads, float scale_log2e, int most_rows,
    float* __restrict__ partial, uint32_t* __restrict__ counters)
{
    paged_columns<BITS, PACK, PARTS, TILES, ALONE, 4 * TILES, WINDOW>(pool, seqs, Q, q_stride, O, q_heads, scale_log2e, most_rows, partial, counters, blockIdx.x, gridDim.x);
}

template <bool WINDOW>
hipError_t launch_columns(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, int columns,
                          int most_rows, int grid, bool alone, void* workspace, hipStream_t stream)
{
    static_assert(3 * kPagedMostWaves * sizeof(uint32_t) <= kPagedLengthAt && 3 * kPagedMostCtas <= 3 * kPagedMostWaves, "three counters a wave or CTA");
    static_assert(2 * kPagedMostCtas * (2 * 32 + 2 * 2048) * sizeof(float) <= kPagedColumnBytes, "two slots a CTA");
    static_assert(2 * kPagedMostWaves * (2 * 16 + 2048) * sizeof(float) <= kPagedColumnBytes, "two slots a wave");
    if (grid < 1 || grid > (alone ? kPagedMostWaves / 4 : kPagedMostCtas) || (alone && columns == 32)) return hipErrorInvalidValue;
    uint32_t* const counters = (uint32_t*)workspace;
    float* const partial = (float*)((char*)workspace + kPagedCounterBytes);
    const float s = scale * 1.4426950408889634f;
    auto pick = [&](auto bits, auto parts) {
        constexpr int BITS = decltype(bits)::value, PARTS = decltype(parts)::value;
        if (alone) return columns == 8 ? paged_columns_kernel<BITS, true, PARTS, 1, true, WINDOW> : paged_columns_kernel<BITS, false, PARTS, 1, true, WINDOW>;
        return columns == 8    ? paged_columns_kernel<BITS, true, PARTS, 1, false, WINDOW>
               : columns == 16 ? paged_columns_kernel<BITS, false, PARTS, 1, false, WINDOW>
                               : paged_columns_kernel<BITS, false, PARTS, 2, false, WINDOW>;
    };
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 2> Two;
    const auto kernel = pool.bits == 8 ? pick(std::integral_constant<int, 8>{}, One{})
                        : pool.run_log == 0 ? pick(std::integral_constant<int, 4>{}, Two{}) : pick(std::integral_constant<int, 4>{}, One{});
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(columns == 32 ? 512 : 256), 0, stream, pool, seqs, Q, q_stride, O, q_heads, s, most_rows, partial, counters);
    return hipGetLastError();
}

}  // namespace

}  // namespace tmw4
