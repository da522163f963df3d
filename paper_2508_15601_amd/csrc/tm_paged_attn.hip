// Attention of few new tokens per sequence over a paged cache: decoding steps and the verification of drafted tokens (tm_paged_attn; many tokens per sequence run
// on tm_paged_rows.hip).
//
// Arithmetic and loading pipeline are those of decode attention over the contiguous cache (tm_attn.hip): a wave multiplies blocks of 4 KiB of key codes and as many of value
// codes with sixteen (or eight) query columns, two blocks ahead in flight, four waves take blocks in turn and meet in LDS.  New here:
//   - Columns are (token, query head) pairs of a sequence and KV head, numbered token by token, each with its own causal length.
//   - The work of the call - (sequence, KV head, column tile) segments of `quads` of four blocks, the length known on the device only - is laid out in one row and cut into
//     equal pieces, one per CTA.  A CTA works through the end of one segment, whole ones, and the beginning of another, so a call takes as long as its work
//     and not as long as its longest sequence; a server's contexts differ by factors of ten.  Beginning a segment costs as much as kSegmentStart quads, which counts as work.  Where
//     segments are few, pieces are cut so that every segment begins with a CTA, if that lengthens them by less than it saves.
//   - ALONE: the same with a wave in place of a CTA, for many segments: a wave takes every block of its segment, and nothing waits for another wave.
//   - A segment that several CTAs share is put together by the one that arrives last, in the order of the pieces, so results do not depend on who that is; above sixteen pieces in
//     two levels, groups of sixteen first, which keeps the chain of loads short without another launch.
//   - A block is one run of 32 tokens (8-bit codes) or two (4-bit); every run has its own address, from a page number that is requested three blocks ahead.  A run on a
//     page that the pool does not have is not read and its tokens are masked.
//
// Measured (32 / 8 heads unless said): 32 sequences of 4096 to 8192 tokens, 8-bit 71 us (5.9 TB/s), 4-bit 45 us (4.7 TB/s); 4 of 60000 down to 30000, 64 / 8 heads, 8-bit 63 us (6.0 TB/s); 64
// skewed ones up to 16384, 4-bit 56 us (5.2 TB/s); one of 2048, 8-bit 8.8 us; 12 x 5 drafted tokens after 3000 to 6000, 40 / 8 heads, 8-bit 34 us (3.4 TB/s), 4-bit 27; 32 x 5 after 4000 to
// 8000, 32 / 8 heads, 91 and 68.  Long contexts are bound by memory (a large copy reaches 5.2 TB/s, both ways together); short ones by a launch, a plan, a chain of three round trips to memory (lengths, page numbers, blocks) and the
// meeting of the pieces, 8 us together; tiles of 32 columns by instruction issue, the codes being converted for each half.
#include "tm_paged_columns_impl.h"

namespace tmw4 {

namespace {

template <int BITS, bool PACK, int PARTS, int TILES, bool ALONE>
__global__ __launch_bounds__(256 * TILES) __attribute__((amdgpu_waves_per_eu(BITS == 4 && PACK ? 1 : 2, 2))) void paged_columns_kernel(
    PagedPool pool, PagedSeqs seqs, const uint16_t* __restrict__ Q, long q_stride, uint16_t* __restrict__ O, int q_heads, float scale_log2e, int most_rows,
    float* __restrict__ partial, uint32_t* __restrict__ counters)
{
    paged_columns<BITS, PACK, PARTS, TILES, ALONE, 4 * TILES>(pool, seqs, Q, q_stride, O, q_heads, scale_log2e, most_rows, partial, counters, blockIdx.x, gridDim.x);
}

}  // namespace

hipError_t launch_paged_columns(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, int columns,
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
        if (alone) return columns == 8 ? paged_columns_kernel<BITS, true, PARTS, 1, true> : paged_columns_kernel<BITS, false, PARTS, 1, true>;
        return columns == 8    ? paged_columns_kernel<BITS, true, PARTS, 1, false>
               : columns == 16 ? paged_columns_kernel<BITS, false, PARTS, 1, false>
                               : paged_columns_kernel<BITS, false, PARTS, 2, false>;
    };
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 2> Two;
    const auto kernel = pool.bits == 8 ? pick(std::integral_constant<int, 8>{}, One{})
                        : pool.run_log == 0 ? pick(std::integral_constant<int, 4>{}, Two{}) : pick(std::integral_constant<int, 4>{}, One{});
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(columns == 32 ? 512 : 256), 0, stream, pool, seqs, Q, q_stride, O, q_heads, s, most_rows, partial, counters);
    return hipGetLastError();
}

}  // namespace tmw4
