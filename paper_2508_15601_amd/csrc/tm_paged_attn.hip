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
#include "tm_paged_columns_launch.h"

namespace tmw4 {

hipError_t launch_paged_columns(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, int columns,
                                int most_rows, int grid, bool alone, void* workspace, hipStream_t stream)
{
    return launch_columns<false>(pool, seqs, Q, q_stride, O, q_heads, scale, columns, most_rows, grid, alone, workspace, stream);
}

}  // namespace tmw4
