// Attention of few new tokens per sequence in a sliding window over a paged cache (tm_paged_attn_window): the kernel of tm_paged_attn.hip, in which a sequence's work is what its new tokens
// see: the first tokens, and from the first new token's window on.  A column's tokens are then two ranges; a block that holds some of either takes both tests in the one pass (a loop over
// the two ranges made the compiler keep every converted code in front of it: 64 at 20000 with 4-bit codes 58 us, like this 52).
//
// Measured (32 / 8 heads), in brackets a full call whose contexts are as long as the window: 64 sequences at 20000, window 4096 and 4 first tokens, 8-bit 89 us (86; 6.1 TB/s), 4-bit 52 us
// (51; 5.5 TB/s); 256 at 10000, 512 and 4, 55 (48) and 40 us (32); 16 x 5 drafted tokens after 8000, 2048 and 4, 8-bit 22 us (20); one at 30000, 1024: 8.9 us (8.8).  What is more than in the
// full call is the block at the window's start that is seen in part, and the block of the first tokens: two of seventeen 4-bit blocks are 12 %, where issue bounds it.
#include "tm_paged_columns_launch.h"

namespace tmw4 {

hipError_t launch_paged_columns_window(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, int columns,
                                int most_rows, int grid, bool alone, void* workspace, hipStream_t stream)
{
    return launch_columns<true>(pool, seqs, Q, q_stride, O, q_heads, scale, columns, most_rows, grid, alone, workspace, stream);
}

}  // namespace tmw4
