// Attention of few new tokens per sequence in a sliding window over a paged cache (tm_paged_attn_window): the kernel of tm_paged_attn.hip, in which a sequence's work is what its new tokens
// see: the first tokens, and from the first new token's window on.
#include "tm_paged_columns_launch.h"

namespace tmw4 {

hipError_t launch_paged_columns_window(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, int columns,
                                int most_rows, int grid, bool alone, void* workspace, hipStream_t stream)
{
    return launch_columns<true>(pool, seqs, Q, q_stride, O, q_heads, scale, columns, most_rows, grid, alone, workspace, stream);
}

}  // namespace tmw4
