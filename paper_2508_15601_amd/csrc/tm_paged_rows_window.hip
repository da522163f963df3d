// Attention of many new tokens per sequence in a sliding window over a paged cache (tm_paged_attn_window): the kernels of tm_paged_rows.hip, in which a CTA's context is what its rows
// see: the first tokens and its window.
#include "tm_paged_rows_impl.h"

namespace tmw4 {

hipError_t paged_rows_window_setup() { return setup<true>(); }

hipError_t launch_paged_rows_window(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, const PagedForm& f,
                                    void* workspace, hipStream_t stream)
{
    return launch_rows_of<true>(pool, seqs, Q, q_stride, O, q_heads, scale, f, workspace, stream);
}

}  // namespace tmw4
