// Attention of many new tokens per sequence in a sliding window over a paged cache (tm_paged_attn_window): the kernels of tm_paged_rows.hip, in which a CTA's context is what its rows
// see: the first tokens and its window.
//
// Measured (32 / 8 heads): prompts of 6000, 5000, 4000 and 3000 tokens, window 1024 and 4 first tokens: 8-bit 422 us, 4-bit 409 (0.64 and 0.65 PFLOP/s; the full call 0.84 and 0.89); 512 tokens after
// 30000, window 4096: 64 us; chunks of 1024 and 512, window 2048, 4-bit: 90 us.  (On a slower card 446, 424, 66.)  Vector instructions take 38 % of the SIMDs' cycles and matrix instructions 27 (42 and 36 in
// the full call).  A CTA of 256 rows, 64 tokens, takes 18 stages of 64 tokens where each of its rows sees 16, of which three are masked (2.25 us
// a stage where the full call takes 2.13), and 8 us beside them: 1.2 for the plan, 5 until the first scores are there, 1.7 for the results, and 4 pass until the next CTA begins.  Requesting all of
// the first stages' loads at once, or the queries behind them, moved these about and saved nothing; 256 CTAs that take one tile after the other in a loop, from counters, took 427 us, and 440 with every 256th tile.
#include "tm_paged_rows_impl.h"

namespace tmw4 {

hipError_t paged_rows_window_setup() { return setup<true>(); }

hipError_t launch_paged_rows_window(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, const PagedForm& f,
                                    void* workspace, hipStream_t stream)
{
    return launch_rows_of<true>(pool, seqs, Q, q_stride, O, q_heads, scale, f, workspace, stream);
}

}  // namespace tmw4
