// Attention of many new tokens per sequence over a paged cache: prompts, chunks of prompts, long drafts (tm_paged_attn).
//
// The kernel is that of prompt attention over the contiguous cache (tm_attn_prefill.hip, tm_attn_rows_impl.h): CTAs of 128 or 256 (token, query head) rows of a KV head,
// codes converted once per CTA.  New here:
//   - Row tiles are numbered over the sequences on the device (tm_paged_device.h), so sequences of any mix of lengths share a launch without a grid for the
//     longest of them.
//   - Where row tiles are too few to fill the chip (a short chunk after a long past), or few of them would outlast the others, contexts are cut into pieces, each a CTA.  How long
//     the pieces are every CTA works out by itself from the sequences' lengths (piece_stages), which the host does not know.  A second kernel puts a row's pieces together in
//     their order, so results do not depend on which is done first.
//
// Measured (32 / 8 heads): prompts of 6000, 5000, 4000 and 3000 tokens, 8-bit: 837 us (0.84 PFLOP/s), 4-bit 797 (0.89); 512 tokens after 30000, 4-bit: 283 us (0.90 PFLOP/s), 1024 without
// pieces; 100 after 8000, 8-bit: 40.5 us, 259 without pieces; one prompt of 4000: 162.  (Calls in a row; after an idle time, until the clock is up, a sixth more.  Cards differ: on another 903, 857, 296, 40.7
// and 172.)  What bounds it is the issue of vector and matrix instructions (tm_attn_prefill.hip).  How page numbers are loaded counts: as vector loads, which made every stage wait for all of its wave's
// loads, 863, 830, 296 and 42.3 in the same run; as scalar loads that every stage's first product waited for 846, 820, 287 and 41.1.  A piece of 256 rows leaves 133 KB in memory.
#include "tm_paged_rows_impl.h"

namespace tmw4 {

hipError_t paged_rows_setup()
{
    const hipError_t e = setup<false>();
    return e == hipSuccess ? paged_rows_window_setup() : e;
}

// Up to 64 rows (tokens times query heads of a KV head) a sequence, everything goes by columns: 12 sequences of 5 tokens and 32 / 8 heads 37 us, by rows 40; with 128 rows and one
// sequence of 8000 tokens it is 38 us against 31.  With more, a sequence of up to 16 rows still does: those of a mixed call are decoding.
// By columns, a CTA to a segment (a sequence's column tile and KV head) at a time, or each of its waves to one of its own, which saves their meeting and lets one wave's start hide
// behind the others' work, but leaves more pieces to merge.  Waves win where segments are many: 8 KV heads, 4-bit, 256 sequences of 300 / 1000 tokens 23.5 / 51 us (a CTA each 52 /
// 77), 64 skewed ones up to 16384 52 (64), 64 of 5 drafted tokens after 500 16 (21), 33 of 300 10.5 (14.4); with a segment per compute unit or less they lose: 32 of 8192 54 (47).
// 8-bit codes take the memory's time sooner: 256 of 300 / 1000 31 / 86 (48 / 98), 128 of 1000 43 (50), but 64 of 1000 26.9 (25.0), 256 skewed ones up to 9000 212 (200), 64 skewed 97 (87),
// 256 x 5 after 1000, whose segments need two column tiles, 183 (152): from four segments a compute unit on.  Below that two CTAs a compute unit hide each other's starts if contexts are
// short: 48 of 300 10.2 us (13.0 with one), 64 of 500 14.2 (15.3), 64 of 2000 42.8 (45), but 40 of 2000 to 4000 50 (45).
// Both in one call go in one launch, the columns' CTAs (eight waves) first, on half the compute units, or 11 / 16 where row tiles are few.  With half, 11 / 16 and in two launches (us; 8-bit, then
// 4-bit; contexts from half of the length given; all with page numbers as vector loads; the first with half takes 117 and 103 now): 40 decoding at 4000 and chunks of 1500 and 750 122, 130, 141 and 113, 122, 131; 64 at 4000 and a chunk of 512 at 4000 116, 136, 141 and 113, 108,
// 118; 128 at 1000 and 512 at 2000 86, 93, 104 and 78, 82, 92; 200 at 2000 and a prompt of 256, where the rule takes 11 / 16, 147, 133, 137 and 90, 80, 90.  Short contexts beside tiles of 128 rows
// it does not tell apart, and takes half: 60 at 500 and 400 at 500 23, 30 and 24, 29, but 300 at 300 and a prompt of 64 46, 41, 48 and 37, 31, 43.  Behind the row tiles the columns' long
// pieces stick out: 2 to 8 % more than with half in the first three; on all compute units first 10 to 14 %.
// In a window both parts' work is known, about: a sequence's context is what it sees.  Where row tiles do not fill the chip by themselves the columns take the compute units that their share
// of the work asks for: a compute unit that has nothing but columns reads 50 GB/s of 8-bit codes, 38 of 4-bit ones, and a stage takes 2.3 us (1.5 with 128 rows).  Half of them, and the share
// (us; 8-bit unless said): 24 decoding and chunks of 1024 and 512, window 2048, 4-bit: 116 and 97 with 16 to 64; 8 decoding and 300, 16 / 2 heads: 41 and 33 with 16 to 64; 96 decoding and 200: 107, and
// 100 with 176; 64 decoding and 512, window 4096: 136 with 128, 157 with 96 and 170 with 176.  Where the tiles fill the chip half is as good as any: 40 decoding and 1500 and 750: 87 with 96 to
// 176, 96 with 32.
// 128 or 256 rows a CTA: a stage of 128 costs 0.66 of one of 256 (the four prompts above: 1154 against 867 us).  So 256, unless the chip does not fill with either and pieces cannot
// make up for it, a context being short (two prompts of 307 and 161 tokens, 2 / 1 heads: 19 against 20 us; 400 and 150, 16 / 1: 34 against 39).  Over 57 random calls (one chunk after
// up to 40000 tokens, up to six prompts, up to 30 decoding sequences with chunks; 1 to 8 KV heads, 1 to 16 query heads each) the rule's choice takes 1.02 of the better one's time,
// always 128 rows 1.08, always 256 1.05.
// Pieces: not where the chip is full of tiles (four times over, if a context may be much longer than its new tokens): the second kernel alone is 4 to 8 us.
PagedForm paged_form(const PagedPool& pool, const PagedSeqs& seqs, int q_heads, int max_count, int max_len, int num_cu)
{
    const int G = q_heads / pool.heads;
    PagedForm f{};
    // no more tokens than sequences and no hint: a decoding step, surely (32 at 8192, 8-bit: 84 us, taken for anything 98; 64 at 1000 23 and 38)
    const long most = (long)(max_count > 0 && max_count < seqs.tokens ? max_count : max_count == 0 && seqs.tokens <= seqs.batch ? 1 : seqs.tokens) * G;
    // the tokens that a sequence's new ones see, about, and those that a tile of rows does
    const bool windowed = seqs.window < seqs.cap;
    const int len = max_len > 0 && max_len < seqs.cap ? max_len : seqs.cap;
    const int reach = windowed ? (int)std::min((long)len, (long)seqs.window + seqs.sinks + most / G) : len;
    f.columns = most > 64 ? G <= 8 ? 8 : 16 : most <= 8 ? 8 : most <= 16 ? 16 : 32;
    f.column_rows = most <= 64 ? 64 : seqs.batch > 1 ? 16 : 0;
    // Where the call has tokens for less than half of the table's rows, the others are not in it (10 of 8000 in a table of 256 rows, 8-bit: 39 us with a segment counted for every row, 34 like this).
    const long segments = (2L * seqs.tokens < seqs.batch ? (long)seqs.tokens : (long)seqs.batch) * pool.heads * (most <= 64 ? (most + f.columns - 1) / f.columns : 1);
    const double most_units = ((double)seqs.tokens * G / 8 + seqs.batch) * pool.heads * (seqs.cap / 32 + 3);      // blocks and starts, were every context as long as the table
    f.alone = (pool.bits == 4 ? segments > num_cu : f.columns < 32 && segments >= 4L * num_cu) && most_units < 2147483648.0;      // (counted in 32 bits)
    if (f.alone && f.columns == 32) f.columns = 16;
    const bool twice = pool.bits == 8 && !f.alone && f.columns < 32 && segments > num_cu && (max_len > 0 || windowed) && reach <= 1024;
    f.column_ctas = std::min(twice ? 2 * num_cu : num_cu, f.alone ? kPagedMostWaves / 4 : kPagedMostCtas);
    if (most <= 64) {
        f.column_rows = 1 << 30;                             // whatever the offsets say
        return f;
    }
    f.least_rows = f.column_rows + 1;
    f.together = f.column_rows && most_units < 2147483648.0;
    const int stages = ((windowed ? (int)std::min((long)len, (long)seqs.window + seqs.sinks + 256 / G + 2 * ST) : len) + ST - 1) / ST;
    const long rows = (long)seqs.tokens * G, big = rows / f.least_rows < seqs.batch ? rows / f.least_rows : seqs.batch, equal = (rows + most - 1) / most;
    const int past_none = (int)((most / G + ST - 1) / ST);   // stages of the longest new tokens alone
    double best = 0.0;
    for (int rw = 4; rw <= 8; rw += 4) {
        const double full = (double)(rows / (32 * rw)) * pool.heads, likely = full + 0.5 * equal * pool.heads;
        const bool cut = stages > kLeastStages && (full < num_cu || (full < 4.0 * num_cu && stages > 2 * past_none));
        const double least = cut ? (double)kLeastStages / stages : 1.0, t = (rw == 4 ? 0.66 : 1.0) * std::max(likely / num_cu, least);
        if (rw == 4 || t < best) {
            best = t;
            f.row_waves = rw;
            f.items = (uint32_t)(rows / (32 * rw) + big + 1);
            f.target = cut ? num_cu : 0;
            f.pieces = cut ? (stages + kLeastStages - 1) / kLeastStages : 1;
        }
    }
    if (f.together) f.column_ctas = std::min(rows / (32 * f.row_waves) * pool.heads >= num_cu / 4 ? num_cu / 2 : num_cu * 11 / 16, kPagedMostWaves / 8);
    if (f.together && windowed) {
        // Rows of the table that have no new tokens are not told apart from decoding ones, but by this: beside the longest new tokens no more sequences decode than tokens are left.  (Taking
        // fewer for decoding than do would cost more than it saves: 64 decoding ones, 8-bit, left to 16 compute units are 700 us of reading.)  64 decoding and 512 in a table of 256 rows, 8-bit: 171 us
        // with all other rows taken for decoding ones, like this 147 (133 in a table of 65); 8 decoding and 300, 16 / 2 heads, 49 and 45 (33); the rest is the plan's loop over the rows.
        const long count = std::max(most / G, 1L), chunks = std::min(std::max((seqs.tokens - seqs.batch + count - 1) / count, 1L), (long)seqs.batch);
        const long decoding = std::max(std::min(seqs.batch - chunks, seqs.tokens - count), 0L);
        const double tiles = (double)(seqs.tokens - decoding) * G / (32 * f.row_waves) * pool.heads;         // (more than 0: tokens beyond `decoding` are at least `count`)
        if (tiles < num_cu) {
            const double columns = (double)decoding * std::min((long)len, (long)seqs.window + seqs.sinks) * pool.heads * (32 * pool.bits + 8) / (pool.bits == 8 ? 50e3 : 38e3);
            const double tall = tiles * (stages + 5.0) * (f.row_waves == 8 ? 2.3 : 1.5);
            f.column_ctas = std::min(std::max((int)(num_cu * columns / (columns + tall)), num_cu / 16), std::min(num_cu * 11 / 16, kPagedMostWaves / 8));
        }
    }
    return f;
}

hipError_t launch_paged_rows(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, const PagedForm& f, void* workspace,
                             hipStream_t stream)
{
    return launch_rows_of<false>(pool, seqs, Q, q_stride, O, q_heads, scale, f, workspace, stream);
}

hipError_t launch_paged_attn(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, int max_count, int max_len,
                             int num_cu, void* workspace, hipStream_t stream)
{
    const PagedForm f = paged_form(pool, seqs, q_heads, max_count, max_len, num_cu);
    const bool window = seqs.window < seqs.cap;
    hipError_t e = hipSuccess;
    if (f.row_waves) e = (window ? launch_paged_rows_window : launch_paged_rows)(pool, seqs, Q, q_stride, O, q_heads, scale, f, workspace, stream);
    if (e == hipSuccess && f.column_rows && !f.together)
        e = (window ? launch_paged_columns_window : launch_paged_columns)(pool, seqs, Q, q_stride, O, q_heads, scale, f.columns, f.column_rows, f.column_ctas, f.alone, workspace, stream);
    return e;
}

}  // namespace tmw4
