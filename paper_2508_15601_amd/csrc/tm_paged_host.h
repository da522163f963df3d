// Host-side declarations of the paged cache and of the rotary positions.
#pragma once
#include "tm_paged_device.h"
#include "tm_rope_device.h"

namespace tmw4 {

// Workspace of tm_paged_attn: arrival counters and the length of a call's pieces, then partial results of contexts that are cut into pieces.
constexpr size_t kPagedCounterBytes = 32 * 1024;
constexpr size_t kPagedLengthAt = kPagedCounterBytes - 64;
constexpr size_t kPagedColumnBytes = 23u << 20;           // two pieces each of 1408 waves
constexpr size_t kPagedRowBytes = 33u << 20;              // 259 pieces of 256 rows
constexpr size_t kPagedWorkspaceBytes = kPagedCounterBytes + kPagedColumnBytes + kPagedRowBytes;

constexpr int kPagedMostCtas = 512;      // of a launch whose CTAs share contexts
constexpr int kPagedMostWaves = 1408;    // of one whose waves do

// CTAs that a launch may have at most: its threads are counted in 32 bits.
constexpr long most_ctas(int threads) { return 0xffffffffL / threads; }

struct PagedRows {                       // a packed array of new tokens: row r at p + r * stride
    const uint16_t* p;
    long stride;
};

// Most runs that the sequences' new tokens can touch.
inline long most_runs(const PagedSeqs& s)
{
    const long spread = s.tokens / kRun + 2L * s.batch;
    return spread < s.tokens ? spread : s.tokens;
}

hipError_t launch_rope(const uint16_t* X, long x_stride, const int32_t* positions, const RopePlan& r, uint16_t* Y, long y_stride, int tokens, int heads,
                       int dim, hipStream_t stream);
// q.p == nullptr: keys and values only; rope == nullptr: stored as they are
hipError_t launch_paged_append(const PagedPool& pool, const PagedSeqs& seqs, PagedRows k, PagedRows v, const RopePlan* rope, PagedRows q, uint16_t* q_out,
                               long q_out_stride, int q_heads, int max_count, int num_cu, hipStream_t stream);
hipError_t launch_paged_read(const PagedPool& pool, const PagedSeqs& seqs, uint16_t* K, uint16_t* V, hipStream_t stream);
// The new tokens of sequences with up to most_rows (token, query head of a KV head) rows; `columns` of them at a time, 8, 16 or 32.  Every CTA of `grid`, or every wave (alone; not
// with 32 columns), takes an equal piece of the work.
hipError_t launch_paged_columns(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, int columns,
                                int most_rows, int grid, bool alone, void* workspace, hipStream_t stream);

// How a call is divided: sequences with at least least_rows rows in CTAs of 32 * row_waves rows (row_waves = 0: none), the others by columns (column_rows = 0: none).
struct PagedForm {
    int columns, column_rows, column_ctas;
    bool alone, together;                // columns: every wave by itself; in one launch with the rows
    int least_rows, row_waves, pieces, target;
    uint32_t items;
};
PagedForm paged_form(const PagedPool& pool, const PagedSeqs& seqs, int q_heads, int max_count, int max_len, int num_cu);
hipError_t paged_rows_setup();                                         // once per device, outside any capture
hipError_t launch_paged_attn(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, int max_count, int max_len,
                             int num_cu, void* workspace, hipStream_t stream);

}  // namespace tmw4
