// Host-side declarations of the paged cache and of the rotary positions.
#pragma once
#include "tm_paged_device.h"
#include "tm_rope_device.h"

namespace tmw4 {

// Workspace of tm_paged_attn: arrival counters, then partial results of contexts that are cut into pieces.
constexpr size_t kPagedCounterBytes = 16 * 1024;
constexpr size_t kPagedPartialBytes = 48u << 20;
constexpr size_t kPagedWorkspaceBytes = kPagedCounterBytes + kPagedPartialBytes;

struct PagedRows {                       // a packed array of new tokens: row r at p + r * stride
    const uint16_t* p;
    long stride;
};

hipError_t launch_rope(const uint16_t* X, long x_stride, const int32_t* positions, const RopePlan& r, uint16_t* Y, long y_stride, int tokens, int heads,
                       int dim, hipStream_t stream);
// q.p == nullptr: keys and values only; rope == nullptr: stored as they are
hipError_t launch_paged_append(const PagedPool& pool, const PagedSeqs& seqs, PagedRows k, PagedRows v, const RopePlan* rope, PagedRows q, uint16_t* q_out,
                               long q_out_stride, int q_heads, hipStream_t stream);
hipError_t launch_paged_read(const PagedPool& pool, const PagedSeqs& seqs, uint16_t* K, uint16_t* V, hipStream_t stream);

}  // namespace tmw4
