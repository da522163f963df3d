// Pages of a free list for the new tokens of a call, and back (tm_paged_assign, tm_paged_release).
//
// Rows' tokens and pages are two prefix sums over the rows: where a row's tokens lie in the packed arrays, and which pages of the list are its.  Everything else is a thread's own: a
// token's page is an entry that the row had, or a page of the list, and the token that begins a page writes the entry.
#include "tm_paged_host.h"

#include <limits.h>

#include <algorithm>

namespace tmw4 {

namespace {

constexpr int kPlanThreads = 1024;       // most rows that a CTA works out at a time
constexpr int kOwnTokens = 8;            // of a row that its own thread places

// Inclusive sum over the CTA, at most 2^32 - 1 each; `total` is the CTA's.  `waves` may be used again behind another barrier.
template <int THREADS>
__device__ __forceinline__ uint32_t block_sums(uint32_t v, uint32_t* waves, uint32_t& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto add = [](uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); };
    v = wave_scan(v, add);
    if (lane == 63) waves[wave] = v;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const uint32_t n = waves[w];
        before = add(before, w < wave ? n : 0u);
        total = add(total, n);
    }
    return add(before, v);
}

// A row: its place in the packed arrays, and number `first - page` of the list is its page `page`.
struct AssignedRow {
    int row, end, len, stop, first;
    bool served;
};

// sums: room for two sums over the CTA.
template <int THREADS>
struct AssignPlan {
    uint32_t tokens, pages;              // of the rows so far: given or not
    uint32_t given;                      // pages given to the thread's rows and all before them, if those were given any
    int available;
    __device__ __forceinline__ AssignedRow next(const AssignJob& j, int b, uint32_t (*sums)[THREADS / 64])
    {
        const int cap = j.cap, page = 1 << j.page_log;
        int len = 0;
        uint32_t count = 0, all;
        if (b < j.batch) {
            len = min(max(j.lens[b], 0), cap);
            count = (uint32_t)max(j.counts[b], 0);
        }
        AssignedRow r;
        const uint32_t end = __builtin_elementwise_add_sat(block_sums<THREADS>(count, sums[0], all), tokens);
        r.end = (int)min(end, (uint32_t)j.tokens);
        r.row = (int)min(end == ~0u ? ~0u : end - count, (uint32_t)j.tokens);
        tokens = __builtin_elementwise_add_sat(tokens, all);
        r.len = len;
        r.stop = (int)min((uint32_t)len + (uint32_t)(r.end - r.row), (uint32_t)cap);
        const int have = (len + page - 1) >> j.page_log;
        const uint32_t need = (uint32_t)max(((r.stop + page - 1) >> j.page_log) - have, 0);
        const uint32_t until = block_sums<THREADS>(need, sums[1], all) + pages;         // (at most tokens / 32 + batch)
        pages += all;
        r.served = need == 0 || until <= (uint32_t)available;
        r.first = available - 1 - (int)(until - need) + have;
        if (r.served && need) given = until;
        return r;
    }
};

__device__ __forceinline__ int available_pages(const AssignJob& j) { return min(max(*j.count, 0), j.capacity); }

// What is known of a row but its length, which other CTAs may still have to read.
__device__ __forceinline__ void write_row(const AssignJob& j, int b, const AssignedRow& r)
{
    j.offsets[b] = r.row;
    if (b == j.batch - 1) j.offsets[j.batch] = r.end;
    j.positions[b] = r.len;
    if (j.lacking) j.lacking[b] = r.served ? 0 : 1;
}

// Token `t` of the packed arrays; offset, len, first, served: of row b, which has it.
__device__ __forceinline__ void place_token(const AssignJob& j, int b, int t, int offset, int len, int first, bool served)
{
    const int page = 1 << j.page_log, at = (int)min((uint32_t)len + (uint32_t)(t - offset), (uint32_t)j.cap), number = at >> j.page_log;
    int id = -1;
    if (at < j.cap) {
        const bool old = number < (len + page - 1) >> j.page_log;
        int32_t* const entry = j.table + (size_t)b * j.max_pages + number;
        if (served) id = old ? *entry : j.pages[first - number];
        if (!old && (at & (page - 1)) == 0) *entry = id;
    }
    if (j.slots) j.slots[t] = (uint32_t)id < (uint32_t)j.pool_pages ? (int64_t)id << j.page_log | (at & (page - 1)) : -1;
}

// Up to THREADS rows: every CTA works out the rows for itself and places its share of the tokens: the first one, a thread a row, those of rows with up to kOwnTokens of them, and the others
// by search.  The lengths and the list's count may be updated in place, so they are written by the CTA that is last to have read them.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void assign_kernel(AssignJob j, uint32_t* arrived)
{
    __shared__ uint32_t sums[2][THREADS / 64], s_last, s_taken;
    __shared__ int s_end[THREADS], s_row[THREADS], s_len[THREADS], s_first[THREADS];
    const int b = threadIdx.x;
    if (b == 0) s_taken = 0;
    AssignPlan<THREADS> plan{0u, 0u, 0u, available_pages(j)};
    const AssignedRow r = plan.next(j, b, sums);
    const bool mine = r.end - r.row <= kOwnTokens;           // to place by its own thread
    const uint32_t given = wave_greatest(plan.given);
    if ((b & 63) == 0 && given) atomicMax(&s_taken, given);
    s_end[b] = b < j.batch ? r.end : j.tokens;
    s_row[b] = r.row;
    s_len[b] = r.len;
    s_first[b] = r.served ? r.first : INT_MIN;
    if (blockIdx.x == 0 && b < j.batch) {
        write_row(j, b, r);
        if (mine)
            for (int t = r.row; t < r.end; ++t) place_token(j, b, t, r.row, r.len, r.first, r.served);
    }
    const bool search = __syncthreads_or(!mine);
    if (gridDim.x > 1) {
        if (b == 0) s_last = atomicAdd(arrived, 1u) == gridDim.x - 1;
        __syncthreads();
    }
    if (gridDim.x == 1 || s_last) {                          // (uniform)
        if (b < j.batch) j.lens_out[b] = r.served ? r.stop : r.len;
        if (b == 0) {
            *j.left = plan.available - (int)s_taken;
            if (gridDim.x > 1) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (!search) return;
    const int all = s_end[j.batch - 1];
    for (int t = (int)blockIdx.x * THREADS + b; t < all; t += (int)gridDim.x * THREADS) {
        int lo = 0;                                          // rows that end at t or before
#pragma unroll
        for (int step = THREADS / 2; step; step >>= 1)
            if (lo + step <= j.batch && s_end[lo + step - 1] <= t) lo += step;
        lo = min(lo, j.batch - 1);
        if (s_end[lo] - s_row[lo] > kOwnTokens) place_token(j, lo, t, s_row[lo], s_len[lo], s_first[lo], s_first[lo] != INT_MIN);
    }
}

// More rows: one CTA works them out, kPlanThreads at a time, the tokens follow in a launch of their own.
__global__ __launch_bounds__(kPlanThreads) void assign_rows_kernel(AssignJob j, int32_t* __restrict__ first)
{
    __shared__ uint32_t sums[2][kPlanThreads / 64], s_taken;
    AssignPlan<kPlanThreads> plan{0u, 0u, 0u, available_pages(j)};
    if (threadIdx.x == 0) s_taken = 0;
    for (int b0 = 0; b0 < j.batch; b0 += kPlanThreads) {
        const int b = b0 + (int)threadIdx.x;
        if (b0) __syncthreads();                             // (the sums have been read)
        const AssignedRow r = plan.next(j, b, sums);
        if (b >= j.batch) continue;
        write_row(j, b, r);
        j.lens_out[b] = r.served ? r.stop : r.len;
        first[b] = r.served ? r.first : INT_MIN;
    }
    atomicMax(&s_taken, plan.given);
    __syncthreads();
    if (threadIdx.x == 0) *j.left = plan.available - (int)s_taken;
}

__global__ __launch_bounds__(256) void assign_tokens_kernel(AssignJob j, const int32_t* __restrict__ first)
{
    const int t = (int)(blockIdx.x * 256 + threadIdx.x);
    if (t >= j.offsets[j.batch]) return;
    int lo = 0;                                              // rows that end at t or before
    for (int step = 1 << 15; step; step >>= 1)
        if (lo + step <= j.batch && j.offsets[lo + step] <= t) lo += step;
    lo = min(lo, j.batch - 1);
    place_token(j, lo, t, j.offsets[lo], j.positions[lo], first[lo], first[lo] != INT_MIN);
}

// ---- back.  Entries of row b whose pages' tokens all lie in the row's range.
__device__ __forceinline__ void released_entries(const ReleaseJob& j, int b, int& e0, int& e1)
{
    const int64_t page = int64_t(1) << j.page_log, from = j.from ? max(j.from[b], 0) : 0;
    const int to = j.to ? max(j.to[b], 0) : INT_MAX;
    e0 = (int)min((from + page - 1) >> j.page_log, (int64_t)j.max_pages);
    e1 = to >= j.cap ? j.max_pages : to >> j.page_log;
}

// counts[b]: pages that row b gives back; counts[batch]: what the list has.
__global__ __launch_bounds__(256) void release_count_kernel(ReleaseJob j, int32_t* __restrict__ counts)
{
    __shared__ int total;
    const int b = (int)blockIdx.x, tid = threadIdx.x;
    int e0, e1, n = 0;
    released_entries(j, b, e0, e1);
    if (tid == 0) total = 0;
    __syncthreads();
    for (int e = e0 + tid; e < e1; e += 256) n += (uint32_t)j.table[(size_t)b * j.max_pages + e] < (uint32_t)j.pool_pages;
    n = (int)wave_total((uint32_t)n);
    if ((tid & 63) == 0 && n) atomicAdd(&total, n);
    __syncthreads();
    if (tid == 0) counts[b] = total;
    if (b == 0 && tid == 0) counts[j.batch] = min(max(*j.count, 0), j.capacity);
}

// The first row's first page comes to lie last, so that it is taken first.
__global__ __launch_bounds__(256) void release_kernel(ReleaseJob j, const int32_t* __restrict__ counts)
{
    __shared__ uint32_t waves[2][4];
    const int b = (int)blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    uint32_t before = 0, all = 0, sum;
    for (int i = tid; i < j.batch; i += 256) {
        const uint32_t n = (uint32_t)counts[i];
        all += n;
        before += i < b ? n : 0u;
    }
    block_sums<256>(before, waves[0], sum);
    before = sum;
    block_sums<256>(all, waves[1], sum);
    all = sum;
    const long top = (long)counts[j.batch] + all;            // pages of the list then
    if (b == 0 && tid == 0) *j.left = (int)min(top, (long)j.capacity);
    if (counts[b] == 0) return;
    int e0, e1;
    released_entries(j, b, e0, e1);
    for (int base = e0; base < e1; base += 256) {
        __syncthreads();                                     // (the sums have been read)
        const int e = base + tid;
        int32_t* const entry = j.table + (size_t)b * j.max_pages + e;
        const int id = e < e1 ? *entry : -1;
        const bool live = (uint32_t)id < (uint32_t)j.pool_pages;
        const uint64_t mask = __builtin_amdgcn_ballot_w64(live);
        const uint32_t until = block_sums<256>(lane == 63 ? (uint32_t)__builtin_popcountll(mask) : 0u, waves[0], sum);     // of the waves up to this one in the last lane, before it in the others
        const uint32_t rank = (lane == 63 ? until - (uint32_t)__builtin_popcountll(mask) : until) + (uint32_t)__builtin_popcountll(mask & ((uint64_t(1) << lane) - 1));
        if (live) {
            const long at = top - 1 - (long)before - rank;
            if (at >= 0 && at < j.capacity) j.pages[at] = id;
            *entry = -1;
        }
        before += sum;
    }
}

}  // namespace

hipError_t launch_assign(const AssignJob& j, int num_cu, void* workspace, hipStream_t stream)
{
    int32_t* const first = (int32_t*)((char*)workspace + kPagedCounterBytes);
    if (j.batch <= kPlanThreads) {
        const unsigned threads = j.batch <= 256 ? 256 : kPlanThreads;
        // tokens that are not more than the rows' own threads place need one CTA
        const long blocks = (long)j.tokens <= kOwnTokens * 64 ? 1 : std::min(((long)j.tokens + threads - 1) / threads, (long)num_cu);
        const auto kernel = threads == 256 ? assign_kernel<256> : assign_kernel<kPlanThreads>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::max(blocks, 1L)), dim3(threads), 0, stream, j, (uint32_t*)((char*)workspace + kPagedArrivedAt));
        return hipGetLastError();
    }
    hipLaunchKernelGGL(assign_rows_kernel, dim3(1), dim3(kPlanThreads), 0, stream, j, first);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || j.tokens == 0) return e;
    hipLaunchKernelGGL(assign_tokens_kernel, dim3((unsigned)(((long)j.tokens + 255) / 256)), dim3(256), 0, stream, j, first);
    return hipGetLastError();
}

hipError_t launch_release(const ReleaseJob& j, void* workspace, hipStream_t stream)
{
    int32_t* const counts = (int32_t*)((char*)workspace + kPagedCounterBytes);
    hipLaunchKernelGGL(release_count_kernel, dim3((unsigned)j.batch), dim3(256), 0, stream, j, counts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(release_kernel, dim3((unsigned)j.batch), dim3(256), 0, stream, j, counts);
    return hipGetLastError();
}

}  // namespace tmw4
