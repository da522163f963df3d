// Pages of a free list for the new tokens of a call, and back (tm_paged_assign, tm_paged_release).
//
// Rows' tokens and pages are two prefix sums over the rows: where a row's tokens lie in the packed arrays, and which pages of the list are its.  Everything else is a thread's own: a
// token's page is an entry that the row had, or a page of the list, and the token that begins a page writes the entry.
//
// Measured: 256 rows of one new token 4.2 us a call (2.7 in a graph), 1000 rows with 45000 tokens 5.1, 64 rows with 66000 6.8, 2048 rows of one token 7.9.  A launch, and a chain of trips to memory:
// lengths, table or list, results, with two sums over the CTA between; the host's part of the call is longer than the kernel's up to some thousand tokens.  Rows of more than kOwnTokens new tokens are
// searched for by each token, 0.5 us.
#include "tm_paged_host.h"

#include <limits.h>

#include <algorithm>

namespace tmw4 {

namespace {

constexpr int kPlanThreads = 1024;       // of the CTA that works out many rows,
constexpr int kPlanRows = 4;             // and rows of each
constexpr int kOwnTokens = 8;            // of a row that its own thread places

__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Sum over the threads before this one, at most 2^32 - 1; `total` is the CTA's.  `waves` may be used again behind another barrier.
template <int THREADS>
__device__ __forceinline__ uint32_t sums_before(uint32_t v, uint32_t* waves, uint32_t& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v = wave_scan(v, add_sat);
    if (lane == 63) waves[wave] = v;
    __syncthreads();
    uint32_t before = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x138, 0xf, 0xf, false);           // of the lane before
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const uint32_t n = waves[w];
        before = add_sat(before, w < wave ? n : 0u);
        total = add_sat(total, n);
    }
    return before;
}

// A row: its place in the packed arrays, and number `first - page` of the list is its page `page`.
struct AssignedRow {
    int row, end, len, stop, first;
    bool served;
};

// A thread has the ROWS rows from b on.
template <int THREADS, int ROWS>
struct AssignPlan {
    uint32_t tokens, pages;              // of the rows so far: given or not
    uint32_t given;                      // pages given to the thread's rows and all before them, if those were given any
    int available;
    __device__ __forceinline__ void next(const AssignJob& j, int b, uint32_t (*sums)[THREADS / 64], AssignedRow (&r)[ROWS])
    {
        const int cap = j.cap, page = 1 << j.page_log;
        uint32_t count[ROWS], need[ROWS], own = 0, all;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            count[i] = 0;
            r[i].len = 0;
            if (b + i < j.batch) {
                r[i].len = min(max(j.lens[b + i], 0), cap);
                count[i] = (uint32_t)max(j.counts[b + i], 0);
            }
            own = add_sat(own, count[i]);
        }
        uint32_t at = add_sat(sums_before<THREADS>(own, sums[0], all), tokens);
        tokens = add_sat(tokens, all);
        own = 0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            r[i].row = (int)min(at, (uint32_t)j.tokens);
            at = add_sat(at, count[i]);
            r[i].end = (int)min(at, (uint32_t)j.tokens);
            r[i].stop = (int)min((uint32_t)r[i].len + (uint32_t)(r[i].end - r[i].row), (uint32_t)cap);
            need[i] = (uint32_t)max(((r[i].stop + page - 1) >> j.page_log) - ((r[i].len + page - 1) >> j.page_log), 0);
            own += need[i];                                  // (all rows' together: at most tokens / 32 + batch)
        }
        uint32_t until = sums_before<THREADS>(own, sums[1], all) + pages;
        pages += all;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            r[i].first = available - 1 - (int)until + ((r[i].len + page - 1) >> j.page_log);
            until += need[i];
            r[i].served = need[i] == 0 || until <= (uint32_t)available;
            if (r[i].served && need[i]) given = until;
        }
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

// Up to THREADS * ROWS rows: every CTA works out the rows for itself and places its share of the tokens: the first one, a thread its rows, those of rows with up to kOwnTokens of them, and
// the others by search.  The lengths and the list's count may be updated in place, so they are written by the CTA that is last to have read them.
template <int THREADS, int ROWS>
__global__ __launch_bounds__(THREADS) void assign_kernel(AssignJob j, uint32_t* arrived)
{
    __shared__ uint32_t sums[2][THREADS / 64], s_last, s_taken;
    __shared__ int s_end[THREADS * ROWS], s_len[THREADS * ROWS], s_first[THREADS * ROWS];
    const int tid = threadIdx.x, b = tid * ROWS;
    if (tid == 0) s_taken = 0;
    AssignPlan<THREADS, ROWS> plan{0u, 0u, 0u, available_pages(j)};
    AssignedRow r[ROWS];
    plan.next(j, b, sums, r);
    bool mine = true;                                        // to place by their own thread
    const uint32_t given = wave_greatest(plan.given);
    if ((tid & 63) == 0 && given) atomicMax(&s_taken, given);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        mine = mine && r[i].end - r[i].row <= kOwnTokens;
        s_end[b + i] = r[i].end;
        s_len[b + i] = r[i].len;
        s_first[b + i] = r[i].served ? r[i].first : INT_MIN;
        if (blockIdx.x == 0 && b + i < j.batch) {
            write_row(j, b + i, r[i]);
            if (r[i].end - r[i].row <= kOwnTokens)
                for (int t = r[i].row; t < r[i].end; ++t) place_token(j, b + i, t, r[i].row, r[i].len, r[i].first, r[i].served);
        }
    }
    const bool search = __syncthreads_or(!mine);
    if (gridDim.x > 1) {
        if (tid == 0) s_last = atomicAdd(arrived, 1u) == gridDim.x - 1;
        __syncthreads();
    }
    if (gridDim.x == 1 || s_last) {                          // (uniform)
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            if (b + i < j.batch) j.lens_out[b + i] = r[i].served ? r[i].stop : r[i].len;
        if (tid == 0) {
            *j.left = plan.available - (int)s_taken;
            if (gridDim.x > 1) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (!search) return;
    const uint32_t all = (uint32_t)s_end[j.batch - 1];
    for (uint32_t at = blockIdx.x * THREADS + tid; at < all; at += gridDim.x * THREADS) {     // (below 2^31, and a step is at most 2^18)
        const int t = (int)at;
        int lo = 0;                                          // rows that end at t or before
#pragma unroll
        for (int step = THREADS * ROWS / 2; step; step >>= 1)
            if (lo + step <= j.batch && s_end[lo + step - 1] <= t) lo += step;
        lo = min(lo, j.batch - 1);
        const int row = lo ? s_end[lo - 1] : 0;
        if (s_end[lo] - row > kOwnTokens) place_token(j, lo, t, row, s_len[lo], s_first[lo], s_first[lo] != INT_MIN);
    }
}

// More rows: one CTA works them out, some thousand at a time, the tokens follow in a launch of their own.
__global__ __launch_bounds__(kPlanThreads) void assign_rows_kernel(AssignJob j, int32_t* __restrict__ first)
{
    __shared__ uint32_t sums[2][kPlanThreads / 64], s_taken;
    AssignPlan<kPlanThreads, kPlanRows> plan{0u, 0u, 0u, available_pages(j)};
    if (threadIdx.x == 0) s_taken = 0;
    for (int b0 = 0; b0 < j.batch; b0 += kPlanThreads * kPlanRows) {
        const int b = b0 + (int)threadIdx.x * kPlanRows;
        if (b0) __syncthreads();                             // (the sums have been read)
        AssignedRow r[kPlanRows];
        plan.next(j, b, sums, r);
#pragma unroll
        for (int i = 0; i < kPlanRows; ++i) {
            if (b + i >= j.batch) continue;
            write_row(j, b + i, r[i]);
            j.lens_out[b + i] = r[i].served ? r[i].stop : r[i].len;
            first[b + i] = r[i].served ? r[i].first : INT_MIN;
        }
    }
    atomicMax(&s_taken, plan.given);
    __syncthreads();
    if (threadIdx.x == 0) *j.left = plan.available - (int)s_taken;
}

__global__ __launch_bounds__(256) void assign_tokens_kernel(AssignJob j, const int32_t* __restrict__ first)
{
    const uint32_t at = blockIdx.x * 256 + threadIdx.x;
    if (at >= (uint32_t)j.offsets[j.batch]) return;
    const int t = (int)at;
    int lo = 0;                                              // rows that end at t or before
    for (int step = 1 << 15; step; step >>= 1)
        if (lo + step <= j.batch && j.offsets[lo + step] <= t) lo += step;
    lo = min(lo, j.batch - 1);
    place_token(j, lo, t, j.offsets[lo], j.positions[lo], first[lo], first[lo] != INT_MIN);
}

// ---- back.  Two launches, up to 4096 rows a CTA a row in each: 6.5 us up to 1000 rows of 300 entries that are gone through, 6.8 for 4000 of 100 (11.8 while rows that give nothing summed the counts too).
// Entries of row b whose pages' tokens all lie in the row's range.
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
    const int b = (int)blockIdx.x, tid = threadIdx.x;
    if (b && counts[b] == 0) return;                         // (in a window most rows give nothing in most steps)
    uint32_t before = 0, all = 0, sum;
    for (int i = tid; i < j.batch; i += 256) {
        const uint32_t n = (uint32_t)counts[i];
        all += n;
        before += i < b ? n : 0u;
    }
    sums_before<256>(before, waves[0], sum);
    before = sum;
    sums_before<256>(all, waves[1], sum);
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
        const uint32_t rank = sums_before<256>(live ? 1u : 0u, waves[0], sum);
        if (live) {
            const long at = top - 1 - (long)before - rank;
            if (at >= 0 && at < j.capacity) j.pages[at] = id;
            *entry = -1;
        }
        before += sum;
    }
}

// More than kGroupsFrom rows: a CTA takes kGroupRows of them, a wave a row at a time, and leaves their sum, so that the CTAs of the second launch sum groups and not rows.  Rows of ten entries that give a
// page each / none, in brackets a CTA a row: 8000 7.4 / 6.7 us (28.5 / 9.9), 20000 10.1 / 7.3 (118 / 19), 65000 27 / 12 (1000 / 54); 8000 of 500 27 / 10 (37 / 10).  With fewer rows a CTA a row
// goes through a long row sooner: 1000 of 1000 7.4 us (35 by groups), 4000 of 500 16.5 (23), while 4000 of ten take 12.3 (6.8).
constexpr int kGroupRows = 16, kGroupsFrom = 4096;
static_assert(kGroupRows % 4 == 0 && kGroupRows <= 64, "rows of four waves, and of the lanes of one");

// counts and groups follow each other: rows, what the list has, groups.
struct GroupedCounts {
    int32_t* counts;
    uint32_t* groups;
    int number;
    __host__ __device__ GroupedCounts(int32_t* at, int batch) : counts(at), groups((uint32_t*)at + batch + 1), number((batch + kGroupRows - 1) / kGroupRows) {}
};

__global__ __launch_bounds__(256) void release_count_groups_kernel(ReleaseJob j, int32_t* at)
{
    __shared__ uint32_t waves[4];
    const GroupedCounts c(at, j.batch);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), first = (int)blockIdx.x * kGroupRows;
    uint32_t total = 0;
    for (int b = first + wave; b < min(first + kGroupRows, j.batch); b += 4) {
        int e0, e1;
        uint32_t n = 0;
        released_entries(j, b, e0, e1);
        for (int e = e0 + lane; e < e1; e += 64) n += (uint32_t)j.table[(size_t)b * j.max_pages + e] < (uint32_t)j.pool_pages;
        n = wave_total(n);
        if (lane == 0) c.counts[b] = (int)n;
        total += n;
    }
    if (lane == 0) waves[wave] = total;
    __syncthreads();
    if (tid == 0) c.groups[blockIdx.x] = waves[0] + waves[1] + waves[2] + waves[3];
    if (blockIdx.x == 0 && tid == 0) c.counts[j.batch] = min(max(*j.count, 0), j.capacity);
}

__global__ __launch_bounds__(256) void release_groups_kernel(ReleaseJob j, int32_t* at)
{
    __shared__ uint32_t waves[2][4];
    const GroupedCounts c(at, j.batch);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), group = (int)blockIdx.x, first = group * kGroupRows;
    if (group && c.groups[group] == 0) return;
    uint32_t before = 0, all = 0, sum;
    for (int i = tid; i < c.number; i += 256) {
        const uint32_t n = c.groups[i];
        all += n;
        before += i < group ? n : 0u;
    }
    sums_before<256>(before, waves[0], sum);
    before = sum;
    sums_before<256>(all, waves[1], sum);
    const long top = (long)c.counts[j.batch] + sum;          // pages of the list then
    if (group == 0 && tid == 0) *j.left = (int)min(top, (long)j.capacity);
    const uint32_t n = lane < kGroupRows && first + lane < j.batch ? (uint32_t)c.counts[first + lane] : 0u, incl = wave_sums(n);      // a lane a row
    for (int r = wave; r < kGroupRows; r += 4) {
        const uint32_t mine = (uint32_t)__builtin_amdgcn_readlane((int)n, r);
        if (mine == 0) continue;
        const int b = first + r;
        uint32_t rank = before + (uint32_t)__builtin_amdgcn_readlane((int)incl, r) - mine;
        int e0, e1;
        released_entries(j, b, e0, e1);
        for (int base = e0; base < e1; base += 64) {
            const int e = base + lane;
            int32_t* const entry = j.table + (size_t)b * j.max_pages + e;
            const int id = e < e1 ? *entry : -1;
            const bool live = (uint32_t)id < (uint32_t)j.pool_pages;
            const uint64_t there = __builtin_amdgcn_ballot_w64(live);
            if (live) {
                const long place = top - 1 - (long)rank - __builtin_popcountll(there & ((1ull << lane) - 1));
                if (place >= 0 && place < j.capacity) j.pages[place] = id;
                *entry = -1;
            }
            rank += (uint32_t)__builtin_popcountll(there);
        }
    }
}

}  // namespace

hipError_t launch_assign(const AssignJob& j, int num_cu, void* workspace, hipStream_t stream)
{
    int32_t* const first = (int32_t*)((char*)workspace + kPagedCounterBytes);
    if (j.batch <= kPlanThreads * kPlanRows) {
        const unsigned threads = j.batch <= 256 ? 256 : kPlanThreads;
        // tokens that are not more than the rows' own threads place need one CTA
        const long blocks = (long)j.tokens <= kOwnTokens * 64 ? 1 : std::min(((long)j.tokens + threads - 1) / threads, (long)num_cu);
        const auto kernel = j.batch <= 256 ? assign_kernel<256, 1> : j.batch <= kPlanThreads ? assign_kernel<kPlanThreads, 1> : assign_kernel<kPlanThreads, kPlanRows>;
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
    static_assert(sizeof(int32_t) * (65535 + 1 + 65535 / kGroupRows + 1) <= kPagedColumnBytes, "counts of rows and groups");
    int32_t* const counts = (int32_t*)((char*)workspace + kPagedCounterBytes);
    if (j.batch > kGroupsFrom) {
        const dim3 groups((unsigned)((j.batch + kGroupRows - 1) / kGroupRows));
        hipLaunchKernelGGL(release_count_groups_kernel, groups, dim3(256), 0, stream, j, counts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(release_groups_kernel, groups, dim3(256), 0, stream, j, counts);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(release_count_kernel, dim3((unsigned)j.batch), dim3(256), 0, stream, j, counts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(release_kernel, dim3((unsigned)j.batch), dim3(256), 0, stream, j, counts);
    return hipGetLastError();
}

}  // namespace tmw4
