// Device-side view of a paged cache and of the sequences a call works on, and how a wave finds its sequence.
#pragma once
#include "tm_w4_device.h"

namespace tmw4 {

constexpr int kRun = 32;                 // tokens of a run: the unit in which codes are laid out

// Pool of pages.  Page p, KV head h, run r of the page: codes at ((p * heads + h) << run_log | r) runs, scale / zero-point words of
// token t of the page at word ((p * heads + h) << (run_log + 5) | t) * 2 (key, value).
struct PagedPool {
    uint8_t* k;
    uint8_t* v;
    uint32_t* pairs;
    int pages, heads, run_log;           // runs of a page = 1 << run_log
    int bits;
};

// The sequences of a call.  Rows offsets[b] .. offsets[b+1] - 1 of the packed arrays are the new tokens of sequence b; row i of it sits
// at position positions[b] + i.
struct PagedSeqs {
    const int32_t* table;                // [batch][max_pages] page numbers; one outside the pool holds no tokens
    const int32_t* offsets;              // [batch + 1]
    const int32_t* positions;            // [batch]
    int batch, max_pages, tokens, cap;   // cap = tokens a row of the table can hold
    int window, sinks;                   // kernels of a sliding window: the token at p sees tokens p - window + 1 .. p and 0 .. sinks - 1, both at most cap
};

// Pieces of `size` tokens that nobody from position `first` on sees: between the first tokens and the window.  What is left is numbered through.
struct Hidden {
    int from, count;                     // pieces 0 .. from - 1 are seen, the next `count` are not
    __device__ __forceinline__ Hidden(const PagedSeqs& s, int first, int size)
    {
        from = (s.sinks + size - 1) / size;
        count = max(max(min(first, s.cap - 1) - s.window + 1, 0) / size - from, 0);
    }
    __device__ __forceinline__ int real(int piece) const { return piece < from ? piece : piece + count; }
};

// An element of an array that no kernel of the launch writes.  With a wave-uniform index it is a scalar load, whatever the kernel stores elsewhere: as a vector load it would
// stand in line with the blocks of codes, and waiting for a page number would be waiting for them.
__device__ __forceinline__ int constant_load(const int32_t* p, size_t i)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return ((const __attribute__((address_space(4))) int32_t*)p)[i];
#else
    return p[i];
#endif
}

struct PagedSeq {
    int row, count, pos;                 // first row, new tokens, position of the first
    __device__ __forceinline__ int first() const { return max(pos, 0); }             // cached positions of the new tokens: [first, last)
    __device__ __forceinline__ int last(int cap) const { return (int)min((long)pos + count, (long)cap); }
};

__device__ __forceinline__ PagedSeq paged_seq(const PagedSeqs& s, int b)
{
    const int o0 = min(max(constant_load(s.offsets, b), 0), s.tokens), o1 = min(max(constant_load(s.offsets, b + 1), 0), s.tokens);
    return PagedSeq{o0, max(o1 - o0, 0), constant_load(s.positions, b)};
}

// Inclusive sum over the lanes of a wave: rows of sixteen lanes, then the rows' totals to the rows behind them.
template <class F>
__device__ __forceinline__ uint32_t wave_scan(uint32_t v, F f)              // f(0, v) = v
{
    auto add = [&](auto CTRL, auto ROWS) {
        v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(CTRL)::value, decltype(ROWS)::value, 0xf, false));
    };
    add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // row_shr by 1, 2, 4, 8
    add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast 15: last lane of a row to the next row
    add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // row_bcast 31: to the upper half
    return v;
}

__device__ __forceinline__ uint32_t wave_sums(uint32_t v)
{
    return wave_scan(v, [](uint32_t a, uint32_t b) { return a + b; });
}
__device__ __forceinline__ uint32_t wave_greatest(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_readlane((int)wave_scan(v, [](uint32_t a, uint32_t b) { return max(a, b); }), 63);
}
__device__ __forceinline__ uint32_t wave_total(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)wave_sums(v), 63); }

// Work laid out sequence after sequence: units_of(b) units belong to sequence b.  Every wave sums them up by itself (a lane takes
// ceil(batch / 64) neighbouring sequences; three loads each, all of them in the L2), so that no plan has to be made by another launch and
// nothing about the lengths has to be known on the host.  The total has to stay below 2^32; whatever the offsets hold, find() names a
// sequence that there is, and its callers check the unit against that sequence.
template <class F>
struct SeqFinder {
    F units_of;
    int per, batch;
    uint32_t mine, incl;                 // units of the lane's sequences; with those of the lanes before
    uint32_t total;

    __device__ __forceinline__ SeqFinder(F f, int sequences, int lane) : units_of(f), per((sequences + 63) / 64), batch(sequences), mine(0)
    {
        for (int j = 0; j < per; ++j) {
            const int b = lane * per + j;
            if (b < batch) mine += units_of(b);
        }
        incl = wave_sums(mine);
        total = (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
    }
    // A lane's work known already.
    __device__ __forceinline__ SeqFinder(F f, int sequences, uint32_t own) : units_of(f), per((sequences + 63) / 64), batch(sequences), mine(own)
    {
        incl = wave_sums(mine);
        total = (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
    }
    // The same again from the lane's two sums.
    __device__ __forceinline__ SeqFinder(F f, int sequences, uint32_t own, uint32_t sum)
        : units_of(f), per((sequences + 63) / 64), batch(sequences), mine(own), incl(sum), total(0)
    {
    }
    // The sequence that unit u < total belongs to, and its first unit (both wave-uniform).
    __device__ __forceinline__ int find(uint32_t u, uint32_t& base) const
    {
        const int l = __builtin_popcountll(__builtin_amdgcn_ballot_w64(incl <= u));
        base = (uint32_t)__builtin_amdgcn_readlane((int)(incl - mine), l);
        int b = l * per;
        for (int j = 1; j < per && b < batch; ++j) {
            const uint32_t n = units_of(b);
            if (u - base < n) break;
            base += n;
            ++b;
        }
        return min(b, batch - 1);
    }
};

// The table's entry for run `run` (counted over the sequence) of sequence b; the run must lie within the table's row.
__device__ __forceinline__ int paged_entry(const PagedPool& p, const PagedSeqs& s, int b, int run) 
{
    return constant_load(s.table, (size_t)b * s.max_pages + (run >> p.run_log));
}
// Its page number, -1 where that names none of the pool's.
__device__ __forceinline__ int paged_page(const PagedPool& p, const PagedSeqs& s, int b, int run)
{
    const int id = paged_entry(p, s, b, run);
    return (uint32_t)id < (uint32_t)p.pages ? id : -1;
}
// Number of a run in the pool.
__device__ __forceinline__ size_t paged_run(const PagedPool& p, int page, int head, int run)
{
    return (((size_t)page * p.heads + head) << p.run_log) + (run & ((1 << p.run_log) - 1));
}

// Runs of the cache in which a sequence has new tokens.
__device__ __forceinline__ uint32_t touched_runs(const PagedSeqs& s, const PagedSeq& q)
{
    const int f = q.first(), l = q.last(s.cap);
    return l > f ? (uint32_t)((l - 1) / kRun - f / kRun + 1) : 0u;
}

// A CTA's run: tokens u0 .. u1 - 1 of run `run` of sequence b are new.
struct RunJob {
    int b, run, u0, u1, page;
    long row;                            // packed row of the run's slot 0 (may lie before the first)
    bool live;
};
__device__ __forceinline__ RunJob run_job(const PagedPool& pool, const PagedSeqs& s, uint32_t item, int lane)
{
    RunJob j{};
    const SeqFinder finder([&](int b) { return touched_runs(s, paged_seq(s, b)); }, s.batch, lane);
    if (item >= finder.total) return j;
    uint32_t base;
    j.b = finder.find(item, base);
    const PagedSeq q = paged_seq(s, j.b);
    const int f = q.first(), l = q.last(s.cap);
    if (item - base >= touched_runs(s, q)) return j;
    j.run = f / kRun + (int)(item - base);
    const int t = j.run * kRun;
    j.u0 = max(f - t, 0);
    j.u1 = min(l - t, kRun);
    j.row = (long)q.row + ((long)t - q.pos);
    j.page = paged_page(pool, s, j.b, j.run);
    j.live = true;
    return j;
}

}  // namespace tmw4
