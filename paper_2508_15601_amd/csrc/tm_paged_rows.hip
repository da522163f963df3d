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
// Measured (32 / 8 heads): prompts of 6000, 5000, 4000 and 3000 tokens, 8-bit: 860 us (0.82 PFLOP/s), 4-bit 853; 512 tokens after 30000, 4-bit: 297 us (0.85 PFLOP/s), 1024 without
// pieces; 100 after 8000, 8-bit: 42 us, 259 without pieces; one prompt of 4000: 163.  (Calls in a row; after an idle time, until the clock is up, a sixth more.)  What bounds it is the issue of
// vector and matrix instructions (tm_attn_prefill.hip) and a wait for memory in every stage (tm_attn_rows_impl.h); a piece of 256 rows leaves 133 KB in memory.
#include "tm_attn_rows_impl.h"
#include "tm_paged_columns_impl.h"
#include "tm_paged_host.h"

#include <algorithm>

namespace tmw4 {

namespace {

struct RowsPlan {
    int least_rows;                      // sequences with fewer rows are not this launch's
    int target;                          // CTAs that fill the chip; 0: no context is cut
    uint32_t slots;                      // pieces of cut contexts at most, KV heads counted: the workspace and the grid have room for them
    int32_t* length;                     // where the launch leaves the stages of a piece for the second kernel
};

constexpr int kLeastStages = 8;          // of 64 tokens: no piece is shorter, but for the last of a context
// Costs in the time of a stage, 2.3 us with 256 rows: what a CTA takes beside its stages; a piece's results on their way through memory (133 KB, twice, at 4.5 TB/s over the chip)
// in CTAs of 256 rows; the second kernel.
constexpr float kCtaCost = 5.0f, kPieceCost = 0.026f, kMergeCost = 2.0f;
constexpr int kWhole = 1 << 24;          // stages: longer than any context

template <int RW>
constexpr size_t kPieceFloats = 32 * RW * (2 + kHeadDim);

// Row tiles of a sequence and stages of its longest row.
struct RowsShape {
    uint32_t tiles, stages;
    float work;                          // stages of all its tiles together, about
};
template <int RW>
__device__ __forceinline__ RowsShape rows_shape(const PagedSeq& s, const PagedSeqs& seqs, int G, const RowsPlan& plan)
{
    constexpr int ROWS = 32 * RW;
    if (s.count * G < plan.least_rows) return RowsShape{0u, 0u, 0.f};
    const uint32_t tiles = (uint32_t)((s.count * G + ROWS - 1) / ROWS), stages = (uint32_t)((max(s.last(seqs.cap), 0) + ST - 1) / ST);
    return RowsShape{tiles, stages, (float)tiles * fmaxf((float)stages - 0.5f / ST * (float)s.count, 0.f)};      // (causal: half the new tokens less)
}
__device__ __forceinline__ uint32_t pieces_of(uint32_t stages, int P) { return max((stages + P - 1) / P, 1u); }

// A lane's sequences lane * per ...; with one a lane its shape is kept.
template <int RW>
struct RowsWork {
    const PagedSeqs& seqs;
    const RowsPlan& plan;
    int G, per, first;
    RowsShape own;
    __device__ __forceinline__ RowsWork(const PagedSeqs& s, const RowsPlan& p, int g, int lane) : seqs(s), plan(p), G(g), per((s.batch + 63) / 64), first(lane * per), own{0u, 0u, 0.f}
    {
        if (per == 1 && lane < s.batch) own = rows_shape<RW>(paged_seq(s, lane), s, g, p);
    }
    __device__ __forceinline__ RowsShape shape(int b) const { return rows_shape<RW>(paged_seq(seqs, b), seqs, G, plan); }
    // f(shape) of the lane's sequences before `end`, and its sum.
    template <class F>
    __device__ __forceinline__ void each(int end, F f) const
    {
        if (per == 1) {
            if (first < end) f(own);
        } else {
            for (int b = first; b < min(first + per, end); ++b) f(shape(b));
        }
    }
    template <class T, class F>
    __device__ __forceinline__ T sum(int end, F f) const
    {
        T v = T(0);
        each(end, [&](const RowsShape& r) { v += f(r); });
        return v;
    }
};

// Stages of a piece, every wave for itself and all alike: those of one kernel, that is; another compilation of this arithmetic may round otherwise, so the second kernel reads the
// number that the first one left.  Where tiles are many, the mean work of a compute unit, so that only what would outlast the others is cut.  Where they are few, the length of
// least cost; a lane tries one, from half that mean to eight times it, the last lane no cut.  CTAs that fit the chip together take as long as the longest.
// More of them take their work's share and what the last one sticks out, or in whole rounds if they are alike (their mean length near the longest).
template <int RW>
__device__ __forceinline__ int piece_stages(const RowsWork<RW>& w, int heads, const RowsPlan& plan, int lane)
{
    if (plan.target == 0) return kWhole;
    float work = w.template sum<float>(w.seqs.batch, [](const RowsShape& r) { return r.work; });
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) work += __shfl_xor(work, m);
    const float target = (float)plan.target, mean = fminf(work * (float)heads / target, (float)kWhole);
    int best = max((int)mean + 1, kLeastStages);
    if (w.per == 1 && (float)wave_total(w.own.tiles) * (float)heads < 2.f * target) {
        const float tried = lane == 63 ? (float)kWhole : fmaxf(floorf(mean * 0.5f * __builtin_amdgcn_exp2f((float)lane * 0.0625f)), (float)kLeastStages), inv = 1.0f / tried;
        float n = 0.f, cut = 0.f, longest = 0.f;
        for (uint64_t left = __builtin_amdgcn_ballot_w64(w.own.tiles != 0u); left; left &= left - 1) {
            const int b = __builtin_ctzll(left);
            const float stages = (float)__builtin_amdgcn_readlane((int)w.own.stages, b), t = (float)__builtin_amdgcn_readlane((int)w.own.tiles, b);
            const float pieces = fmaxf(ceilf(stages * inv), 1.f);
            n += t * pieces;
            cut += pieces > 1.f ? t * pieces : 0.f;
            longest = fmaxf(longest, stages);
        }
        n *= (float)heads;
        cut *= (float)heads;
        const float cta = fminf(tried, longest) + kCtaCost, rounds = n / target, share = mean + kCtaCost * rounds, alike = mean / (rounds * (cta - kCtaCost));
        float cost = cta;
        if (rounds > 1.f) {
            cost = fmaxf(cta, share + cta * (1.f - 1.f / rounds));
            cost += fmaxf(ceilf(rounds) * cta - cost, 0.f) * fmaxf(fminf(2.f * alike - 1.f, 1.f), 0.f);
        }
        if (cut > 0.f) cost += kMergeCost + kPieceCost * (RW / 8.f) * cut;
        if (cut > (float)plan.slots) cost = 3e38f;
        float least = cost;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) least = fminf(least, __shfl_xor(least, m));
        best = __builtin_amdgcn_readlane((int)tried, __builtin_ctzll(__builtin_amdgcn_ballot_w64(cost == least) | 1ull << 63));
    }
    // The workspace has room for `slots` pieces of cut contexts: a little longer if need be, and never more than twice the mean work.
    best = __builtin_amdgcn_readfirstlane(best);
    const int tries[4] = {best, best + best / 8 + 1, best + best / 2 + 1, max(best, (int)fminf(2.f * work * (float)heads / (float)plan.slots, (float)kWhole) + 1)};
    uint32_t cut[4] = {0u, 0u, 0u, 0u};
    w.each(w.seqs.batch, [&](const RowsShape& r) {
#pragma unroll
        for (int i = 0; i < 4; ++i) cut[i] += r.stages > (uint32_t)tries[i] ? r.tiles * pieces_of(r.stages, tries[i]) : 0u;
    });
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((uint64_t)wave_total(cut[i]) * (uint32_t)heads <= plan.slots) return __builtin_amdgcn_readfirstlane(tries[i]);
    return kWhole;
}

// Piece `unit` of the launch, or with MERGE row tile `unit` of those that are cut: its sequence, first row, context, pieces, and where its pieces' results go.  False: there
// is none, or it has no row to write; the length of the pieces is set all the same.
struct RowsTile {
    PagedSeq s;
    int b, row0, len, stages, pieces, piece, piece_stages;
    uint32_t slot;                       // of piece 0
};
template <int RW, bool MERGE>
__device__ __forceinline__ bool rows_tile(RowsTile& t, const PagedSeqs& seqs, int G, int heads, const RowsPlan& plan, uint32_t unit, int lane)
{
    constexpr int ROWS = 32 * RW;
    const RowsWork<RW> w(seqs, plan, G, lane);
    const int P = MERGE ? constant_load(plan.length, 0) : piece_stages<RW>(w, heads, plan, lane);
    t.piece_stages = P;
    auto units = [&](const RowsShape& r) {
        const uint32_t n = pieces_of(r.stages, P);
        return MERGE ? n > 1 ? r.tiles : 0u : r.tiles * n;
    };
    const SeqFinder finder([&](int b) { return units(w.shape(b)); }, seqs.batch, w.template sum<uint32_t>(seqs.batch, units));
    if (unit >= finder.total) return false;
    uint32_t base;
    t.b = finder.find(unit, base);
    t.s = paged_seq(seqs, t.b);
    const RowsShape r = rows_shape<RW>(t.s, seqs, G, plan);
    const uint32_t most = pieces_of(r.stages, P), at = unit - base, tile = MERGE ? at : at / most;
    if (tile >= r.tiles) return false;
    t.piece = MERGE ? 0 : (int)(at - tile * most);
    t.slot = 0;
    if (most > 1) {
        t.slot = wave_total(w.template sum<uint32_t>(t.b, [&](const RowsShape& o) { return o.stages > (uint32_t)P ? o.tiles * pieces_of(o.stages, P) : 0u; })) + tile * most;
        if (((uint64_t)t.slot + most) * heads > plan.slots) return false;            // (offsets that are out of order)
    }
    t.row0 = (int)(r.tiles - 1 - tile) * ROWS;               // the longest rows first
    const int tok_first = t.row0 / G;
    if (tok_first >= t.s.count || (long)t.s.pos + tok_first >= seqs.cap) return false;
    t.len = (int)min(max((long)t.s.pos + min(t.s.count, (t.row0 + ROWS - 1) / G + 1), 0L), (long)seqs.cap);
    t.stages = (t.len + ST - 1) / ST;
    t.pieces = (int)pieces_of(t.stages, P);
    return t.len > 0 && t.piece < t.pieces;
}

template <int BITS, int RW>
__device__ __forceinline__ void paged_rows(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* __restrict__ Q, long q_stride, uint16_t* __restrict__ O, int q_heads,
                                           float scale_log2e, const RowsPlan& plan, float* __restrict__ partial, uint32_t block, unsigned char* smem)
{
    const uint32_t heads = (uint32_t)pool.heads, hk = block % heads;
    const int G = q_heads / pool.heads;
    RowsTile t;
    const bool any = rows_tile<RW, false>(t, seqs, G, pool.heads, plan, block / heads, threadIdx.x & 63);
    if (block == 0 && threadIdx.x == 0) *plan.length = t.piece_stages;
    if (!any) return;                                        // (uniform)
    const int first = t.piece * t.piece_stages;
    const int stages = t.piece == t.pieces - 1 ? t.stages - first : t.piece_stages;
    float* const part = t.pieces > 1 ? partial + ((size_t)(t.slot + t.piece) * heads + hk) * kPieceFloats<RW> : nullptr;
    const size_t at = (size_t)hk * G * kHeadDim;
    const long o_stride = (long)q_heads * kHeadDim;
    const RowsJob job{Q + t.s.row * q_stride + at, q_stride, O + t.s.row * o_stride + at, o_stride, t.s.count, G, t.row0, seqs.cap, t.s.pos, first, stages, part};
    attn_rows<BITS, RW, true>(job, pool.k, pool.v, pool.pairs, PagedWhere{pool, seqs, t.b, (int)hk}, t.len, scale_log2e, smem);
}

template <int BITS, int RW>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_rows_kernel(PagedPool pool, PagedSeqs seqs, const uint16_t* __restrict__ Q, long q_stride,
                                                                                                    uint16_t* __restrict__ O, int q_heads, float scale_log2e, RowsPlan plan,
                                                                                                    float* __restrict__ partial)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    paged_rows<BITS, RW>(pool, seqs, Q, q_stride, O, q_heads, scale_log2e, plan, partial, blockIdx.x, smem);
}

// Sequences of few rows in the same launch, every wave by itself (tm_paged_columns_impl.h): its first `ctas` CTAs.  They wait for memory where the rows multiply; in a launch of their
// own they would begin when the last row is done.
struct ColumnsPart {
    int most_rows;
    uint32_t ctas;
    float* partial;
    uint32_t* counters;
};
template <int BITS, int RW, bool PACK, int PARTS>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_mixed_kernel(PagedPool pool, PagedSeqs seqs, const uint16_t* __restrict__ Q, long q_stride,
                                                                                                     uint16_t* __restrict__ O, int q_heads, float scale_log2e, RowsPlan plan,
                                                                                                     float* __restrict__ partial, ColumnsPart few)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    if (blockIdx.x < few.ctas)
        paged_columns<BITS, PACK, PARTS, 1, true, 8>(pool, seqs, Q, q_stride, O, q_heads, scale_log2e, few.most_rows, few.partial, few.counters, blockIdx.x, few.ctas);
    else
        paged_rows<BITS, RW>(pool, seqs, Q, q_stride, O, q_heads, scale_log2e, plan, partial, blockIdx.x - few.ctas, smem);
}

// Puts the pieces of rows together: a CTA of 256 threads takes kMergeRows rows, eight at a time, a thread four dimensions of one; kLoads pieces in flight at once.
constexpr int kMergeRows = 16;
template <int RW>
__global__ __launch_bounds__(256) void paged_rows_merge_kernel(int heads, PagedSeqs seqs, uint16_t* __restrict__ O, int q_heads, RowsPlan plan, const float* __restrict__ partial)
{
    constexpr int ROWS = 32 * RW, kLoads = 8;
    const uint32_t chunk = blockIdx.x % (ROWS / kMergeRows), rest = blockIdx.x / (ROWS / kMergeRows), hk = rest % (uint32_t)heads;
    const int G = q_heads / heads;
    RowsTile t;
    if (!rows_tile<RW, true>(t, seqs, G, heads, plan, rest / (uint32_t)heads, threadIdx.x & 63)) return;
    if (t.pieces <= 1) return;                               // written already
    const size_t step = heads * kPieceFloats<RW>;            // from piece to piece
    const float* const base = partial + t.slot * step + hk * kPieceFloats<RW>;
    const int d = 4 * (int)(threadIdx.x & 31);
    for (int r = (int)chunk * kMergeRows + (int)(threadIdx.x >> 5); r < (int)(chunk + 1) * kMergeRows; r += 8) {
        const int row = t.row0 + r, tok = row / G, head = row - tok * G;
        const long pos = (long)t.s.pos + tok;
        if (tok >= t.s.count || pos < 0 || pos >= seqs.cap) continue;
        float M = kMaskFloor, L = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        for (int p0 = 0; p0 < t.pieces; p0 += kLoads) {
            float m[kLoads], l[kLoads];
            f32x4 v[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const float* const p = base + (size_t)(p0 + i < t.pieces ? p0 + i : p0) * step;
                m[i] = p[r];
                l[i] = p[ROWS + r];
                v[i] = *(const f32x4*)(p + 2 * ROWS + r * kHeadDim + d);
            }
            float up = M;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) up = fmaxf(up, m[i]);
            const float old = exp2f(M - up);
            M = up;
            L *= old;
            o *= old;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const float f = p0 + i < t.pieces ? exp2f(m[i] - M) : 0.f;
                L += l[i] * f;
                o += v[i] * f;
            }
        }
        const float inv = L > 0.f ? 1.0f / L : 0.f;
        u32x2 w;
        w.x = (uint32_t)f32_to_f16_bits(o[0] * inv) | ((uint32_t)f32_to_f16_bits(o[1] * inv) << 16);
        w.y = (uint32_t)f32_to_f16_bits(o[2] * inv) | ((uint32_t)f32_to_f16_bits(o[3] * inv) << 16);
        *(u32x2*)(O + ((size_t)(t.s.row + tok) * q_heads + (size_t)hk * G + head) * kHeadDim + d) = w;
    }
}

template <int BITS, int RW, bool PACK, int PARTS>
hipError_t allow_lds_mixed()
{
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_mixed_kernel<BITS, RW, PACK, PARTS>), hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
}
template <int BITS, int RW>
hipError_t allow_lds()
{
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_rows_kernel<BITS, RW>), hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
    if (e == hipSuccess) e = allow_lds_mixed<BITS, RW, true, 1>();
    if (e == hipSuccess) e = allow_lds_mixed<BITS, RW, false, 1>();
    if constexpr (BITS == 4) {
        if (e == hipSuccess) e = allow_lds_mixed<BITS, RW, true, 2>();
        if (e == hipSuccess) e = allow_lds_mixed<BITS, RW, false, 2>();
    }
    return e;
}

template <int BITS, int RW>
hipError_t launch(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, const PagedForm& f, void* workspace,
                  hipStream_t stream)
{
    constexpr int ROWS = 32 * RW;
    char* const space = (char*)workspace + kPagedCounterBytes;
    float* const partial = (float*)(space + kPagedColumnBytes);
    const RowsPlan plan{f.least_rows, f.target, (uint32_t)std::min(kPagedRowBytes / (kPieceFloats<RW> * sizeof(float)), (size_t)f.target * 2),
                        (int32_t*)((char*)workspace + kPagedLengthAt)};
    const unsigned long tiles = (unsigned long)f.items * pool.heads, ctas = tiles + plan.slots, cut = std::min(tiles, (unsigned long)plan.slots / 2);
    const float s = scale * 1.4426950408889634f;
    if (ctas < 1 || ctas + kPagedMostCtas > (unsigned long)most_ctas(512)) return hipErrorInvalidConfiguration;
    if (f.together) {
        const ColumnsPart few{f.column_rows, (uint32_t)f.column_ctas, (float*)space, (uint32_t*)workspace};
        auto pick = [&](auto parts) {
            constexpr int PARTS = decltype(parts)::value;
            return f.columns == 8 ? paged_mixed_kernel<BITS, RW, true, PARTS> : paged_mixed_kernel<BITS, RW, false, PARTS>;
        };
        auto kernel = pick(std::integral_constant<int, 1>{});
        if constexpr (BITS == 4)
            if (pool.run_log == 0) kernel = pick(std::integral_constant<int, 2>{});
        hipLaunchKernelGGL(kernel, dim3((unsigned)(ctas + few.ctas)), dim3(512), kLdsBytes, stream, pool, seqs, Q, q_stride, O, q_heads, s, plan, partial, few);
    } else {
        hipLaunchKernelGGL((paged_rows_kernel<BITS, RW>), dim3((unsigned)ctas), dim3(512), kLdsBytes, stream, pool, seqs, Q, q_stride, O, q_heads, s, plan, partial);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.target == 0) return e;
    hipLaunchKernelGGL((paged_rows_merge_kernel<RW>), dim3((unsigned)(cut * (ROWS / kMergeRows))), dim3(256), 0, stream, pool.heads, seqs, O, q_heads, plan, partial);
    return hipGetLastError();
}

}  // namespace

hipError_t paged_rows_setup()
{
    hipError_t e = allow_lds<8, 8>();
    if (e == hipSuccess) e = allow_lds<8, 4>();
    if (e == hipSuccess) e = allow_lds<4, 8>();
    if (e == hipSuccess) e = allow_lds<4, 4>();
    return e;
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
// 4-bit; contexts from half of the length given): 40 decoding at 4000 and chunks of 1500 and 750 122, 130, 141 and 113, 122, 131; 64 at 4000 and a chunk of 512 at 4000 116, 136, 141 and 113, 108,
// 118; 128 at 1000 and 512 at 2000 86, 93, 104 and 78, 82, 92; 200 at 2000 and a prompt of 256, where the rule takes 11 / 16, 147, 133, 137 and 90, 80, 90.  Short contexts beside tiles of 128 rows
// it does not tell apart, and takes half: 60 at 500 and 400 at 500 23, 30 and 24, 29, but 300 at 300 and a prompt of 64 46, 41, 48 and 37, 31, 43.  Behind the row tiles the columns' long
// pieces stick out: 2 to 8 % more than with half in the first three; on all compute units first 10 to 14 %.
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
    f.columns = most > 64 ? G <= 8 ? 8 : 16 : most <= 8 ? 8 : most <= 16 ? 16 : 32;
    f.column_rows = most <= 64 ? 64 : seqs.batch > 1 ? 16 : 0;
    const long segments = (long)seqs.batch * pool.heads * (most <= 64 ? (most + f.columns - 1) / f.columns : 1);
    const double most_units = ((double)seqs.tokens * G / 8 + seqs.batch) * pool.heads * (seqs.cap / 32 + 3);      // blocks and starts, were every context as long as the table
    f.alone = (pool.bits == 4 ? segments > num_cu : f.columns < 32 && segments >= 4L * num_cu) && most_units < 2147483648.0;      // (counted in 32 bits)
    if (f.alone && f.columns == 32) f.columns = 16;
    const bool twice = pool.bits == 8 && !f.alone && f.columns < 32 && segments > num_cu && max_len > 0 && max_len <= 1024;
    f.column_ctas = std::min(twice ? 2 * num_cu : num_cu, f.alone ? kPagedMostWaves / 4 : kPagedMostCtas);
    if (most <= 64) {
        f.column_rows = 1 << 30;                             // whatever the offsets say
        return f;
    }
    f.least_rows = f.column_rows + 1;
    f.together = f.column_rows && most_units < 2147483648.0;
    const int len = max_len > 0 && max_len < seqs.cap ? max_len : seqs.cap, stages = (len + ST - 1) / ST;
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
    return f;
}

hipError_t launch_paged_attn(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, int max_count, int max_len,
                             int num_cu, void* workspace, hipStream_t stream)
{
    const PagedForm f = paged_form(pool, seqs, q_heads, max_count, max_len, num_cu);
    hipError_t e = hipSuccess;
    if (f.row_waves) {
        if (pool.bits == 8)
            e = f.row_waves == 8 ? launch<8, 8>(pool, seqs, Q, q_stride, O, q_heads, scale, f, workspace, stream) : launch<8, 4>(pool, seqs, Q, q_stride, O, q_heads, scale, f, workspace, stream);
        else
            e = f.row_waves == 8 ? launch<4, 8>(pool, seqs, Q, q_stride, O, q_heads, scale, f, workspace, stream) : launch<4, 4>(pool, seqs, Q, q_stride, O, q_heads, scale, f, workspace, stream);
    }
    if (e == hipSuccess && f.column_rows && !f.together)
        e = launch_paged_columns(pool, seqs, Q, q_stride, O, q_heads, scale, f.columns, f.column_rows, f.column_ctas, f.alone, workspace, stream);
    return e;
}

}  // namespace tmw4
