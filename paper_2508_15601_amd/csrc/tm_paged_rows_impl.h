// The kernels of many rows per sequence over pages; tm_paged_rows.hip, which describes them, and tm_paged_rows_window.hip build them.
#pragma once
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
// WINDOW: of the stages that are left, and no tile has more than `seen` of those.
template <int RW, bool WINDOW>
__device__ __forceinline__ RowsShape rows_shape(const PagedSeq& s, const PagedSeqs& seqs, int G, const RowsPlan& plan)
{
    constexpr int ROWS = 32 * RW;
    if (s.count * G < plan.least_rows) return RowsShape{0u, 0u, 0.f};
    const uint32_t tiles = (uint32_t)((s.count * G + ROWS - 1) / ROWS), stages = (uint32_t)((max(s.last(seqs.cap), 0) + ST - 1) / ST);
    const float causal = fmaxf((float)stages - 0.5f / ST * (float)s.count, 0.f);     // (half the new tokens less)
    if constexpr (WINDOW) {
        const uint32_t seen = (uint32_t)(((seqs.window + ROWS / G + 1) / kRun + 2 + (seqs.sinks + kRun - 1) / kRun + 1) / 2);
        return RowsShape{tiles, min(stages, seen), (float)tiles * fminf(causal, (float)seen)};
    }
    return RowsShape{tiles, stages, (float)tiles * causal};
}
__device__ __forceinline__ uint32_t pieces_of(uint32_t stages, int P) { return max((stages + P - 1) / P, 1u); }

// A lane's sequences lane * per ...; with one a lane its shape is kept.
template <int RW, bool WINDOW>
struct RowsWork {
    const PagedSeqs& seqs;
    const RowsPlan& plan;
    int G, per, first;
    RowsShape own;
    __device__ __forceinline__ RowsWork(const PagedSeqs& s, const RowsPlan& p, int g, int lane) : seqs(s), plan(p), G(g), per((s.batch + 63) / 64), first(lane * per), own{0u, 0u, 0.f}
    {
        if (per == 1 && lane < s.batch) own = rows_shape<RW, WINDOW>(paged_seq(s, lane), s, g, p);
    }
    __device__ __forceinline__ RowsShape shape(int b) const { return rows_shape<RW, WINDOW>(paged_seq(seqs, b), seqs, G, plan); }
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
template <int RW, bool WINDOW>
__device__ __forceinline__ int piece_stages(const RowsWork<RW, WINDOW>& w, int heads, const RowsPlan& plan, int lane)
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
template <int RW, bool WINDOW, bool MERGE>
__device__ __forceinline__ bool rows_tile(RowsTile& t, const PagedSeqs& seqs, int G, int heads, const RowsPlan& plan, uint32_t unit, int lane)
{
    constexpr int ROWS = 32 * RW;
    const RowsWork<RW, WINDOW> w(seqs, plan, G, lane);
    const int P = MERGE ? constant_load(plan.length, 0) : piece_stages<RW, WINDOW>(w, heads, plan, lane);
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
    const RowsShape r = rows_shape<RW, WINDOW>(t.s, seqs, G, plan);
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
    if constexpr (WINDOW) t.stages = ((t.len + kRun - 1) / kRun - Hidden(seqs, (int)min(max((long)t.s.pos + tok_first, 0L), (long)seqs.cap), kRun).count + 1) / 2;
    t.pieces = (int)pieces_of(t.stages, P);
    return t.len > 0 && t.piece < t.pieces;
}

template <int BITS, int RW, bool WINDOW>
__device__ __forceinline__ void paged_rows(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* __restrict__ Q, long q_stride, uint16_t* __restrict__ O, int q_heads,
                                           float scale_log2e, const RowsPlan& plan, float* __restrict__ partial, uint32_t block, unsigned char* smem)
{
    const uint32_t heads = (uint32_t)pool.heads, hk = block % heads;
    const int G = q_heads / pool.heads;
    RowsTile t;
    const bool any = rows_tile<RW, WINDOW, false>(t, seqs, G, pool.heads, plan, block / heads, threadIdx.x & 63);
    if (block == 0 && threadIdx.x == 0) *plan.length = t.piece_stages;
    if (!any) return;                                        // (uniform)
    const int first = t.piece * t.piece_stages;
    const int stages = t.piece == t.pieces - 1 ? t.stages - first : t.piece_stages;
    float* const part = t.pieces > 1 ? partial + ((size_t)(t.slot + t.piece) * heads + hk) * kPieceFloats<RW> : nullptr;
    const size_t at = (size_t)hk * G * kHeadDim;
    const long o_stride = (long)q_heads * kHeadDim;
    const RowsJob job{Q + t.s.row * q_stride + at, q_stride, O + t.s.row * o_stride + at, o_stride, t.s.count, G, t.row0, seqs.cap, t.s.pos, first, stages, part};
    attn_rows<BITS, RW, true, WINDOW>(job, pool.k, pool.v, pool.pairs, PagedWhere{pool, seqs, t.b, (int)hk}, t.len, scale_log2e, smem);
}

template <int BITS, int RW, bool WINDOW>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_rows_kernel(PagedPool pool, PagedSeqs seqs, const uint16_t* __restrict__ Q, long q_stride,
                                                                                                    uint16_t* __restrict__ O, int q_heads, float scale_log2e, RowsPlan plan,
                                                                                                    float* __restrict__ partial)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    paged_rows<BITS, RW, WINDOW>(pool, seqs, Q, q_stride, O, q_heads, scale_log2e, plan, partial, blockIdx.x, smem);
}

// Sequences of few rows in the same launch, every wave by itself (tm_paged_columns_impl.h): its first `ctas` CTAs.  They wait for memory where the rows multiply; in a launch of their
// own they would begin when the last row is done.
struct ColumnsPart {
    int most_rows;
    uint32_t ctas;
    float* partial;
    uint32_t* counters;
};
template <int BITS, int RW, bool PACK, int PARTS, bool WINDOW>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_mixed_kernel(PagedPool pool, PagedSeqs seqs, const uint16_t* __restrict__ Q, long q_stride,
                                                                                                     uint16_t* __restrict__ O, int q_heads, float scale_log2e, RowsPlan plan,
                                                                                                     float* __restrict__ partial, ColumnsPart few)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    if (blockIdx.x < few.ctas)
        paged_columns<BITS, PACK, PARTS, 1, true, 8, WINDOW>(pool, seqs, Q, q_stride, O, q_heads, scale_log2e, few.most_rows, few.partial, few.counters, blockIdx.x, few.ctas);
    else
        paged_rows<BITS, RW, WINDOW>(pool, seqs, Q, q_stride, O, q_heads, scale_log2e, plan, partial, blockIdx.x - few.ctas, smem);
}

// Puts the pieces of rows together: a CTA of 256 threads takes kMergeRows rows, eight at a time, a thread four dimensions of one; kLoads pieces in flight at once.
constexpr int kMergeRows = 16;
template <int RW, bool WINDOW>
__global__ __launch_bounds__(256) void paged_rows_merge_kernel(int heads, PagedSeqs seqs, uint16_t* __restrict__ O, int q_heads, RowsPlan plan, const float* __restrict__ partial)
{
    constexpr int ROWS = 32 * RW, kLoads = 8;
    const uint32_t chunk = blockIdx.x % (ROWS / kMergeRows), rest = blockIdx.x / (ROWS / kMergeRows), hk = rest % (uint32_t)heads;
    const int G = q_heads / heads;
    RowsTile t;
    if (!rows_tile<RW, WINDOW, true>(t, seqs, G, heads, plan, rest / (uint32_t)heads, threadIdx.x & 63)) return;
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

template <int BITS, int RW, bool PACK, int PARTS, bool WINDOW>
hipError_t allow_lds_mixed()
{
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_mixed_kernel<BITS, RW, PACK, PARTS, WINDOW>), hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
}
template <int BITS, int RW, bool WINDOW>
hipError_t allow_lds()
{
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_rows_kernel<BITS, RW, WINDOW>), hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
    if (e == hipSuccess) e = allow_lds_mixed<BITS, RW, true, 1, WINDOW>();
    if (e == hipSuccess) e = allow_lds_mixed<BITS, RW, false, 1, WINDOW>();
    if constexpr (BITS == 4) {
        if (e == hipSuccess) e = allow_lds_mixed<BITS, RW, true, 2, WINDOW>();
        if (e == hipSuccess) e = allow_lds_mixed<BITS, RW, false, 2, WINDOW>();
    }
    return e;
}

template <int BITS, int RW, bool WINDOW>
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
            return f.columns == 8 ? paged_mixed_kernel<BITS, RW, true, PARTS, WINDOW> : paged_mixed_kernel<BITS, RW, false, PARTS, WINDOW>;
        };
        auto kernel = pick(std::integral_constant<int, 1>{});
        if constexpr (BITS == 4)
            if (pool.run_log == 0) kernel = pick(std::integral_constant<int, 2>{});
        hipLaunchKernelGGL(kernel, dim3((unsigned)(ctas + few.ctas)), dim3(512), kLdsBytes, stream, pool, seqs, Q, q_stride, O, q_heads, s, plan, partial, few);
    } else {
        hipLaunchKernelGGL((paged_rows_kernel<BITS, RW, WINDOW>), dim3((unsigned)ctas), dim3(512), kLdsBytes, stream, pool, seqs, Q, q_stride, O, q_heads, s, plan, partial);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.target == 0) return e;
    hipLaunchKernelGGL((paged_rows_merge_kernel<RW, WINDOW>), dim3((unsigned)(cut * (ROWS / kMergeRows))), dim3(256), 0, stream, pool.heads, seqs, O, q_heads, plan, partial);
    return hipGetLastError();
}

template <bool WINDOW>
hipError_t setup()
{
    hipError_t e = allow_lds<8, 8, WINDOW>();
    if (e == hipSuccess) e = allow_lds<8, 4, WINDOW>();
    if (e == hipSuccess) e = allow_lds<4, 8, WINDOW>();
    if (e == hipSuccess) e = allow_lds<4, 4, WINDOW>();
    return e;
}

template <bool WINDOW>
hipError_t launch_rows_of(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, const PagedForm& f, void* workspace,
                          hipStream_t stream)
{
    const auto run = pool.bits == 8 ? f.row_waves == 8 ? launch<8, 8, WINDOW> : launch<8, 4, WINDOW> : f.row_waves == 8 ? launch<4, 8, WINDOW> : launch<4, 4, WINDOW>;
    return run(pool, seqs, Q, q_stride, O, q_heads, scale, f, workspace, stream);
}

}  // namespace

}  // namespace tmw4
