// Attention of many new tokens per sequence over a paged cache: prompts, chunks of prompts, long drafts (tm_paged_attn).
//
// The kernel is that of prompt attention over the contiguous cache (tm_attn_prefill.hip, tm_attn_rows_impl.h): CTAs of 128 or 256 (token, query head) rows of a KV head,
// codes converted once per CTA.  New here:
//   - Row tiles are numbered over the sequences on the device (tm_paged_device.h), so sequences of any mix of lengths share a launch without a grid for the
//     longest of them.
//   - Where row tiles are too few to fill the chip (a short chunk after a long past) the context is cut into pieces, each a CTA; a second kernel puts a row's pieces together, in
//     their order, so results do not depend on which is done first.
#include "tm_attn_rows_impl.h"
#include "tm_paged_host.h"

namespace tmw4 {

namespace {

struct RowsPlan {
    int least_rows;                      // sequences with fewer rows are not this launch's
    uint32_t items;                      // row tiles the grid has room for
    int pieces, piece_stages;            // pieces of a context at most, stages of 64 tokens each (the last takes what is left)
};

template <int RW>
constexpr size_t kPieceFloats = 32 * RW * (2 + kHeadDim);

// Row tile `item` of the launch: its sequence, first row, context and pieces.  False: there is none, or it has no row to write.
struct RowsTile {
    PagedSeq s;
    int b, row0, len, stages, pieces;
};
template <int RW>
__device__ __forceinline__ bool rows_tile(RowsTile& t, const PagedSeqs& seqs, int G, const RowsPlan& plan, uint32_t item, int lane)
{
    constexpr int ROWS = 32 * RW;
    auto tiles_of = [&](const PagedSeq& s) { return s.count * G < plan.least_rows ? 0u : (uint32_t)((s.count * G + ROWS - 1) / ROWS); };
    const SeqFinder finder([&](int b) { return tiles_of(paged_seq(seqs, b)); }, seqs.batch, lane);
    if (item >= finder.total) return false;
    uint32_t base;
    t.b = finder.find(item, base);
    t.s = paged_seq(seqs, t.b);
    const uint32_t tiles = tiles_of(t.s);
    if (item - base >= tiles) return false;
    t.row0 = (int)(tiles - 1 - (item - base)) * ROWS;        // the longest rows first
    const int tok_first = t.row0 / G;
    if (tok_first >= t.s.count || (long)t.s.pos + tok_first >= seqs.cap) return false;
    t.len = (int)min(max((long)t.s.pos + min(t.s.count, (t.row0 + ROWS - 1) / G + 1), 0L), (long)seqs.cap);
    t.stages = (t.len + ST - 1) / ST;
    t.pieces = min((t.stages + plan.piece_stages - 1) / plan.piece_stages, plan.pieces);
    return t.len > 0;
}

template <int BITS, int RW>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_rows_kernel(PagedPool pool, PagedSeqs seqs, const uint16_t* __restrict__ Q, long q_stride,
                                                                                                    uint16_t* __restrict__ O, int q_heads, float scale_log2e, RowsPlan plan,
                                                                                                    float* __restrict__ partial)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const uint32_t heads = (uint32_t)pool.heads, hk = blockIdx.x % heads, rest = blockIdx.x / heads;
    const uint32_t piece = rest / plan.items, item = rest - piece * plan.items;
    const int G = q_heads / pool.heads;
    RowsTile t;
    if (!rows_tile<RW>(t, seqs, G, plan, item, threadIdx.x & 63)) return;            // (uniform)
    if ((int)piece >= t.pieces) return;
    const int first = (int)piece * plan.piece_stages;
    const int stages = (int)piece == t.pieces - 1 ? t.stages - first : plan.piece_stages;
    float* const part = t.pieces > 1 ? partial + (((size_t)item * heads + hk) * plan.pieces + piece) * kPieceFloats<RW> : nullptr;
    const size_t at = (size_t)hk * G * kHeadDim;
    const long o_stride = (long)q_heads * kHeadDim;
    const RowsJob job{Q + t.s.row * q_stride + at, q_stride, O + t.s.row * o_stride + at, o_stride, t.s.count, G, t.row0, seqs.cap, t.s.pos, first, stages, part};
    attn_rows<BITS, RW, true>(job, pool.k, pool.v, pool.pairs, PagedWhere{pool, seqs, t.b, (int)hk}, t.len, scale_log2e, smem);
}

// Puts the pieces of rows together: a CTA of 256 threads takes eight rows, a thread four dimensions of one; kLoads pieces in flight at once.
template <int RW>
__global__ __launch_bounds__(256) void paged_rows_merge_kernel(int heads, PagedSeqs seqs, uint16_t* __restrict__ O, int q_heads, RowsPlan plan, const float* __restrict__ partial)
{
    constexpr int ROWS = 32 * RW, kLoads = 8;
    const uint32_t chunk = blockIdx.x % (ROWS / 8), rest = blockIdx.x / (ROWS / 8), hk = rest % (uint32_t)heads, item = rest / (uint32_t)heads;
    const int G = q_heads / heads;
    RowsTile t;
    if (!rows_tile<RW>(t, seqs, G, plan, item, threadIdx.x & 63)) return;
    if (t.pieces <= 1) return;                               // written already
    const int r = (int)chunk * 8 + (int)(threadIdx.x >> 5), d = 4 * (int)(threadIdx.x & 31);
    const int row = t.row0 + r, tok = row / G, head = row - tok * G;
    const long pos = (long)t.s.pos + tok;
    if (tok >= t.s.count || pos < 0 || pos >= seqs.cap) return;
    const float* const base = partial + ((size_t)item * heads + hk) * plan.pieces * kPieceFloats<RW>;
    float M = kMaskFloor, L = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < t.pieces; p0 += kLoads) {
        float m[kLoads], l[kLoads];
        f32x4 v[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const float* const p = base + (size_t)(p0 + i < t.pieces ? p0 + i : p0) * kPieceFloats<RW>;
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

template <int BITS, int RW>
hipError_t launch(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, const RowsPlan& plan, float* partial,
                  hipStream_t stream)
{
    const unsigned long tiles = (unsigned long)plan.items * pool.heads, ctas = tiles * plan.pieces;
    if (ctas < 1 || ctas > 0x7fffffffUL || tiles * (32 * RW / 8) > 0x7fffffffUL) return hipErrorInvalidValue;
    if (plan.pieces > 1 && ctas * kPieceFloats<RW> * sizeof(float) > kPagedPartialBytes) return hipErrorInvalidValue;
    hipLaunchKernelGGL((paged_rows_kernel<BITS, RW>), dim3((unsigned)ctas), dim3(512), kLdsBytes, stream, pool, seqs, Q, q_stride, O, q_heads, scale * 1.4426950408889634f, plan,
                       partial);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.pieces == 1) return e;
    hipLaunchKernelGGL((paged_rows_merge_kernel<RW>), dim3((unsigned)(tiles * (32 * RW / 8))), dim3(256), 0, stream, pool.heads, seqs, O, q_heads, plan, partial);
    return hipGetLastError();
}

template <int BITS, int RW>
hipError_t allow_lds()
{
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_rows_kernel<BITS, RW>), hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
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

PagedForm paged_form(const PagedPool& pool, const PagedSeqs& seqs, int q_heads, int max_count, int max_len, int num_cu)
{
    const int G = q_heads / pool.heads;
    PagedForm f{};
    const long most = (long)(max_count > 0 && max_count < seqs.tokens ? max_count : seqs.tokens) * G;
    f.columns = most > 64 ? G <= 8 ? 8 : 16 : most <= 8 ? 8 : most <= 16 ? 16 : 32;
    f.column_rows = most <= 64 ? 64 : seqs.batch > 1 ? 16 : 0;
    f.column_ctas = num_cu < kPagedMostCtas ? num_cu : kPagedMostCtas;
    if (most <= 64) {
        f.column_rows = 1 << 30;                             // whatever the offsets say
        return f;
    }
    f.least_rows = f.column_rows + 1;
    const int len = max_len > 0 && max_len < seqs.cap ? max_len : seqs.cap, stages = (len + ST - 1) / ST;
    double best = 0.0;
    for (int rw = 4; rw <= 8; rw += 4) {
        const long rows = (long)seqs.tokens * G, big = rows / f.least_rows < seqs.batch ? rows / f.least_rows : seqs.batch;
        const long items = rows / (32 * rw) + big + 1, ctas = items * pool.heads;
        const size_t piece_bytes = (size_t)(32 * rw) * (2 + kHeadDim) * sizeof(float);
        long pieces = ctas < num_cu ? num_cu / ctas : 1;
        if (pieces > stages / 4) pieces = stages / 4;
        if (pieces > 32) pieces = 32;
        if (pieces > (long)(kPagedPartialBytes / piece_bytes) / ctas) pieces = (long)(kPagedPartialBytes / piece_bytes) / ctas;
        if (pieces < 1) pieces = 1;
        const double rounds = (double)ctas * pieces / num_cu;
        const double t = (rw == 4 ? 2.4 : 3.85) * (rounds < 1.0 ? 1.0 : rounds) / pieces;
        if (rw == 4 || t < best) {
            best = t;
            f.row_waves = rw;
            f.items = (uint32_t)items;
            f.pieces = (int)pieces;
            f.piece_stages = (int)((stages + pieces - 1) / pieces);
        }
    }
    return f;
}

hipError_t launch_paged_attn(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* Q, long q_stride, uint16_t* O, int q_heads, float scale, int max_count, int max_len,
                             int num_cu, void* workspace, hipStream_t stream)
{
    const PagedForm f = paged_form(pool, seqs, q_heads, max_count, max_len, num_cu);
    hipError_t e = hipSuccess;
    if (f.row_waves) {
        const RowsPlan plan{f.least_rows, f.items, f.pieces, f.piece_stages};
        float* const partial = (float*)((char*)workspace + kPagedCounterBytes);
        if (pool.bits == 8)
            e = f.row_waves == 8 ? launch<8, 8>(pool, seqs, Q, q_stride, O, q_heads, scale, plan, partial, stream)
                                 : launch<8, 4>(pool, seqs, Q, q_stride, O, q_heads, scale, plan, partial, stream);
        else
            e = f.row_waves == 8 ? launch<4, 8>(pool, seqs, Q, q_stride, O, q_heads, scale, plan, partial, stream)
                                 : launch<4, 4>(pool, seqs, Q, q_stride, O, q_heads, scale, plan, partial, stream);
    }
    if (e == hipSuccess && f.column_rows)
        e = launch_paged_columns(pool, seqs, Q, q_stride, O, q_heads, scale, f.columns, f.column_rows, f.column_ctas, workspace, stream);
    return e;
}

}  // namespace tmw4
