// The kernel of prompt attention over a quantised cache; tm_attn_prefill.hip (contiguous cache, which describes it) and tm_paged_rows.hip (paged cache) build it.
#pragma once
#include "tm_attn_device.h"
#include "tm_paged_device.h"

namespace tmw4 {

namespace {

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

constexpr int ST = 64;                           // tokens per stage
constexpr int kStageBytes = ST * kHeadDim * 2;   // one stage of keys (or values) in fp16
constexpr int kStagePairs = ST * 10;             // one stage of scales and zero-points
// Keys are read one stage ahead of the barrier that ends it, values after it: two key buffers, three value buffers, and
// four sets of pairs (read from the conversion of a stage to its last product).
constexpr int kLdsBytes = 5 * kStageBytes + 4 * kStagePairs;

// A CTA's rows and context.  Paged cache: where a run of 32 tokens lies is asked for run by run, the context may be cut into pieces (first_stage, stages), and a run on
// a page that the pool does not have is not read and its tokens are masked.
struct RowsJob {
    const uint16_t* q;                                     // row 0 of the sequence (KV head included), and values from token to token
    long q_stride;
    uint16_t* o;
    long o_stride;
    int cnt, G, row0, cap;                                 // tokens of the sequence, query heads a token has here, first row
    long pos0;                                             // position of its first token
    int first_stage, stages;                               // of the context: stages of ST tokens to attend over
    float* partial;                                        // where the results of a piece go, nullptr: the piece is the whole context
};
struct PagedWhere {
    PagedPool pool;
    PagedSeqs seqs;
    int b, hk;
};

// WINDOW (paged): a row attends over the first tokens and those of its window; runs that no row of the CTA sees are left out (`hidden`), a stage is two of those that are left, and
// job.first_stage and job.stages count such stages.
template <int BITS, int RW, bool PAGED, bool WINDOW = false>
__device__ __forceinline__ void attn_rows(const RowsJob& job, const uint8_t* kcodes, const uint8_t* vcodes, const uint32_t* words, const PagedWhere& where, int len_all,
                                          float scale_log2e, unsigned char* smem)
{
    constexpr int KS = 8 / RW;                             // wave groups along the context
    constexpr int NB = 2 / KS;                             // 32-token runs per wave and stage
    unsigned char* const kbase = smem;
    unsigned char* const vbase = smem + 2 * kStageBytes;
    unsigned char* const pbase = vbase + 3 * kStageBytes;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rg = wave % RW, ksg = wave / RW;
    const int hl = lane >> 5;
    const int cnt = job.cnt, G = job.G, row0 = job.row0;
    const long pos0 = job.pos0;
    const int tok_first = row0 / G;
    const int nst = job.stages;
    const int tok0 = PAGED && !WINDOW ? job.first_stage * ST : 0;      // first token of the piece
    const int sinks = WINDOW ? where.seqs.sinks : 0, tile_first = WINDOW ? (int)min(max(pos0 + tok_first, 0L), (long)job.cap) : 0;
    const Hidden hidden(where.seqs, tile_first, kRun);
    auto run_of = [&](int st, int n) { return WINDOW ? hidden.real(2 * (job.first_stage + st) + n) : (tok0 >> 5) + 2 * st + n; };      // of the sequence

    // this wave's rows, and this lane's
    const int w0 = row0 + rg * 32;
    const int wtok = w0 / G;
    int wlen = (int)min(max(pos0 + min(cnt, (w0 + 31) / G + 1), 0L), (long)job.cap);  // tokens its longest row attends over
    if (wtok >= cnt) wlen = 0;
    const long wmin = pos0 + wtok + 1;                                              // and its shortest
    const int row = w0 + (lane & 31);
    int tok = row / G;
    const int head = row - tok * G;
    const long pos = pos0 + tok;
    const bool real = tok < cnt && pos >= 0 && pos < job.cap;
    const int len = real ? (int)pos + 1 : 0;
    const int lo = WINDOW ? len - where.seqs.window : 0, most_lo = WINDOW ? wlen - where.seqs.window : 0;      // the row's window begins there, the wave's last one
    if (!real) tok = tok_first;                                                     // an address that exists
    const uint16_t* const qrow = job.q + tok * job.q_stride + head * kHeadDim;

    f16x8 qf[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) qf[t] = *(const f16x8*)(qrow + 16 * t + 8 * hl);

    // ---- staging: codes in registers one stage ahead of their conversion, scale/zero pairs two
    constexpr int kCodeBytes = kHeadDim * BITS / 8;                                 // of one token
    constexpr int kRunBytes = kRun * kCodeBytes;
    const uint32_t code_end = (uint32_t)(len_all + 31) / 32 * 32 * kCodeBytes;
    const __amdgpu_buffer_rsrc_t krs = make_rsrc(kcodes, code_end);
    const __amdgpu_buffer_rsrc_t vrs = make_rsrc(vcodes, code_end);
    const __amdgpu_buffer_rsrc_t zrs = make_rsrc(words, (uint32_t)len_all * 8u);    // zeros past the context
    u32x4 codes[BITS == 8 ? 2 : 1];                                                 // 16-byte chunks of a thread and stage
    u32x2 pairs = {0u, 0u};
    // Paged: numbers in the pool of a stage's two runs, -1 where there is none; the run whose codes this wave stages is `mine`.  (A pool of 2^31 runs would take 4 TB.)
    struct StageRuns {
        int at[2];
    };
    constexpr int kChunks = BITS == 8 ? 256 : 128;                                  // of 16 bytes a run
    const int mine = (BITS == 8 ? wave >> 2 : wave >> 1) & 1;
    // The table's entries are scalar loads, requested a stage before they are looked at: as vector loads they would stand in line with the codes and pairs, and a wait for them would be
    // one for those.  Scalar loads share their counter with LDS, out of order, so a wait for LDS is one for them: they go out with the stage's first products, from where the compiler moves
    // them in front of the barrier, at which waves wait for each other anyway.  In front of the products every stage's first one waited for them (4-bit: four prompts 820 us, like this 797; chunks of
    // 1500 and 750 92.1 and 88.5, 90.5 as vector loads).
    struct StageEntries {
        int id[2];
    };
    const int last_run = max(len_all - 1, 0) / kRun;
    auto entries_of = [&](int st) {
        StageEntries e{{-1, -1}};
        if constexpr (PAGED) {
#pragma unroll
            for (int n = 0; n < 2; ++n) e.id[n] = paged_entry(where.pool, where.seqs, where.b, min(run_of(st, n), last_run));
        }
        return e;
    };
    auto runs_of = [&](int st, const StageEntries& e) {
        StageRuns r{{-1, -1}};
        if constexpr (PAGED) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int run = run_of(st, n);
                if (run <= last_run && (uint32_t)e.id[n] < (uint32_t)where.pool.pages) r.at[n] = (int)paged_run(where.pool, e.id[n], where.hk, run);
            }
        }
        return r;
    };
    // which runs of stages st, st + 1, ... are there: bits 2 * (st & 3), 2 * (st & 3) + 1 of `present`
    uint32_t present = ~0u;
    auto note = [&](int st, const StageRuns& r) {
        if constexpr (PAGED) {
            const int sh = 2 * (st & 3);
            present = (present & ~(3u << sh)) | ((uint32_t)(r.at[0] >= 0) << sh) | ((uint32_t)(r.at[1] >= 0) << (sh + 1));
        }
    };
    auto load_codes = [&](int st, const StageRuns& r) {
        if constexpr (PAGED) {
            const int run = mine ? r.at[1] : r.at[0];
            const uint32_t bytes = run >= 0 ? kRunBytes : 0u;
            const size_t at = (size_t)(run >= 0 ? run : 0) * kRunBytes;
            const int off = (tid & (kChunks - 1)) * 16;
            if constexpr (BITS == 8) {
                codes[0] = __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(kcodes + at, bytes), off, 0, 0);
                codes[1] = __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(vcodes + at, bytes), off, 0, 0);
            } else {
                codes[0] = __builtin_amdgcn_raw_buffer_load_b128(make_rsrc((wave < 4 ? kcodes : vcodes) + at, bytes), off, 0, 0);
            }
            (void)st;
        } else if constexpr (BITS == 8) {
            codes[0] = __builtin_amdgcn_raw_buffer_load_b128(krs, st * (ST * 128) + tid * 16, 0, 0);
            codes[1] = __builtin_amdgcn_raw_buffer_load_b128(vrs, st * (ST * 128) + tid * 16, 0, 0);
        } else {                                           // half the waves take the keys, half the values
            codes[0] = wave < 4 ? __builtin_amdgcn_raw_buffer_load_b128(krs, st * (ST * 64) + tid * 16, 0, 0)
                                : __builtin_amdgcn_raw_buffer_load_b128(vrs, st * (ST * 64) + (tid - 256) * 16, 0, 0);
        }
    };
    auto load_pairs = [&](int st, const StageRuns& r) {
        if constexpr (PAGED) {
            if (tid < ST)                                  // wave 0: lanes 0 .. 31 the first run.  What stands in for a run that is not there (the pool's first) is masked.
                pairs = *(const u32x2*)(words + ((size_t)(uint32_t)max(tid < kRun ? r.at[0] : r.at[1], 0) * kRun + (tid & (kRun - 1))) * 2);
            (void)st;
        } else {
            if (tid < ST) pairs = __builtin_amdgcn_raw_buffer_load_b64(zrs, (st * ST + tid) * 8, 0, 0);
        }
    };
    // LDS image of a stage's pairs: [ST] K scales times scale * log2(e) in fp32 (in the query's fp16 values the factor's rounding
    // would be a fifth of the result's error), then [ST] V scales, [ST] K zero-points, [ST] V zero-points (fp16).
    // A token that was never stored may hold anything; its scores are masked, and with finite numbers here its values
    // cannot reach a sum (0 * q).
    auto store_pairs = [&](int st) {
        if (tid < ST) {
            unsigned char* const p = pbase + (st & 3) * kStagePairs;
            const f16x2 k = as_f16x2(pairs.x), v = as_f16x2(pairs.y);
            const _Float16 top = BITS == 8 ? (_Float16)255.0f : (_Float16)15.0f, nul = (_Float16)0.0f;
            const _Float16 vs = v.x < (_Float16)65504.0f && v.x > (_Float16)-65504.0f ? v.x : nul;
            const _Float16 kz = __builtin_fminf16(__builtin_fmaxf16(k.y, nul), top);
            const _Float16 vz = __builtin_fminf16(__builtin_fmaxf16(v.y, nul), top);
            ((float*)p)[tid] = (float)k.x * scale_log2e;
            ((_Float16*)(p + ST * 4))[tid] = vs;
            ((_Float16*)(p + ST * 6))[tid] = kz;
            ((_Float16*)(p + ST * 8))[tid] = vz;
        }
    };
    const Magic mg = make_magic();
    // one 16-byte chunk of the cache -> fp16 fragments (32 bytes of 8-bit codes, 64 of 4-bit ones)
    auto convert_k = [&](int id, const u32x4& w, unsigned char* kb, const unsigned char* zk) {
        constexpr int CPB = BITS == 8 ? 256 : 128;                                  // chunks per 32 tokens
        const int blk = id / CPB, chunk = id % CPB;
        const int c = chunk & 15, hh = (chunk >> 4) & 3, j = BITS == 8 ? chunk >> 7 : chunk >> 6;
        const int r = 16 * (c >> 3) + 8 * j + (c & 7);                              // operand row of token 16j + c
        const _Float16 z = ((const _Float16*)zk)[blk * 32 + 16 * j + c];
        const _Float16 a = (_Float16)-1024.0f - z;
        const f16x2 hi = {a, a};
        unsigned char* const dst = kb + blk * 8192 + r * 16;
        if constexpr (BITS == 8) {
            const int t = 2 * hh + ((chunk >> 6) & 1);
            *(f16x8*)(dst + t * 1024) = add_pairs(biased8_w8(w.x, w.y), hi, hi, hi, hi);
            *(f16x8*)(dst + t * 1024 + 512) = add_pairs(biased8_w8(w.z, w.w), hi, hi, hi, hi);
        } else {
            const _Float16 e = (_Float16)-64.0f - z;
            const f16x2 lo = {e, e};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(f16x8*)(dst + (2 * hh + (i >> 1)) * 1024 + (i & 1) * 512) = add_pairs(biased8(w[i], mg), hi, lo, hi, lo);
        }
    };
    auto convert_v = [&](int id, const u32x4& w, unsigned char* vb, const unsigned char* zv) {
        constexpr int CPB = BITS == 8 ? 256 : 128;
        const int blk = id / CPB, chunk = id % CPB;
        const int c = chunk & 15, hh = (chunk >> 4) & 3, ii = chunk >> 6;
        // the chunk's tokens: 4hh .. 4hh + 3 and 16 + 4hh .. 16 + 4hh + 3
        const u32x2 z0 = *(const u32x2*)(zv + (blk * 32 + 4 * hh) * 2), z1 = *(const u32x2*)(zv + (blk * 32 + 16 + 4 * hh) * 2);
        const f16x2 b1024 = {(_Float16)-1024.0f, (_Float16)-1024.0f};
        const f16x2 blo = BITS == 8 ? b1024 : f16x2{(_Float16)-64.0f, (_Float16)-64.0f};
        const f16x2 p0 = b1024 - as_f16x2(z0.x), p1 = blo - as_f16x2(z0.y), p2 = b1024 - as_f16x2(z1.x), p3 = blo - as_f16x2(z1.y);
        unsigned char* const dst = vb + blk * 8192 + (hh >> 1) * 1024 + (hh & 1) * 512 + c * 16;
        if constexpr (BITS == 8) {
            *(f16x8*)(dst + ii * 2048) = add_pairs(biased8_w8(w.x, w.y), p0, p1, p2, p3);
            *(f16x8*)(dst + ii * 2048 + 256) = add_pairs(biased8_w8(w.z, w.w), p0, p1, p2, p3);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(f16x8*)(dst + (2 * ii + (i >> 1)) * 2048 + (i & 1) * 256) = add_pairs(biased8(w[i], mg), p0, p1, p2, p3);
        }
    };
    auto convert_stage = [&](int st) {
        unsigned char* const kb = kbase + (st & 1) * kStageBytes;
        unsigned char* const vb = vbase + (st % 3) * kStageBytes;
        const unsigned char* const zk = pbase + (st & 3) * kStagePairs + ST * 6;
        const unsigned char* const zv = zk + ST * 2;
        if constexpr (BITS == 8) {
            convert_k(tid, codes[0], kb, zk);
            convert_v(tid, codes[1], vb, zv);
        } else if (wave < 4) {
            convert_k(tid, codes[0], kb, zk);
        } else {
            convert_v(tid - 256, codes[0], vb, zv);
        }
    };
    auto barrier = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                          // LDS only: loads stay in flight
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    StageEntries next = entries_of(2), after = entries_of(3);
    StageRuns run0 = runs_of(0, entries_of(0)), run1 = runs_of(1, entries_of(1));      // of the stages whose codes and pairs are requested next
    note(0, run0);
    note(1, run1);
    load_codes(0, run0);
    load_pairs(0, run0);
    store_pairs(0);
    load_pairs(1, run1);
    store_pairs(1);
    run0 = runs_of(2, next);
    note(2, run0);
    load_pairs(2, run0);
    barrier();
    convert_stage(0);
    load_codes(1, run1);
    run1 = runs_of(3, after);
    next = entries_of(4);

#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) qf[t][e] = real ? qf[t][e] : (_Float16)0.0f;
    barrier();

    f32x16 o[4];
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float m_run = kMaskFloor, l_run = 0.f;
    f32x16 x;                                              // the current 32 tokens' scores, less the reference
    f32x4 ks[4];                                           // their keys' scales
    u32x2 vs[4];                                           // and their values' (fp16)
    float mx;

    // raw scores of the 32 tokens whose keys start at kb
    auto multiply_k = [&](const unsigned char* kb) -> f32x16 {
        f32x16 s;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int t = 0; t < 8; ++t) s = mfma32x32x16(*(const f16x8*)(kb + t * 1024 + lane * 16), qf[t], s);
        return s;
    };
    // scales of the lane's tokens: element i of register g is token {0, 16, 8, 24}[g] + 4 * hl + i of the run
    auto read_scales = [&](const unsigned char* p, int run) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int token = run * 32 + (g & 1) * 16 + (g >> 1) * 8 + 4 * hl;
            ks[g] = *(const f32x4*)(p + token * 4);
            vs[g] = *(const u32x2*)(p + ST * 4 + token * 2);
        }
    };
    // x = s * scale - ref; masked: tokens from the row's length on get kNegBig.  t0: first of the 32 tokens
    auto scale_scores = [&](const f32x16& s, float ref, bool masked, int t0, bool there) {
        const int rem = !PAGED || there ? len - t0 - 4 * hl : -1;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = __builtin_fmaf(s[e], ks[e >> 2][e & 3], -ref);
        if (masked) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int at = ((e >> 2) & 1) * 16 + (e >> 3) * 8 + (e & 3);
                bool live = at < rem;
                if constexpr (WINDOW) live = live && (at + t0 + 4 * hl >= lo || at + t0 + 4 * hl < sinks);
                x[e] = live ? x[e] : kNegBig;
            }
        }
        mx = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
    };
    auto first_token = [&](int st, int sub) { return WINDOW ? run_of(st, KS > 1 ? ksg : sub) * kRun : tok0 + st * ST + (KS > 1 ? ksg : sub) * 32; };
    auto at_edge = [&](int t0) { return t0 + 32 > wmin || (WINDOW && t0 < most_lo && t0 + 32 > sinks); };           // not every row sees all 32
    auto is_there = [&](int st, int sub) { return !PAGED || (present >> (2 * (st & 3) + (KS > 1 ? ksg : sub)) & 1u); };

    {
        const int t0 = first_token(0, 0);
        const f32x16 s = multiply_k(kbase + (KS > 1 ? ksg : 0) * 8192);
        read_scales(pbase, KS > 1 ? ksg : 0);
        scale_scores(s, 0.f, true, t0, is_there(0, 0));
        m_run = fmaxf(fmaxf(mx, other_half(mx)), kMaskFloor);
        scale_scores(s, m_run, true, t0, is_there(0, 0));
    }

    for (int st = 0; st < nst; ++st) {
        convert_stage(st + 1);
        store_pairs(st + 2);
        load_codes(st + 2, run0);
        load_pairs(st + 3, run1);
        if constexpr (PAGED) {
            run0 = run1;
            note(st + 3, run0);                            // (stage st - 1 has been scored)
            run1 = runs_of(st + 4, next);
        }
#pragma unroll
        for (int sub = 0; sub < NB; ++sub) {
            const int t0 = first_token(st, sub);
            const int st_n = sub + 1 < NB ? st : st + 1, sub_n = sub + 1 < NB ? sub + 1 : 0;
            if (sub + 1 == NB) barrier();                  // the next stage is in LDS
            if (t0 < wlen) {                               // wave-uniform
                if (__any(mx > kSlack<BITS>)) {
                    const float up = fmaxf(fmaxf(mx, other_half(mx)), 0.f);
                    const float alpha = __builtin_amdgcn_exp2f(-up);
                    m_run += up;
                    l_run *= alpha;
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] -= up;
#pragma unroll
                    for (int d = 0; d < 4; ++d) o[d] *= alpha;
                }
                // the next scores next to the exponentials of these
                const int run_n = KS > 1 ? ksg : sub_n;
                const f32x16 s = multiply_k(kbase + (st_n & 1) * kStageBytes + run_n * 8192);
                if (PAGED && sub == 0) next = entries_of(st + 5);
                f16x8 p[2];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float pe = __builtin_amdgcn_exp2f(x[e]);
                    l_run += pe;
                    const f16x2 two = as_f16x2((e & 2) ? vs[e >> 2].y : vs[e >> 2].x);
                    p[e >> 3][e & 7] = (_Float16)__builtin_fmaf((float)((e & 1) ? two.y : two.x), pe, 0.0f);
                }
                // the products with V next to the scaling of the next scores
                const unsigned char* const vb = vbase + (st % 3) * kStageBytes + (KS > 1 ? ksg : sub) * 8192 + lane * 16;
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int d = 0; d < 4; ++d) o[d] = mfma32x32x16(*(const f16x8*)(vb + (2 * d + k) * 1024), p[k], o[d]);
                read_scales(pbase + (st_n & 3) * kStagePairs, run_n);
                const int t_n = first_token(st_n, sub_n);
                const bool there = is_there(st_n, sub_n);
                if constexpr (PAGED) {
                    // A row that has met no token yet, all its pages so far being none of the pool's, takes its reference from these scores as from the first ones: a move
                    // up from the lowest reference would leave nothing of them.  (Its sums are still zero.  The branch parts the scaling below from the products with V, beside which
                    // it runs in the kernel of the contiguous cache.)
                    const bool fresh = m_run == kMaskFloor && len > t_n;
                    if (__any(fresh)) {
                        scale_scores(s, 0.f, true, t_n, there);
                        const float ref = fmaxf(fmaxf(mx, other_half(mx)), kMaskFloor);
                        if (fresh) m_run = ref;
                    }
                }
                scale_scores(s, m_run, at_edge(t_n) || !there, t_n, there);
            } else if (PAGED && sub == 0) {
                next = entries_of(st + 5);
            }
        }
    }

    float l = l_run + other_half(l_run);
    if constexpr (KS > 1) {
        // the second group hands its reference, denominator and rows to the first: [row wave][66][64 lanes]
        float* const part = (float*)smem;
        barrier();
        float* const slot = part + rg * (66 * 64) + lane;
        if (ksg > 0) {
            slot[0] = m_run;
            slot[64] = l;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) slot[(2 + 16 * d + e) * 64] = o[d][e];
        }
        barrier();
        if (ksg > 0) return;
        const float M = fmaxf(m_run, slot[0]);
        const float f0 = __builtin_amdgcn_exp2f(m_run - M), f1 = __builtin_amdgcn_exp2f(slot[0] - M);
        l = l * f0 + slot[64] * f1;
        m_run = M;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[d][e] = o[d][e] * f0 + slot[(2 + 16 * d + e) * 64] * f1;
    }
    if constexpr (PAGED) {
        if (job.partial) {                                 // [RW * 32] references, as many denominators, [RW * 32][128] unnormalised rows
            const int at = rg * 32 + (lane & 31);
            if (hl == 0) {
                job.partial[at] = m_run;
                job.partial[32 * RW + at] = l;
            }
            float* const out = job.partial + 64 * RW + at * kHeadDim + 4 * hl;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int g = 0; g < 4; ++g) *(f32x4*)(out + 32 * d + 8 * g) = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
            return;
        }
    }
    if (!real) return;
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    uint16_t* const out = job.o + tok * job.o_stride + head * kHeadDim + 4 * hl;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            u32x2 w;
            w.x = (uint32_t)f32_to_f16_bits(o[d][4 * g] * inv) | ((uint32_t)f32_to_f16_bits(o[d][4 * g + 1] * inv) << 16);
            w.y = (uint32_t)f32_to_f16_bits(o[d][4 * g + 2] * inv) | ((uint32_t)f32_to_f16_bits(o[d][4 * g + 3] * inv) << 16);
            *(u32x2*)(out + 32 * d + 8 * g) = w;
        }
}

static_assert(4 * 66 * 64 * sizeof(float) <= kLdsBytes, "the merge of the wave groups reuses the stages' LDS");

}  // namespace

}  // namespace tmw4
