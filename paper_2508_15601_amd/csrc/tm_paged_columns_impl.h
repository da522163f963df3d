// The kernel of few rows per sequence over pages; tm_paged_attn.hip, which describes it, and tm_paged_rows.hip build it.
#pragma once
#include "tm_attn_device.h"
#include "tm_paged_host.h"

namespace tmw4 {

namespace {

constexpr int kGroupPieces = 16;         // pieces merged at a time
constexpr int kAgentScope = 16;          // cache-policy bit (sc1) of a store that goes through to memory, and of a load that sees such stores of other XCDs
constexpr uint32_t kSegmentStart = 2;    // what beginning a segment costs, in quads
constexpr uint32_t kUnaligned = 4;       // what a CTA pays for not beginning with a segment: most of them have one more to begin, and two to hand on

// Page numbers of the parts of a block.
template <int PARTS>
struct BlockPages {
    int id[PARTS];
};

// What query column c of a tile of columns that begins at row r0 is: a token and a query head of the KV head's; not real: no row, or one whose position the table does not
// reach, and the sequence's first row stands in as an address that exists.
struct Column {
    int tok, head;
    bool real;
    __device__ __forceinline__ Column(int c, int r0, const PagedSeq& s, int G, int cap)
    {
        const int row = r0 + c;
        tok = row / G;
        head = row - tok * G;
        const long pos = (long)s.pos + tok;
        real = row < s.count * G && pos >= 0 && pos < cap;
        if (!real) tok = 0, head = 0;
    }
};

// The value plus those of lanes 16 and 32 apart, and plus that of the lane 8 apart, without a trip through LDS.
__device__ __forceinline__ float fold_halves(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    auto add = [](auto r) { return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]); };
    uint32_t a = __builtin_bit_cast(uint32_t, v);
    v = add(__builtin_amdgcn_permlane16_swap(a, a, false, false));
    a = __builtin_bit_cast(uint32_t, v);
    v = add(__builtin_amdgcn_permlane32_swap(a, a, false, false));
#endif
    return v;
}
__device__ __forceinline__ float fold_row(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x128, 0xf, 0xf, true));       // row_ror 8
}

// A wave's part: sixteen query columns, or eight (PACK), on the 16x16x32 instruction, with the arithmetic of decode attention over the contiguous cache (tm_attn_device.h).
template <int BITS, bool PACK>
struct Columns {
    static constexpr int kCols = PACK ? 8 : 16;
    f16x8 qf[4];
    float qsum, scale_log2e;
    f32x4 neg_qbias;
    SoftmaxState st;
    f32x4 acc[8];

    static __device__ __forceinline__ int column(int lane) { return lane & (kCols - 1); }
    static __device__ __forceinline__ bool owns(int lane) { return (lane & 15) < kCols; }          // the others are copies

    // q: the row of the lane's column
    f16x8 raw[4];
    __device__ __forceinline__ void request_query(const uint16_t* q, int lane)
    {
#pragma unroll
        for (int t = 0; t < 4; ++t) raw[t] = *(const f16x8*)(q + 32 * (lane >> 4) + 8 * t);
    }
    __device__ __forceinline__ void begin(bool real, float scale)
    {
        scale_log2e = scale;
        float qbias = 0.f;
        qsum = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int e = 0; e < 8; ++e) qf[t][e] = real ? raw[t][e] : (_Float16)0.0f;
            u32x4 bits = __builtin_bit_cast(u32x4, qf[t]);
            asm volatile("" : "+v"(bits.x), "+v"(bits.y), "+v"(bits.z), "+v"(bits.w));            // (keeps this arithmetic behind the requests before it)
            qf[t] = __builtin_bit_cast(f16x8, bits);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                qsum += (float)qf[t][e];
                qbias += ((e & 2) ? 64.0f : 1024.0f) * (float)qf[t][e];
            }
        }
        qsum = xor_add(xor_add(qsum, 16), 32);
        qbias = BITS == 8 ? 1024.0f * qsum : xor_add(xor_add(qbias, 16), 32);
        neg_qbias = f32x4{-qbias, -qbias, -qbias, -qbias};
        // the reference starts above the mask value: a wave may meet blocks in which a column has no live token
        st = SoftmaxState{kMaskFloor, 0.f, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    template <int PARTS, int STEP, bool WINDOW>
    __device__ __forceinline__ void block(const BlockRegs& r, const uint32_t* words, const Magic& mg, int blk, int len, int len_all, int lane, uint32_t present, int lo, int first)
    {
        if constexpr (PARTS == 1)
            process_block<BITS, PACK, false, STEP, WINDOW>(r, words, qf, scale_log2e, qsum, neg_qbias, mg, blk, present ? len : 0, len_all, lane, st, acc, ~0u, present ? lo : 0, first);
        else
            process_block<BITS, PACK, true, STEP, WINDOW>(r, words, qf, scale_log2e, qsum, neg_qbias, mg, blk, len, len_all, lane, st, acc, present, lo, first);
    }
    // The four waves that share the columns meet in LDS: wave `wave` gets the unnormalised values o[i] of dimensions 16 * (2 * wave + i) + 4 * (lane / 16) ... of its lane's column, the
    // reference M and the denominator L.  (One barrier; another has to follow before the next segment's.)
    struct Join {
        float ml[4][2][16];
        float out[4][8][4][64];
    };
    __device__ __forceinline__ f32x4 values(int i, float corr) const
    {
        f32x4 v;
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) v[rr] = (BITS == 8 ? acc[i][rr] + st.bias[rr] : acc[i][rr]) - corr;
        return v;
    }
    __device__ __forceinline__ void sums(float& l, float& corr) const
    {
        l = fold_halves(st.l_run), corr = fold_halves(st.corr);
        if constexpr (PACK) l = fold_row(l), corr = fold_row(corr);
    }
    // A wave that has its columns to itself: o[i] are dimensions 16 * i + 4 * (lane / 16) ...
    __device__ __forceinline__ void alone(float& M, float& L, f32x4 (&o)[8])
    {
        float corr;
        sums(L, corr);
        M = st.m_run;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = values(i, corr);
    }
    __device__ __forceinline__ void join(Join& lds, int wave, int lane, float& M, float& L, f32x4 (&o)[2])
    {
        const int c = lane & 15;
        float l, corr;
        sums(l, corr);
        if (lane < 16) {
            lds.ml[wave][0][c] = st.m_run;
            lds.ml[wave][1][c] = l;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f32x4 v = values(i, corr);
#pragma unroll
            for (int rr = 0; rr < 4; ++rr) lds.out[wave][i][rr][lane] = v[rr];
        }
        __syncthreads();
        M = kNegBig;
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, lds.ml[w][0][c]);
        float f[4];
        L = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[w] = exp2f(lds.ml[w][0][c] - M);
            L += lds.ml[w][1][c] * f[w];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) v += lds.out[w][2 * wave + (i >> 2)][i & 3][lane] * f[w];
            o[i >> 2][i & 3] = v;
        }
    }
};

// PARTS: pieces of a block that may lie on pages of their own: 2 for 4-bit codes on pages of a single run, else 1.
// TILES: tiles of columns that a CTA takes at once, four waves each: with two, the waves that share a block ask for it at the same time, and it comes from memory once.  (Tiles one after
// the other read it twice: 12 x 5 drafted tokens after 6000, 25 columns, 8-bit codes: 45 us, like this 36.  The codes are then not loaded as data that nobody else wants, which
// cost the second wave a quarter of its hits: 32 x 5 after 8000 120 us, so 104.)
// block, blocks: the CTA and how many there are; WAVES: of a CTA.
// WINDOW: blocks that none of a sequence's new tokens sees are left out, and what is left is numbered through; a block that its tile does not see is not read.
template <int BITS, bool PACK, int PARTS, int TILES, bool ALONE, int WAVES, bool WINDOW = false>
__device__ __forceinline__ void paged_columns(const PagedPool& pool, const PagedSeqs& seqs, const uint16_t* __restrict__ Q, long q_stride, uint16_t* __restrict__ O, int q_heads,
                                              float scale_log2e, int most_rows, float* __restrict__ partial, uint32_t* __restrict__ counters, uint32_t block, uint32_t blocks)
{
    static_assert(ALONE ? TILES == 1 : WAVES == 4 * TILES, "four waves a tile");
    constexpr int TOK = 256 / BITS, RUNS = TOK / kRun;       // tokens and runs of a block
    constexpr int kStep = ALONE ? 1 : 4;                     // blocks of a quad
    constexpr int kValues = ALONE ? 8 : 2;                   // vectors of four values that a thread has of the result
    constexpr uint32_t kLeastQuads = ALONE || BITS == 8 ? 2 : 1;      // of a piece (1 x 2048 tokens, 8 heads, pieces of 1 / 2 / 3: 8-bit 9.8 / 9.0 / 9.2 us, 4-bit 9.5 / 10.6 / 11.6)
    static_assert(PARTS == 1 || (BITS == 4 && PARTS == RUNS), "a part is a run, or the whole block");
    typedef Columns<BITS, PACK> Form;
    constexpr int COLS = Form::kCols * TILES;                // of a segment
    constexpr int kMergeLoads = ALONE ? 2 : 8;               // pieces in flight at once when they are merged
    constexpr int kPartial = 2 * COLS + 2048 * TILES;        // M and L of every column, eight unnormalised values a thread
    // scale/zero words of the blocks in flight; one array per ring slot so that the compiler can tell which direct-to-LDS load a read depends on
    __shared__ __attribute__((aligned(16))) uint32_t sz_ring0[WAVES][2 * TOK];
    __shared__ __attribute__((aligned(16))) uint32_t sz_ring1[WAVES][2 * TOK];
    __shared__ __attribute__((aligned(16))) uint32_t sz_ring2[WAVES][2 * TOK];
    __shared__ typename std::conditional<ALONE, int, typename Form::Join>::type s_join[TILES];
    __shared__ uint32_t s_last;
    __shared__ u32x2 s_sums[WAVES][64];
    __shared__ u32x4 s_seqs[WAVES][64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int any_wave = __builtin_amdgcn_readfirstlane(tid >> 6), wave = ALONE ? 0 : any_wave / TILES, part = ALONE ? 0 : any_wave % TILES;      // part: the wave's tile
    const int c = Form::kCols * part + Form::column(lane);   // column of the segment
    const int G = q_heads / pool.heads;

    // ---- this CTA's piece of the work
    auto tiles_of = [&](const PagedSeq& s) { return s.count * G <= most_rows ? (s.count * G + COLS - 1) / COLS : 0; };
    auto quads_of = [&](const PagedSeq& s) {
        const int end = max(s.last(seqs.cap), 0);
        return WINDOW ? ((end + TOK - 1) / TOK - Hidden(seqs, s.first(), TOK).count + kStep - 1) / kStep : (end + kStep * TOK - 1) / (kStep * TOK);
    };
    const uint32_t ctas = ALONE ? WAVES * blocks : blocks, me = ALONE ? WAVES * block + any_wave : block;      // CTAs, or waves, that share the work
    // Up to 64 sequences a lane holds one, loaded once: a launch of few short contexts is a chain of memory round trips, and this one is its first.
    const bool one_each = seqs.batch <= 64;
    PagedSeq own{0, 0, 0};
    uint32_t piece = 0;                                      // not 0: aligned, every piece of a segment but its last is as long, and every segment begins with a CTA
    if (one_each) {
        uint32_t n = 0, q = 0;
        if (lane < seqs.batch) {
            own = paged_seq(seqs, lane);
            q = (uint32_t)quads_of(own);
            n = q ? (uint32_t)(tiles_of(own) * pool.heads) : 0u;
        }
        const uint32_t segments = wave_total(n), all = wave_total(n * q);
        if (!ALONE && segments <= ctas) {
            const uint32_t ideal = max((all + ctas - 1) / ctas, kLeastQuads), loose = (all + kSegmentStart * segments) / ctas + kUnaligned;
            uint32_t p = ideal;
            while (p <= loose && wave_total(n * ((q + p - 1) / p)) > ctas) p += 1 + (p >> 4);
            // up to sixteen pieces are merged in one level, and a second one costs as much as three quads of 8-bit codes, two of 4-bit ones (one context of 8192, 8 heads, 8-bit: 16 pieces
            // of four quads 11.8 us, 32 of two 13.8; of 16384, 4-bit: 16 of four 15.1, 32 of two 15.7); three quads take no longer than a merge
            const uint32_t longest = wave_greatest(q), single = (longest + kGroupPieces - 1) / kGroupPieces;
            if (single <= p + (BITS == 8 ? 3 : 2)) p = max(p, single);
            if (longest <= 3) p = max(p, longest);
            if (p <= loose) piece = p;
        }
    }
    const bool aligned = piece != 0;
    const uint32_t start = aligned ? 0u : kSegmentStart;
    auto units_of = [&](const PagedSeq& s) {                 // of a segment
        const uint32_t q = (uint32_t)quads_of(s);
        return aligned ? (q + piece - 1) / piece * piece : q ? kSegmentStart + q : 0u;
    };
    auto work_of = [&](const PagedSeq& s) { return (uint32_t)(tiles_of(s) * pool.heads) * units_of(s); };
    auto work_at = [&](int b) { return work_of(paged_seq(seqs, b)); };
    uint32_t total;
    {
        const SeqFinder finder = one_each ? SeqFinder(work_at, seqs.batch, work_of(own)) : SeqFinder(work_at, seqs.batch, lane);
        s_sums[any_wave][lane] = u32x2{finder.mine, finder.incl};            // (not in registers through the loops below)
        s_seqs[any_wave][lane] = u32x4{(uint32_t)own.row, (uint32_t)own.count, (uint32_t)own.pos, 0u};
        total = finder.total;
    }
    if (!aligned) piece = max((total + ctas - 1) / ctas, kLeastQuads);
    uint32_t at = me * piece;
    if (at >= total) return;
    const uint32_t end = min(at + piece, total);
    auto ring = [&](int i) { return i == 0 ? sz_ring0[any_wave] : i == 1 ? sz_ring1[any_wave] : sz_ring2[any_wave]; };
    const Magic mg = make_magic();

    while (at < end) {
        uint32_t base;
        const u32x2 sums = s_sums[any_wave][lane];
        const int b = SeqFinder(work_at, seqs.batch, sums[0], sums[1]).find(at, base);
        auto sequence = [&](int i) {
            if (!one_each) return paged_seq(seqs, i);
            const u32x4 held = s_seqs[any_wave][lane];
            return PagedSeq{__builtin_amdgcn_readlane((int)held[0], i), __builtin_amdgcn_readlane((int)held[1], i), __builtin_amdgcn_readlane((int)held[2], i)};
        };
        const PagedSeq s = sequence(b);
        const uint32_t units = max(units_of(s), 1u), tiles = (uint32_t)max(tiles_of(s), 1);
        const uint32_t segment = (at - base) / units, ua = (at - base) - segment * units;
        const uint32_t seg_first = at - ua, ub = min(units, ua + (end - at));
        const int tile = (int)(segment % tiles), hk = min((int)(segment / tiles), pool.heads - 1);
        at += ub - ua;
        if (ub <= start) continue;                           // (uniform) its quads are all the next CTA's
        const uint32_t quads = (uint32_t)quads_of(s), qa = max(ua, start) - start, qb = min(ub - start, quads);
        if (qa >= qb) continue;

        // ---- columns
        const int rows = s.count * G, r0 = tile * COLS;
        const Column col(c, r0, s, G, seqs.cap);
        const int len = col.real ? (int)(s.pos + col.tok) + 1 : 0;
        const int last_tok = (min(r0 + COLS, rows) - 1) / G;
        const int len_all = (int)min(max((long)s.pos + last_tok + 1, 0L), (long)seqs.cap);
        Form form;
        form.request_query(Q + (size_t)(s.row + col.tok) * q_stride + ((size_t)hk * G + col.head) * kHeadDim, lane);
        const Hidden hidden(seqs, WINDOW ? s.first() : 0, TOK);
        auto real = [&](int k) { return WINDOW ? hidden.real(k) : k; };
        const int tile_lo = WINDOW ? (int)min(max((long)s.pos + r0 / G, 0L), (long)seqs.cap) - seqs.window + 1 : 0;      // of the tile's first row; the lane's:
        const int lo = WINDOW ? len - seqs.window : 0;
        const int blk1 = min((int)qb * kStep, (len_all + TOK - 1) / TOK - (WINDOW ? hidden.count : 0));
        int blk = (int)qa * kStep + wave;

        constexpr uint32_t kPart = 4096 / PARTS, kPartTokens = TOK / PARTS;
        // Unchecked, and of the context's last part where the block lies behind it: what is done with a page number waits for it, so that happens a step later.
        const int last_part = max(len_all - 1, 0) / (int)kPartTokens;
        auto pages_of = [&](int k) {
            BlockPages<PARTS> p;
#pragma unroll
            for (int n = 0; n < PARTS; ++n) p.id[n] = paged_entry(pool, seqs, b, min(real(k) * PARTS + n, last_part) * (RUNS / PARTS));
            return p;
        };
        // Requests a block; a part that is not there is a buffer of no bytes, whose loads return zeros without memory traffic.  Returns which parts are there.
        auto load = [&](BlockRegs& r, uint32_t* slot, int k, const BlockPages<PARTS>& p) {
            uint32_t present = 0;
            int off = lane * 16;                             // (opaque, so that the loads' distances go into the instructions and not into registers)
            asm volatile("" : "+v"(off));
#pragma unroll
            for (int n = 0; n < PARTS; ++n) {
                const int at = real(k) * PARTS + n;
                bool ok = k < blk1 && at <= last_part && (uint32_t)p.id[n] < (uint32_t)pool.pages;
                if constexpr (WINDOW) ok = ok && ((at + 1) * (int)kPartTokens > tile_lo || at * (int)kPartTokens < seqs.sinks);
                present |= (uint32_t)ok << n;
                const size_t run = paged_run(pool, ok ? p.id[n] : 0, hk, real(k) * RUNS + n);
                const __amdgpu_buffer_rsrc_t rk = make_rsrc(pool.k + run * (512 * BITS), ok ? kPart : 0u), rv = make_rsrc(pool.v + run * (512 * BITS), ok ? kPart : 0u),
                                             rz = make_rsrc(pool.pairs + run * kRun * 2, ok ? kPartTokens * 8u : 0u);
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
                for (int i = 0; i < (int)kPartTokens / kRun; ++i)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rz, (__attribute__((address_space(3))) void*)(slot + 64 * (n + i)), 4, lane * 4 + i * 256, 0, 0, 0);
#else
                (void)rz, (void)slot;
#endif
                // key loads 0 .. 3 of a block: [16-token tile][half] of 8-bit codes, [run][16-token tile] of 4-bit ones
#pragma unroll
                for (int i = 0; i < 4 / PARTS; ++i) {
                    const int at = 4 / PARTS * n + i;
                    r.k[at >> 1][at & 1] = __builtin_amdgcn_raw_buffer_load_b128(rk, off + i * 1024, 0, TILES > 1 ? 0 : kNonTemporal);
                }
#pragma unroll
                for (int i = 0; i < 4 / PARTS; ++i) r.v[4 / PARTS * n + i] = __builtin_amdgcn_raw_buffer_load_b128(rv, off + i * 1024, 0, TILES > 1 ? 0 : kNonTemporal);
            }
            return present;
        };

        BlockRegs g[3];
        uint32_t there[3];
        BlockPages<PARTS> next = pages_of(blk), after = pages_of(blk + kStep);
        there[0] = load(g[0], ring(0), blk, next);
        next = pages_of(blk + 2 * kStep);
        there[1] = load(g[1], ring(1), blk + kStep, after);
        form.begin(col.real, scale_log2e);
        auto step = [&](int use) {
            const int fill = (use + 2) % 3;
            there[fill] = load(g[fill], ring(fill), blk + 2 * kStep, next);
            next = pages_of(blk + 3 * kStep);
            form.template block<PARTS, kStep, WINDOW>(g[use], ring(use), mg, real(blk), len, len_all, lane, there[use], lo, WINDOW ? seqs.sinks : 0);
            blk += kStep;
            return blk < blk1;
        };
        if (blk < blk1)
            while (step(0) && step(1) && step(2)) {
            }
        float M, L;                                          // of the thread's column
        f32x4 o[kValues];
        if constexpr (ALONE) form.alone(M, L, o);
        else form.join(s_join[part], wave, lane, M, L, o);
        auto sync = [&]() {
            if constexpr (!ALONE) __syncthreads();
        };

        // What the loop above does not need is worked out again here rather than kept in registers through it.
        int b_again = b, r0_again = r0;
        asm volatile("" : "+s"(b_again), "+s"(r0_again));
        const PagedSeq t = sequence(b_again);
        const Column out(c, r0_again, t, G, seqs.cap);
        auto finish = [&](float m_l) {
            const float inv = m_l > 0.f ? 1.0f / m_l : 0.f;
#pragma unroll
            for (int i = 0; i < kValues; ++i) {
                const float v[4] = {o[i][0] * inv, o[i][1] * inv, o[i][2] * inv, o[i][3] * inv};
                if (out.real && Form::owns(lane)) store_out4(O, t.row + out.tok, q_heads, hk * G + out.head, 16 * (kValues * wave + i) + 4 * (lane >> 4), v);
            }
        };
        if (qa == 0 && qb == quads) {                        // (uniform) the whole segment was this CTA's
            finish(L);
            sync();
            continue;
        }

        // ---- a piece of a segment.  Its slot: 2k + 1 for the segment that begins in CTA k, 2k for one that began before it.
        const bool column = Form::owns(lane) && c + r0_again < t.count * G;
        // Slots are written through to memory and read past the caches of this XCD, sixteen bytes a lane: M and L of every column, then the threads' values in two rounds of 1 KiB a wave.
        const __amdgpu_buffer_rsrc_t slots = make_rsrc(partial, (uint32_t)kPagedColumnBytes);
        const int value_at = 2 * COLS * 4 + (ALONE ? 0 : any_wave * 2048) + lane * 16;
        auto put = [&](uint32_t slot) {
            const int base = (int)(slot * (uint32_t)(kPartial * 4));
            if (!column) return;
            if (wave == 0 && lane < Form::kCols) {
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, M), slots, base + c * 4, 0, kAgentScope);
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, L), slots, base + (COLS + c) * 4, 0, kAgentScope);
            }
#pragma unroll
            for (int i = 0; i < kValues; ++i) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o[i]), slots, base + value_at + i * 1024, 0, kAgentScope);
        };
        // Bumps a counter once all of this CTA's stores have arrived; true in every thread of the CTA that is the last of n, which also resets it.
        auto arrive = [&](uint32_t* counter, uint32_t n) {
            wait_stores_done();
            if constexpr (ALONE) {
                uint32_t prev = 0;
                if (lane == 0) prev = atomicAdd(counter, 1u);
                prev = (uint32_t)__builtin_amdgcn_readfirstlane((int)prev);
                if (prev == n - 1u && lane == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                asm volatile("" ::: "memory");
                return prev == n - 1u;
            }
            __syncthreads();
            if (tid == 0) {
                const uint32_t prev = atomicAdd(counter, 1u);
                s_last = prev == n - 1u;
                if (prev == n - 1u) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            return s_last != 0u;
        };
        const uint32_t k0 = (seg_first + start) / piece, pieces = (seg_first + start + quads - 1) / piece - k0 + 1;
        auto slot_of = [&](uint32_t j) { return j == 0 ? 2 * k0 + 1 : 2 * (k0 + j); };
        // M, L, o := pieces j0, j0 + step, ... (n of them), in that order
        auto merge = [&](uint32_t j0, uint32_t stride, uint32_t n) {
            M = kNegBig, L = 0.f;
#pragma unroll
            for (int i = 0; i < kValues; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (!column) return;
            for (uint32_t j = 0; j < n; j += kMergeLoads) {
                float ms[kMergeLoads], ls[kMergeLoads];
                f32x4 v[kMergeLoads][kValues];
#pragma unroll
                for (int k = 0; k < kMergeLoads; ++k) {
                    const int base = (int)(slot_of(j0 + stride * (j + k < n ? j + k : 0)) * (uint32_t)(kPartial * 4));
                    ms[k] = __builtin_bit_cast(float, (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(slots, base + c * 4, 0, kAgentScope));
                    ls[k] = __builtin_bit_cast(float, (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(slots, base + (COLS + c) * 4, 0, kAgentScope));
#pragma unroll
                    for (int i = 0; i < kValues; ++i) v[k][i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(slots, base + value_at + i * 1024, 0, kAgentScope));
                }
                float up = M;
#pragma unroll
                for (int k = 0; k < kMergeLoads; ++k) up = fmaxf(up, j + k < n ? ms[k] : kNegBig);
                const float old = exp2f(M - up);
                M = up;
                L *= old;
#pragma unroll
                for (int i = 0; i < kValues; ++i) o[i] *= old;
#pragma unroll
                for (int k = 0; k < kMergeLoads; ++k) {
                    const float f = j + k < n ? exp2f(ms[k] - M) : 0.f;
                    L += ls[k] * f;
#pragma unroll
                    for (int i = 0; i < kValues; ++i) o[i] += v[k][i] * f;
                }
            }
        };
        const uint32_t mine = (at - 1) / piece - k0;         // this piece's number
        const uint32_t groups = (pieces + kGroupPieces - 1) / kGroupPieces, group = mine / kGroupPieces;
        const uint32_t in_group = min((uint32_t)kGroupPieces, pieces - group * kGroupPieces);
        put(slot_of(mine));
        // Counters: of the first group, [CTA in which the segment begins]; of a later one, [CTA of its first piece] - only one segment enters a CTA from before; of the
        // groups of a segment, [CTA in which it begins].
        if (!arrive(counters + (group == 0 ? k0 : ctas + k0 + group * kGroupPieces), in_group)) continue;
        merge(group * kGroupPieces, 1, in_group);
        if (groups > 1) {
            sync();                                          // all of the group has been read before its first slot is written
            put(slot_of(group * kGroupPieces));
            if (!arrive(counters + 2 * ctas + k0, groups)) continue;
            merge(0, kGroupPieces, groups);
        }
        finish(L);
    }
}

}  // namespace

}  // namespace tmw4
