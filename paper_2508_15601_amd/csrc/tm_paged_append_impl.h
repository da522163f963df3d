// Writing new keys and values into the pages of a quantised cache (tm_paged_append); built by tm_attn.hip, whose quantiser it uses.
//
// Where a sequence has many new tokens it works on runs of 32 tokens of one KV head, a CTA a run: the unit in which codes are laid out (tm_attn.h).  The runs that the call
// touches are numbered over the sequences on the device, so the grid is an upper bound (every run has a token, and a sequence of n tokens touches at most n / 32 + 2) and
// surplus CTAs end at once.
//
// Measured: 10 prompts of 451 to 901 tokens, 28 / 4 heads, 4-bit, keys and queries turned, nothing in the caches: 29 us (114 MB, 3.9 TB/s, most of it the queries, a wave a token);
// 4 x 2000, 32 / 8 heads, 8-bit 42 us (4.3 TB/s): memory and, for the keys, 64-bit arithmetic.  With norms (AppendHeads) 42.8 us; 6 prompts of 801 to 1601 tokens, 28 / 4 heads, 4-bit, three axes: 31.0 us
// (28.6 without norms); 64 sequences of one token 4.5 us (4.2).  Norms put a sum over sixteen lanes and a root into every vector's chain.
#pragma once

namespace tmw4 {

namespace {

constexpr int kAppendLds = 2 * 4096;

// 256 threads, heads h0 .. h1 - 1.  Sixteen lanes hold a token's vector, eight dimensions each; a thread takes two tokens, keys then values (the layout of the block-wise append
// of the contiguous cache).  All four vectors are requested before the angles are worked out, which hides behind them: sines and cosines of the run's new tokens,
// a thread a pair at a time, go through LDS.  The next head's vectors are requested while this one's codes are stored.
template <int BITS, class Heads>
__device__ __forceinline__ void append_run(const PagedPool& pool, const PagedSeqs& seqs, PagedRows k, PagedRows v, const RopePlan& rope, const Heads& heads, uint32_t item, int h0,
                                           int h1, unsigned char* lds, CosSin* cs)
{
    constexpr bool kHeads = std::is_same<Heads, AppendHeads>::value;
    const int tid = threadIdx.x, lane = tid & 63, sub = tid & 15;
    const RunJob job = run_job(pool, seqs, item, lane);
    if (!job.live || job.page < 0) return;                             // CTA-uniform
    const int u0 = job.u0, u1 = job.u1;
    int slot[2];
    u32x4 raw[4];
    auto request = [&](int h) {
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int u = (tid >> 6) * 8 + (it & 1) * 4 + (lane >> 4);
            slot[it & 1] = u;
            raw[it] = u32x4{0u, 0u, 0u, 0u};
            if (u >= u0 && u < u1) {
                const PagedRows& r = it >> 1 ? v : k;
                raw[it] = *(const u32x4*)(r.p + (job.row + u) * r.stride + h * kHeadDim + 8 * sub);
            }
        }
    };
    request(h0);
    SixteenthNorm<Heads> norm(rope, lane);
    if constexpr (kHeads) norm.request(heads.k, h0);
    if (rope.rot) {
        const int pairs = rope.rot / 2, at_once = 64 / pairs, tok = lane / pairs, p = lane - tok * pairs;      // tokens of a wave at a time
        if (tok < at_once) {
            const RopeTurn turn = rope.turns[p];
            for (int u = u0 + (tid >> 6) * at_once + tok; u < u1; u += 4 * at_once) {
                int pos = job.run * kRun + u;
                if constexpr (kHeads) {
                    if (heads.positions) pos = heads.positions[(job.row + u) * rope.axes + turn.axis];
                }
                cs[u * (kHeadDim / 2) + p] = rope_angle(rope, pos, turn);
            }
        }
        __syncthreads();
    }
    uint32_t* const words = reinterpret_cast<uint32_t*>(lds);          // 4-bit: keys in cache order, then value codes [token][136]
    uint8_t* const vcodes = lds + 2048;
    const bool whole = u0 == 0 && u1 == kRun;
    for (int h = h0; h < h1; ++h) {
        const size_t run = paged_run(pool, job.page, h, job.run);
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int which = it >> 1, u = slot[it & 1];
            const bool live = u >= u0 && u < u1;
            if constexpr (kHeads) {
                if (which == 0) raw[it] = head_sixteenth(raw[it], norm.w, norm.at, heads.k, rope, cs + (live ? u : u0) * (kHeadDim / 2), lane);
            } else {
                if (which == 0 && rope.rot) raw[it] = rope_sixteenth(raw[it], rope, cs + (live ? u : u0) * (kHeadDim / 2), lane);
            }
            uint32_t q[8];
            const uint32_t pair = quantise_row8<BITS>(raw[it], q);
            u32x2 bytes;
            bytes[0] = q[0] | (q[1] << 8) | (q[2] << 16) | (q[3] << 24);
            bytes[1] = q[4] | (q[5] << 8) | (q[6] << 16) | (q[7] << 24);
            if constexpr (BITS == 8) {
                if (which == 0) {
                    const int d = 8 * sub, chunk = ((u >> 4) * 2 + ((d & 31) >> 4)) * 64 + 16 * (d >> 5) + (u & 15);
                    *reinterpret_cast<u32x2*>(lds + chunk * 16 + (d & 15)) = bytes;
                } else {
                    const int hh = (u & 15) >> 2, e = (u & 3) + 4 * (u >> 4);
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        const int d = 8 * sub + n, i = d >> 4;
                        lds[4096 + ((i >> 1) * 64 + 16 * hh + (d & 15)) * 16 + (i & 1) * 8 + e] = (uint8_t)q[n];
                    }
                }
            } else {
                if (which == 0) {
                    const int chunk = (u >> 4) * 64 + 16 * (sub >> 2) + (u & 15);
                    uint32_t w = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) w |= q[e] << (4 * ((e >> 1) + 4 * (e & 1)));
                    words[chunk * 4 + (sub & 3)] = w;
                } else {
                    *reinterpret_cast<u32x2*>(vcodes + u * 136 + 8 * sub) = bytes;
                }
            }
            if (live && sub == 0) pool.pairs[(run * kRun + u) * 2 + which] = pair;
        }
        __syncthreads();
        if (h + 1 < h1) request(h + 1);
        if constexpr (kHeads) {
            if (h + 1 < h1 && heads.k.stride) norm.request(heads.k, h + 1);
        }
        if constexpr (BITS == 8) {
            const u32x4 kc = *reinterpret_cast<const u32x4*>(lds + tid * 16);
            u32x4 vc = *reinterpret_cast<const u32x4*>(lds + 4096 + tid * 16);
            u32x4* const kd = reinterpret_cast<u32x4*>(pool.k + run * 4096) + tid;
            u32x4* const vd = reinterpret_cast<u32x4*>(pool.v + run * 4096) + tid;
            const int ku = (tid >> 7) * 16 + (tid & 15);                   // a key chunk is one token's
            if (whole || (ku >= u0 && ku < u1)) *kd = kc;
            if (!whole) {                                                  // a value chunk holds eight: e % 4 + 4 * hh + 16 * (e / 4)
                const int hh = (tid & 63) >> 4;
                uint32_t lo = 0, hi = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int a = e + 4 * hh;
                    if (a >= u0 && a < u1) lo |= 0xffu << (8 * e);
                    if (a + 16 >= u0 && a + 16 < u1) hi |= 0xffu << (8 * e);
                }
                const u32x4 old = *vd;
                const u32x4 keep = {lo, hi, lo, hi};
                vc = (vc & keep) | (old & ~keep);
            }
            *vd = vc;
        } else {
            const int chunk = tid & 127;
            if (tid < 128) {
                const int ku = (chunk >> 6) * 16 + (chunk & 15);
                if (whole || (ku >= u0 && ku < u1))
                    reinterpret_cast<u32x4*>(pool.k + run * 2048)[chunk] = *reinterpret_cast<const u32x4*>(words + chunk * 4);
            } else {
                const int ii = chunk >> 6, hh = (chunk & 63) >> 4, c = chunk & 15;
                u32x4 vc = {0u, 0u, 0u, 0u};
                uint32_t keep = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int u = (e & 3) + 4 * hh + 16 * (e >> 2), sh = 4 * ((e >> 1) + 4 * (e & 1));
                    if (u >= u0 && u < u1) keep |= 0xfu << sh;
#pragma unroll
                    for (int w = 0; w < 4; ++w) vc[w] |= (uint32_t)vcodes[u * 136 + 16 * (4 * ii + w) + c] << sh;
                }
                u32x4* const vd = reinterpret_cast<u32x4*>(pool.v + run * 2048) + chunk;
                if (!whole) {
                    const u32x4 old = *vd, mask = {keep, keep, keep, keep};
                    vc = (vc & mask) | (old & ~mask);
                }
                *vd = vc;
            }
        }
        if (h + 1 < h1) __syncthreads();
    }
}

// Queries of one token, heads h0 .. h1 - 1, by one wave.
template <class Heads>
__device__ __forceinline__ void rotate_row(const PagedSeqs& seqs, PagedRows q, uint16_t* out, long out_stride, int q_heads, const RopePlan& rope, const Heads& heads, uint32_t row,
                                           int h0, int h1, CosSin* cs, int lane)
{
    constexpr bool kHeads = std::is_same<Heads, AppendHeads>::value;
    const SeqFinder finder([&](int b) { return (uint32_t)paged_seq(seqs, b).count; }, seqs.batch, lane);
    const bool live = row < finder.total;
    long at = 0;
    if (live) {
        uint32_t base;
        const PagedSeq s = paged_seq(seqs, finder.find(row, base));
        at = min((long)s.row + (row - base), (long)seqs.tokens - 1);
        bool own = true;
        if constexpr (kHeads) own = !heads.positions;
        if (own) rope_angles<kHeads>(cs, rope, (int)((uint32_t)s.pos + (row - base)), lane);
        if constexpr (kHeads) {
            if (!own) rope_angles_of<true>(cs, rope, heads.positions + at * rope.axes, lane);
        }
    }
    __syncthreads();
    if constexpr (kHeads) {
        if (live) turn_heads(q.p + at * q.stride, out + at * out_stride, h0, h1, heads.q, rope, cs, lane);
    } else {
        if (live) rope_heads(q.p + at * q.stride, out + at * out_stride, h0, h1, kHeadDim, rope, cs, lane);
    }
}

// Blocks 0 .. kv_blocks - 1: runs of keys and values, heads of a run next to each other; the blocks behind them: queries, a wave `per_wave` heads of a row.
template <int BITS, class Heads>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedPool pool, PagedSeqs seqs, PagedRows k, PagedRows v, RopePlan rope, unsigned kv_blocks, int kv_heads,
                                                           PagedRows q, uint16_t* q_out, long q_out_stride, int q_heads, int per_wave, Heads heads)
{
    __shared__ __align__(16) unsigned char lds[kAppendLds];
    __shared__ CosSin cs[kRun * kHeadDim / 2];
    if (blockIdx.x < kv_blocks) {
        const unsigned groups = (unsigned)((pool.heads + kv_heads - 1) / kv_heads), run = blockIdx.x / groups;
        const int h0 = (int)(blockIdx.x - run * groups) * kv_heads;
        append_run<BITS>(pool, seqs, k, v, rope, heads, run, h0, min(h0 + kv_heads, pool.heads), lds, cs);
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned parts = (unsigned)((q_heads + per_wave - 1) / per_wave);
    const unsigned long job = (unsigned long)(blockIdx.x - kv_blocks) * 4 + wave;
    const unsigned row = (unsigned)(job / parts);
    const int h0 = (int)(job - (unsigned long)row * parts) * per_wave;
    rotate_row(seqs, q, q_out, q_out_stride, q_heads, rope, heads, row, h0, min(h0 + per_wave, q_heads), cs + wave * turns_of(kHeadDim / 2), lane);
}

// Few new tokens a sequence (a decoding step, drafts): a wave takes four of a token's vectors - keys of the KV heads, their values, then query heads - and puts codes where they
// belong by itself; the CTAs above would each go through LDS for a token or a few.  Waves are numbered over the sequences, `step` tokens each; a sequence with more has the further
// ones follow in the same waves.  4-bit values of a sequence's tokens share bytes, so there a sequence's tokens all go through the same waves (step = 1).
template <int BITS>
constexpr int kFewTokens = BITS == 8 ? 8 : 1;
template <int BITS, class Heads>
__global__ __launch_bounds__(256) void paged_append_tokens_kernel(PagedPool pool, PagedSeqs seqs, PagedRows k, PagedRows v, RopePlan rope, PagedRows q, uint16_t* q_out,
                                                                  long q_out_stride, int q_heads, int per_token, int step, Heads heads)
{
    constexpr bool kHeads = std::is_same<Heads, AppendHeads>::value;
    __shared__ CosSin cs[4][kHeadDim / 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = lane & 15;
    const uint32_t job = blockIdx.x * 4 + wave;
    const uint32_t token = job / (uint32_t)per_token;
    const int b = (int)(token / (uint32_t)step), vec = (int)(job - token * per_token) * 4 + (lane >> 4);
    if (b >= seqs.batch) return;
    const PagedSeq s = paged_seq(seqs, b);
    const int which = vec < pool.heads ? 0 : vec < 2 * pool.heads ? 1 : 2, h = vec - which * pool.heads;   // keys, values, queries
    SixteenthNorm<Heads> norm(rope, lane);
    if constexpr (kHeads) norm.request(which == 2 ? heads.q : heads.k, which == 2 ? max(min(h, q_heads - 1), 0) : h);
    for (int i = (int)(token - (uint32_t)b * step); i < s.count; i += step) {
        const int pos = (int)((uint32_t)s.pos + (uint32_t)i);
        const long row = (long)s.row + i;
        const int page = pos >= 0 && pos < seqs.cap ? paged_page(pool, seqs, b, pos / kRun) : -1;
        const PagedRows& from = which == 0 ? k : which == 1 ? v : q;
        u32x4 raw = {0u, 0u, 0u, 0u};
        if (which < 2 || h < q_heads) raw = *(const u32x4*)(from.p + row * from.stride + h * kHeadDim + 8 * sub);
        if (kHeads || rope.rot) {
            bool own = true;
            if constexpr (kHeads) {
                own = !heads.positions;
                if (!own) rope_angles_of(cs[wave], rope, heads.positions + row * rope.axes, lane);
            }
            if (own) rope_angles(cs[wave], rope, pos, lane);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if constexpr (kHeads) {
                if (which != 1) raw = head_sixteenth(raw, norm.w, norm.at, which == 2 ? heads.q : heads.k, rope, cs[wave], lane);
            } else {
                const u32x4 turned = rope_sixteenth(raw, rope, cs[wave], lane);
                if (which != 1) raw = turned;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        if (which == 2) {
            if (h < q_heads) *(u32x4*)(q_out + row * q_out_stride + h * kHeadDim + 8 * sub) = raw;
        }
        uint32_t code[8];
        const uint32_t pair = quantise_row8<BITS>(raw, code);
        if (page < 0 || which == 2) continue;
        const int u = pos & (kRun - 1), hh = (u & 15) >> 2, e = (u & 3) + 4 * (u >> 4);
        const size_t run = paged_run(pool, page, h, pos / kRun);
        if (sub == 0) pool.pairs[(run * kRun + u) * 2 + which] = pair;
        if constexpr (BITS == 8) {
            if (which == 0) {
                const int d = 8 * sub, chunk = ((u >> 4) * 2 + ((d & 31) >> 4)) * 64 + 16 * (d >> 5) + (u & 15);
                *reinterpret_cast<u32x2*>(pool.k + run * 4096 + chunk * 16 + (d & 15)) =
                    u32x2{code[0] | (code[1] << 8) | (code[2] << 16) | (code[3] << 24), code[4] | (code[5] << 8) | (code[6] << 16) | (code[7] << 24)};
            } else {
                uint8_t* const at = pool.v + run * 4096 + ((sub >> 2) * 64 + 16 * hh + 8 * (sub & 1)) * 16 + (sub >> 1 & 1) * 8 + e;
#pragma unroll
                for (int n = 0; n < 8; ++n) at[16 * n] = (uint8_t)code[n];
            }
        } else if (which == 0) {
            uint32_t w = 0;
#pragma unroll
            for (int n = 0; n < 8; ++n) w |= code[n] << (4 * ((n >> 1) + 4 * (n & 1)));
            reinterpret_cast<uint32_t*>(pool.k + run * 2048)[((u >> 4) * 64 + 16 * (sub >> 2) + (u & 15)) * 4 + (sub & 3)] = w;
        } else {                                                       // a word holds a dimension of eight tokens, which this thread writes one after another
            uint32_t* const at = reinterpret_cast<uint32_t*>(pool.v + run * 2048) + ((sub >> 3) * 64 + 16 * hh + 8 * (sub & 1)) * 4 + (sub >> 1 & 3);
            const int sh = 4 * ((e >> 1) + 4 * (e & 1));
            uint32_t old[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) old[n] = at[4 * n];
#pragma unroll
            for (int n = 0; n < 8; ++n) at[4 * n] = (old[n] & ~(0xfu << sh)) | (code[n] << sh);
        }
    }
}

}  // namespace

namespace {

template <class Heads>
hipError_t launch_append(const PagedPool& pool, const PagedSeqs& seqs, PagedRows k, PagedRows v, const RopePlan& plan, const Heads& of_heads, PagedRows q, uint16_t* q_out,
                         long q_out_stride, int q_heads, int max_count, int num_cu, hipStream_t stream)
{
    // Measured (32 / 8 heads, 8-bit, queries too), in brackets by runs: one token each of 1, 16, 64 and 256 sequences 3.7, 4.0, 4.0 and 5.3 us (5.2, 5.4, 7.2, 19.5); five each of
    // 12, 64 and 256 sequences 4.1, 6.4 and 14.4 us (5.5, 7.9, 27.6), eight 4.4, 7.9 and 20.1 (5.8, 8.5, 31.2).  Beyond that runs, whose tokens share their way to the page;
    // with 4-bit codes from two tokens on (with atomic operations on the shared bytes 64 sequences of five took 11.9 us, by runs 7.8).
    const int heads = q.p ? q_heads : 0, per_token = (2 * pool.heads + heads + 3) / 4;
    if (max_count >= 1 && max_count <= (pool.bits == 8 ? kFewTokens<8> : kFewTokens<4>) && (long)seqs.batch * max_count * per_token <= 4 * most_ctas(256)) {
        const long blocks = ((long)seqs.batch * max_count * per_token + 3) / 4;
        const auto kernel = pool.bits == 8 ? paged_append_tokens_kernel<8, Heads> : paged_append_tokens_kernel<4, Heads>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, stream, pool, seqs, k, v, plan, q, q_out, q_out_stride, heads, per_token, max_count, of_heads);
        return hipGetLastError();
    }
    // KV heads a CTA: they share a run's sines and cosines, but take their turns, so that only pays where a compute unit has more CTAs than it holds at a time.  By runs x heads (us; one, two
    // and four heads a CTA; 8 / 32 heads 8-bit, then 4 / 28 heads 4-bit).  Queries too, which fill the chip beside fewer CTAs: 128 11.2 / 13.7 / 19.8, 11.8 / 14.2 / 19.7; 280 14.2 / 15.7 / 21,
    // 20.0 / 18.0 / 22.4; 400 18.4 / 17.6 / 22.5, 26.2 / 24.8 / 24.5; 650 28.3 / 25.1 / 26.3, 35.0 / 33.0 / 33.0; 744 31.6 / 28.0 / 26.6, 41.5 / 35.4 / 35.3; 944 37.9 / 34.0 / 32.0, 49.2 / 44.8 /
    // 43.3; 2100 69 / 67 / 63, 94 / 90 / 86.  Keys turned and no queries (three CTAs a compute unit): 496 15.3 / 16.0 / 21, 15.1 / 15.5 / 20; 744 19.1 / 19.0 / 22, 18.6 / 18.4 / 22; 816 21.2 /
    // 19.6 / 23, 20.8 / 18.6 / 22; 1600 29.2 / 28.8 / 29.3, 28.9 / 27.2 / 28.2.  Not turned one and two are within 5 % of each other.
    const double each = (double)most_runs(seqs) * pool.heads / num_cu;
    const int kv_heads = std::min(!plan.rot ? 1 : q.p ? each >= 2.75 ? 4 : each >= 1.2 ? 2 : 1 : each >= 3.0 ? 2 : 1, pool.heads);
    const long kv = most_runs(seqs) * ((pool.heads + kv_heads - 1) / kv_heads);
    const int per_wave = (long)seqs.tokens * q_heads >= 16384L * 8 ? q_heads : 8;
    const long jobs = q.p ? (long)seqs.tokens * ((q_heads + per_wave - 1) / per_wave) : 0, blocks = kv + (jobs + 3) / 4;
    if (blocks <= 0 || blocks > most_ctas(256)) return hipErrorInvalidConfiguration;
    const auto kernel = pool.bits == 8 ? paged_append_kernel<8, Heads> : paged_append_kernel<4, Heads>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, stream, pool, seqs, k, v, plan, (unsigned)kv, kv_heads, q, q_out, q_out_stride, q_heads, per_wave, of_heads);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const PagedPool& pool, const PagedSeqs& seqs, PagedRows k, PagedRows v, const RopePlan* rope, const AppendHeads* heads, PagedRows q, uint16_t* q_out,
                               long q_out_stride, int q_heads, int max_count, int num_cu, hipStream_t stream)
{
    const RopePlan plan = rope ? *rope : RopePlan{nullptr, 1.0, 0, 0, 1};
    return heads ? launch_append(pool, seqs, k, v, plan, *heads, q, q_out, q_out_stride, q_heads, max_count, num_cu, stream)
                 : launch_append(pool, seqs, k, v, plan, NoHeads{}, q, q_out, q_out_stride, q_heads, max_count, num_cu, stream);
}

}  // namespace tmw4
