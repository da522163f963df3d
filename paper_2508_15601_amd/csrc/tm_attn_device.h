// Device-side building blocks of attention over a quantised cache, shared by the contiguous and the paged cache: the
// quantiser, and the decode form's arithmetic on a block of the cache.
#pragma once
#include "tm_w4_device.h"

namespace tmw4 {

namespace {

constexpr int kHeadDim = 128;
constexpr float kNegBig = -1.0e30f;     // "minus infinity" that stays finite under subtraction
constexpr float kMaskFloor = -1.0e20f;  // far below any score, far above kNegBig: exp2(kNegBig - kMaskFloor) is 0
constexpr int kNonTemporal = 2;         // cache-policy bit of a buffer load: streamed once, do not keep

// 2^x by the hardware instruction alone: arguments here are at most kSlack (a score less a reference that may lag behind the largest
// score by that much; the product with a value's scale still fits fp16, see SoftmaxState), and a result below the smallest
// normal number may flush to zero (the library function spends four more instructions per call on that range).
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16 mfma32x32x16(f16x8 a, f16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f16x8 add_pairs(f16x8 v, f16x2 a, f16x2 b, f16x2 c, f16x2 d)
{
    const f16x2 r0 = f16x2{v[0], v[1]} + a, r1 = f16x2{v[2], v[3]} + b, r2 = f16x2{v[4], v[5]} + c, r3 = f16x2{v[6], v[7]} + d;
    return f16x8{r0.x, r0.y, r1.x, r1.y, r2.x, r2.y, r3.x, r3.y};
}

__device__ __forceinline__ float xor_max(float v, int mask) { return fmaxf(v, __shfl_xor(v, mask)); }
__device__ __forceinline__ float xor_add(float v, int mask) { return v + __shfl_xor(v, mask); }

// ------------------------------------------------------------------------------------------------ decode attention
// The codes of a block travel in registers (they are the in-flight memory of the pipeline: two blocks ahead).  The 64
// scale/zero words of a block would cost as many registers per lane as its 8 KiB of codes, so they go through LDS
// instead: one direct-to-LDS load per block and wave (lane l fetches word l) into a slot private to the wave.
struct BlockRegs {
    u32x4 k[2][2];      // two 16-token tiles: 32 key bytes of the lane's token (dimensions 32h .. 32h+31)
    u32x4 v[4];         // 64 value bytes: eight 16-row tiles x the lane's eight tokens
};

// Descriptors of one (sequence, head): its K blocks, V blocks and scale/zero words, each cut off after the last block
// of the context.  A load past that end returns zeros without touching memory, which lets the pipeline issue its loads
// unconditionally (the surplus ones at the end of a wave's range cost nothing).
struct HeadRsrc {
    __amdgpu_buffer_rsrc_t k, v, sz;
};

// A block is 4096 bytes of key codes and as many of value codes: 32 tokens of 8-bit codes, or 64 tokens of 4-bit codes
// (two 32-token halves of 2048 bytes each, r.k[half][tile], r.v[2*half + i/4]); the load instructions are the same.
template <int BITS>
__device__ __forceinline__ void load_block(BlockRegs& r, uint32_t* sz_slot, const HeadRsrc& rs, int blk, int lane)
{
    // (the host pass of the compiler only needs the kernel's signature; it cannot express the LDS pointer)
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (BITS == 8) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs.sz, (__attribute__((address_space(3))) void*)sz_slot, 4,
                                                 lane * 4 + blk * 256, 0, 0, 0);
    } else {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs.sz, (__attribute__((address_space(3))) void*)sz_slot, 4,
                                                 lane * 4 + blk * 512, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs.sz, (__attribute__((address_space(3))) void*)(sz_slot + 64), 4,
                                                 lane * 4 + blk * 512 + 256, 0, 0, 0);
    }
#else
    (void)sz_slot;
#endif
    // every load instruction of the wave reads 1 KiB of consecutive bytes: the blocks are stored in operand order.
    // The block offset sits in the per-lane offset, which the descriptor's range check covers.
    const int off = lane * 16 + blk * 4096;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        r.k[j][0] = __builtin_amdgcn_raw_buffer_load_b128(rs.k, off + (j * 2 + 0) * 1024, 0, kNonTemporal);
        r.k[j][1] = __builtin_amdgcn_raw_buffer_load_b128(rs.k, off + (j * 2 + 1) * 1024, 0, kNonTemporal);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = __builtin_amdgcn_raw_buffer_load_b128(rs.v, off + i * 1024, 0, kNonTemporal);
}

// Running state of one wave (per query head m = lane % 16; m_run is equal in the four lanes that share an m, l_run and
// corr are per-lane partial sums over the lane's own tokens).  m_run is the reference the exponents are taken against: the
// largest score up to a factor of 2^kSlack.  It moves only when a score exceeds it by more than that, so a block normally
// needs no exchange between lanes and no rescaling: the shuffles of a running maximum were the longest part of the chain of
// dependent instructions that two waves per SIMD cannot hide.  Probabilities of at most 2^kSlack times a scale fit fp16.
struct SoftmaxState {
    float m_run, l_run, corr;
    f32x4 bias;                            // 8-bit codes: minus the value bias that acc carries at the moment
};
template <int BITS>
constexpr float kSlack = BITS == 8 ? 6.0f : 2.0f;      // 2^6 * (2 * 65504 / 255), 2^2 * (2 * 65504 / 15) < 65504

__device__ __forceinline__ uint32_t swap_half_rows(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xf, 0xf, true);      // row_ror:8 = lane c <-> c ^ 8
}

// Moves the reference to the largest score of every query head so far (mx: the lane's largest new score, not reduced).
template <int BITS, bool PACK>
__device__ __forceinline__ void move_reference(float mx, SoftmaxState& st, f32x4 (&acc)[8])
{
    if constexpr (PACK) mx = fmaxf(mx, __builtin_bit_cast(float, swap_half_rows(__builtin_bit_cast(uint32_t, mx))));
    mx = xor_max(xor_max(mx, 16), 32);
    const float m_new = fmaxf(st.m_run, mx);
    const float alpha = fast_exp2(st.m_run - m_new);
    st.m_run = m_new;
    st.l_run *= alpha;
    st.corr *= alpha;
    if constexpr (BITS == 8) st.bias *= alpha;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] *= alpha;
}

// Runs N0 .. N0 + NH - 1 of thirty-two tokens of a block (8-bit codes: one run, 4-bit codes: two).  qsum =
// sum of the query's 128 values; neg_qbias = minus the sum of the conversion bias of each code position times the query
// value it meets.  len: tokens the lane's query column attends over (the same in every lane at a decoding step; at prefill
// every column has its own causal limit).
// STEP: a wave takes every STEP-th block.
// HOLES (paged cache): bit i of `present` tells whether run i of the block lies on a page of the pool; without it the run has no tokens.
//
// PACK: at most eight query heads share the KV head.  The query operand then carries every head twice
// (column c and c + 8 both hold head c % 8), so both score tiles of a run come out with all 16 columns live, and a lane keeps
// tile c / 8 only - four scores instead of eight, half the softmax arithmetic.  The probabilities of the other tile's
// tokens reach the lane through one exchange with lane c ^ 8 before the second product; running sums are per lane over
// its own tokens and meet at the end (xor 8, 16, 32).
template <int BITS, bool PACK, int N0, int NH, bool HOLES = false, int STEP = 4>
__device__ __forceinline__ void process_runs(const BlockRegs& r, const uint32_t* sz_slot, const f16x8 (&qf)[4],
                                              float scale_log2e, float qsum, const f32x4& neg_qbias, const Magic& mg, int blk, int len,
                                              int lane, SoftmaxState& st, f32x4 (&acc)[8], uint32_t present = ~0u)
{
    constexpr int NS = PACK ? 1 : 2;                         // score tiles a lane keeps of a run
    const int h = lane >> 4, jl = PACK ? (lane >> 3) & 1 : 0;      // jl: the 16-token tile this lane keeps
    const int rem_all = len - blk * (256 / BITS) - 32 * N0 - 4 * h - 16 * jl;  // slot (n, j, rr) is a live token iff 32*n + 16*j + rr < rem
    auto rem_of = [&](int n) { return !HOLES || (present >> (N0 + n) & 1u) ? rem_all : -1; };
    float t[NH][NS][4];                                      // scores before the key's scale
    f16x2 kp[NH][NS][4];                                     // (scale, zero-point) of the slot's key
    uint32_t vw[NH][NS][4];                                  // and of its value; 0 for a dead token
#pragma unroll
    for (int n = 0; n < NH; ++n) {
        const int rem = rem_of(n);
        // S^T for the two 16-token tiles: rows = tokens, columns = query heads.  The accumulator starts at minus the bias
        // term: sum_d (bias_d + q_d) Q_d - sum_d bias_d Q_d = sum_d q_d Q_d
        f32x4 d[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if constexpr (BITS == 8) {
                d[j] = mfma16x16x32(biased8_w8(r.k[j][0].x, r.k[j][0].y), qf[0], neg_qbias);
                d[j] = mfma16x16x32(biased8_w8(r.k[j][0].z, r.k[j][0].w), qf[1], d[j]);
                d[j] = mfma16x16x32(biased8_w8(r.k[j][1].x, r.k[j][1].y), qf[2], d[j]);
                d[j] = mfma16x16x32(biased8_w8(r.k[j][1].z, r.k[j][1].w), qf[3], d[j]);
            } else {
                const u32x4 w = r.k[N0 + n][j];
                d[j] = mfma16x16x32(biased8(w.x, mg), qf[0], neg_qbias);
                d[j] = mfma16x16x32(biased8(w.y, mg), qf[1], d[j]);
                d[j] = mfma16x16x32(biased8(w.z, mg), qf[2], d[j]);
                d[j] = mfma16x16x32(biased8(w.w, mg), qf[3], d[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            // (K pair, V pair) of the lane's four tokens 16*(j or jl) + 4h .. +3: eight consecutive words of the slot
            const uint32_t* const z = sz_slot + 64 * (N0 + n) + 32 * (PACK ? jl : j) + 8 * h;
            const u32x4 p0 = *(const u32x4*)z, p1 = *(const u32x4*)(z + 4);
#pragma unroll
            for (int rr = 0; rr < 4; ++rr) {
                // a dead token contributes nothing, whatever its pair holds: scale 0 and zero-point 0 for its values
                const bool live = 32 * n + 16 * j + rr < rem;
                kp[n][j][rr] = as_f16x2(rr < 2 ? p0[2 * rr] : p1[2 * (rr - 2)]);
                vw[n][j][rr] = live ? (rr < 2 ? p0[2 * rr + 1] : p1[2 * (rr - 2) + 1]) : 0u;
                // sum_d q_d Q_d  -  z sum_d Q_d  =  sum_d (q_d - z) Q_d, times scale * log2(e).  (The pair enters a multiply-add,
                // which takes fp16 directly.  The scale goes here, in fp32, and not into the query's fp16 values, where its rounding
                // would be a fifth of the result's error.)
                const float dm = PACK ? (jl ? d[1][rr] : d[0][rr]) : d[j][rr];
                t[n][j][rr] = scale_log2e * __builtin_fmaf(-(float)kp[n][j][rr].y, qsum, dm);
            }
        }
    }
    // scores in base 2 less the reference
    float x[NH][NS][4], mx = kNegBig;
    auto scores = [&](float ref) {
        mx = kNegBig;
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            const int rem = rem_of(n);
#pragma unroll
            for (int j = 0; j < NS; ++j)
#pragma unroll
                for (int rr = 0; rr < 4; ++rr) {
                    const float v = __builtin_fmaf((float)kp[n][j][rr].x, t[n][j][rr], -ref);
                    x[n][j][rr] = 32 * n + 16 * j + rr < rem ? v : kNegBig;
                    mx = fmaxf(mx, x[n][j][rr]);
                }
        }
    };
    scores(st.m_run);
    if (__any(mx > kSlack<BITS>)) {
        scores(0.0f);
        move_reference<BITS, PACK>(mx, st, acc);
        scores(st.m_run);
    }
    // probability times the value scale of that token, rounded to fp16: the operand of the second product.  The zero-point
    // term must be built from the very fp16 values the matrix core multiplies: a zero-point is as large as the codes and the
    // two sums cancel, so a disagreement of one fp16 ulp per probability would stay in the result at full size.  Left to itself
    // the compiler rounds p * vs once for the operand (fused multiply-and-convert) and once more, through fp32, for the sum
    // below; the two differ when the fp32 product lands on an fp16 tie.  Pinning the packed operand makes it the only copy.
    float psum = 0.f, zsum = 0.f;
    f16x8 pb[NH];
#pragma unroll
    for (int n = 0; n < NH; ++n) {
        uint32_t own[NS][2];
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            _Float16 q[4];
#pragma unroll
            for (int rr = 0; rr < 4; ++rr) {
                const float p = fast_exp2(x[n][j][rr]);      // 0 for masked tokens
                psum += p;
                q[rr] = (_Float16)__builtin_fmaf((float)as_f16x2(vw[n][j][rr]).x, p, 0.0f);
            }
            own[j][0] = (uint32_t)__builtin_bit_cast(uint16_t, q[0]) | ((uint32_t)__builtin_bit_cast(uint16_t, q[1]) << 16);
            own[j][1] = (uint32_t)__builtin_bit_cast(uint16_t, q[2]) | ((uint32_t)__builtin_bit_cast(uint16_t, q[3]) << 16);
            asm volatile("" : "+v"(own[j][0]), "+v"(own[j][1]));
            // sum over the lane's tokens of z * p'
#pragma unroll
            for (int rr = 0; rr < 4; ++rr) {
                const f16x2 two = as_f16x2(own[j][rr >> 1]);
                const float pv = (float)(rr & 1 ? two.y : two.x);
                zsum = __builtin_fmaf((float)as_f16x2(vw[n][j][rr]).y, pv, zsum);
            }
        }
        u32x4 bits;                                          // k-values 0..3: tile 0, 4..7: tile 1
        if constexpr (PACK) {
            const uint32_t x0 = swap_half_rows(own[0][0]), x1 = swap_half_rows(own[0][1]);
            bits.x = jl ? x0 : own[0][0];
            bits.y = jl ? x1 : own[0][1];
            bits.z = jl ? own[0][0] : x0;
            bits.w = jl ? own[0][1] : x1;
        } else {
            bits = u32x4{own[0][0], own[0][1], own[NS - 1][0], own[NS - 1][1]};
        }
        pb[n] = __builtin_bit_cast(f16x8, bits);
    }
    st.l_run += psum;
    st.corr += zsum;
    // The bias of a value code is several times the payload (4-bit codes: up to a hundred times): carried along to the end of
    // a long context it would cost the sums their low bits, in proportion to the context.  Products with the constant operand -bias
    // (1024; 64 at the k-values 2, 3, 6 and 7 of a 4-bit word) sum up what has to leave.  4-bit codes: per block, before the codes
    // that carry it go in.  8-bit codes: every fourth block (128 tokens times 1151 are a seventh of the 8192 times 127 that the codes
    // themselves sum up to over 32768 tokens; taken out of every code before the product it cost the 16-column prompt form up to 8 %:
    // 64 tokens after 12000, 8 heads: 65.2 us, like this 60.9).
    const _Float16 bias_a = (_Float16)-1024.0f, bias_b = BITS == 8 ? bias_a : (_Float16)-64.0f;
    const f16x8 minus_bias = {bias_a, bias_a, bias_b, bias_b, bias_a, bias_a, bias_b, bias_b};
    if constexpr (BITS == 4) {
        f32x4 bias = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < NH; ++n) bias = mfma16x16x32(minus_bias, pb[n], bias);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += bias;
    } else {
        st.bias = mfma16x16x32(minus_bias, pb[0], st.bias);
    }
    // O^T += V^T P'^T : rows = dimensions (eight 16-row tiles), k = the 32 tokens of a run
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f16x8 a;
            if constexpr (BITS == 8) {
                const u32x4 w = r.v[i >> 1];
                a = (i & 1) ? biased8_w8(w.z, w.w) : biased8_w8(w.x, w.y);
            } else {
                a = biased8(r.v[2 * (N0 + n) + (i >> 2)][i & 3], mg);
            }
            acc[i] = mfma16x16x32(a, pb[n], acc[i]);
        }
    if constexpr (BITS == 8) {
        if (((uint32_t)blk / STEP & 3) == 3) {               // (wave-uniform)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += st.bias;
            st.bias = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
}

// A whole block.  The two runs of a 4-bit block go through together, which gives each wave two independent chains of
// instructions; with two score tiles a lane that takes more registers than there are, so there they go one after the other.
template <int BITS, bool PACK, bool HOLES = false, int STEP = 4>
__device__ __forceinline__ void process_block(const BlockRegs& r, const uint32_t* sz_slot, const f16x8 (&qf)[4],
                                              float scale_log2e, float qsum, const f32x4& neg_qbias, const Magic& mg, int blk, int len, int len_all,
                                              int lane, SoftmaxState& st, f32x4 (&acc)[8], uint32_t present = ~0u)
{
    if constexpr (BITS == 8 || PACK) {
        process_runs<BITS, PACK, 0, BITS == 8 ? 1 : 2, HOLES, STEP>(r, sz_slot, qf, scale_log2e, qsum, neg_qbias, mg, blk, len, lane, st, acc, present);
    } else {
        process_runs<BITS, PACK, 0, 1, HOLES, STEP>(r, sz_slot, qf, scale_log2e, qsum, neg_qbias, mg, blk, len, lane, st, acc, present);
        if (blk * 64 + 32 < len_all)                         // (wave-uniform) the second run may lie wholly behind the context
            process_runs<BITS, PACK, 1, 1, HOLES, STEP>(r, sz_slot, qf, scale_log2e, qsum, neg_qbias, mg, blk, len, lane, st, acc, present);
    }
}

// Four consecutive dimensions d0 .. d0+3 of query head `head` of sequence b, rounded to fp16.
__device__ __forceinline__ void store_out4(uint16_t* O, int b, int q_heads, int head, int d0, const float (&o)[4])
{
    u32x2 out;
    out.x = (uint32_t)f32_to_f16_bits(o[0]) | ((uint32_t)f32_to_f16_bits(o[1]) << 16);
    out.y = (uint32_t)f32_to_f16_bits(o[2]) | ((uint32_t)f32_to_f16_bits(o[3]) << 16);
    *(u32x2*)(O + ((size_t)b * q_heads + head) * kHeadDim + d0) = out;
}

}  // namespace

}  // namespace tmw4
