// Prompt attention over the quantised KV cache: a chunk of query tokens, causal (paper Sec. 3.3: the attention pipeline's
// prefill side; Sec. 4.3 conversion between the matrix instructions, Sec. 4.4 loading pipeline).
//
// A prompt multiplies every cached key and value with hundreds of query rows, so unlike at a decoding step the matrix cores
// and the softmax arithmetic bound the kernel, not the cache's bytes.  The split of the work follows from that:
//   - A CTA is eight waves over up to 256 query rows of one KV head.  A row is a (token, query head) pair and rows are
//     numbered token by token, so that any group size fills the tiles; a wave owns 32 rows.
//   - The codes are converted ONCE per CTA: all waves turn a stage of 64 tokens into fp16 values q - z (exact) in LDS, in
//     the order in which the 32x32x16 matrix instruction takes its operands (fragment by fragment, lane by lane: reads and
//     writes are conflict-free without padding), one stage ahead of the multiplication.  The 16-column kernel of the decoding
//     step converts per 16 rows and spends more instructions on that than on the softmax.
//   - Scores are computed transposed (S^T = K Q^T).  The rows of the K operand are the stage's tokens in the order
//     0-7, 16-23, 8-15, 24-31, so that the result layout hands a lane the probabilities of exactly the tokens whose values it
//     multiplies as the k-index of O^T = V^T P^T: P never leaves its registers.
//   - Per score the vector ALU does: one multiply-add (the key's scale, minus the running reference), half a maximum, one
//     exponential, one addition (denominator), one multiply-and-round (the value's scale).  The reference moves only when a
//     score exceeds it by 2^kSlack, which makes the rescaling of the 64 output registers rare; probabilities up to 2^kSlack
//     times a scale still fit fp16.
//   - The scores of the next 32 tokens are computed while the exponentials of the current ones are, the products with V while
//     the next scores are scaled: each half of a step has matrix work and independent vector work.
// With fewer rows two groups of four waves (RW = 4, 128 rows) split the context instead: each takes every second run of 32
// tokens, and they meet in LDS at the end.
//
// Measured (32 query / 8 KV heads, 4000 tokens, 8-bit / 4-bit codes; the 16-column kernel ran this before): 345 -> 152-162 us /
// 289 -> 150 us; 64 / 8 heads, 2048 tokens after 6000, 4-bit: 880 -> 465 us = 1.0 PFLOP/s, half of what an MFMA-only loop sustains
// on this chip.  What bounds it is vector and matrix issue together, and the uneven end of a causal launch: a 32-token run is 16
// MFMAs of 32 clocks and 140-150 vector instructions (conversion included), two waves per SIMD; over the whole launch of 4000 tokens
// the matrix pipe is busy 35-37 % of the clocks, the vector pipes issue in 27 % of the waves' time.  Forced interleaving of the two
// (scheduling groups of one MFMA, seven vector instructions, one LDS read) is 6-9 % slower than the compiler's own order, wave
// priorities change nothing.
#include "tm_attn_rows_impl.h"
#include "tm_w4_host.h"

namespace tmw4 {

namespace {

template <int BITS, int RW>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_prefill_kernel(
    AttnCache kv, const uint16_t* __restrict__ Q, const int32_t* __restrict__ positions, const int32_t* __restrict__ counts,
    int count, uint16_t* __restrict__ O, int q_heads, float scale_log2e)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    constexpr int ROWS = 32 * RW;
    const int hk = blockIdx.x, b = blockIdx.y;
    const int tile = (int)gridDim.z - 1 - (int)blockIdx.z;  // the longest rows first
    const int G = q_heads / kv.heads;
    const size_t bh = (size_t)b * kv.heads + hk;

    const int cnt = counts ? min(max(counts[b], 0), count) : count;
    const long pos0 = positions[b];
    const int row0 = tile * ROWS;
    const int tok_first = row0 / G;
    if (tok_first >= cnt || pos0 + tok_first >= kv.cap) return;                     // (uniform) no row to write
    const int len_all = (int)min(max(pos0 + min(cnt, (row0 + ROWS - 1) / G + 1), 0L), (long)kv.cap);
    if (len_all == 0) return;
    const size_t first = ((size_t)b * count * q_heads + (size_t)hk * G) * kHeadDim;
    const long stride = (long)q_heads * kHeadDim;
    const RowsJob job{Q + first, stride, O + first, stride, cnt, G, row0, kv.cap, pos0, 0, (len_all + ST - 1) / ST, nullptr};
    constexpr int kCodeBytes = kHeadDim * BITS / 8;                                 // of one token
    attn_rows<BITS, RW, false>(job, kv.k + bh * kv.cap * kCodeBytes, kv.v + bh * kv.cap * kCodeBytes, kv.sz + bh * kv.cap * 2, PagedWhere{}, len_all, scale_log2e,
                               smem);
}

template <int BITS, int RW>
hipError_t launch(const AttnCache& kv, const uint16_t* Q, const int32_t* positions, const int32_t* counts, int count, uint16_t* O,
                  int q_heads, float scale, hipStream_t stream)
{
    const long rows = (long)count * (q_heads / kv.heads);
    const long tiles = (rows + 32 * RW - 1) / (32 * RW);
    if (kv.heads > 65535 || kv.batch > 65535 || tiles > 65535 || tiles < 1) return hipErrorInvalidValue;
    hipLaunchKernelGGL((attn_prefill_kernel<BITS, RW>), dim3(kv.heads, kv.batch, (unsigned)tiles), dim3(512), kLdsBytes, stream, kv, Q,
                       positions, counts, count, O, q_heads, scale * 1.4426950408889634f);
    return hipGetLastError();
}

template <int BITS, int RW>
hipError_t allow_lds()
{
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&attn_prefill_kernel<BITS, RW>), hipFuncAttributeMaxDynamicSharedMemorySize,
                               kLdsBytes);
}

}  // namespace

hipError_t attn_prefill_setup()
{
    hipError_t e = allow_lds<8, 8>();
    if (e == hipSuccess) e = allow_lds<8, 4>();
    if (e == hipSuccess) e = allow_lds<4, 8>();
    if (e == hipSuccess) e = allow_lds<4, 4>();
    return e;
}

// Rows per CTA for a chunk of `count` tokens: 256 or 128 here, 0 = the 16-column kernel.  The context is known on the device
// only, so the rule compares what one token of it costs in each form: rounds of CTAs (512 of the 16-column form fit the
// chip, 256 of these) times the time of a round relative to a round of 16-column CTAs.  What the host does know is the
// capacity.  Where that is little more than the chunk, the CTAs of a launch attend over anything between nothing and all of it:
// further rounds fill up evenly, but a launch of one round lasts as long as its longest CTA, up to twice the average (less in
// short chunks, where fixed costs count).  Where the capacity is much larger the CTAs are taken to be alike and rounds to be whole.
// With 2.4 and 3.85 none of 110 random launches (16 ... 8192 tokens, 0 ... 16384 before them, 1 ... 32 KV heads, batch 1 ... 8, capacity
// one, two or eight times the context) that leave the 16-column form is slower for it; all of them average 1.32 times its speed and that
// of the fastest form of each, the worst is 26 % behind it (profiles/attn_prefill_rule__random_launches.txt).
int attn_prefill_rows(const AttnCache& kv, int count, int q_heads, int num_cu)
{
    const long bh = (long)kv.batch * kv.heads;
    const int group = q_heads / kv.heads, gw = group < 16 ? group : 16;
    const long rows = (long)count * group, groups = (count + 16 / gw - 1) / (16 / gw) * ((group + 15) / 16);
    const double longest = count < kv.cap ? kv.cap / (kv.cap - 0.5 * count) : 2.0;      // over the average, if the cache fills up
    auto rounds = [&](long ctas) {
        if (ctas <= num_cu) return 1.0 + (longest - 1.0) * (count < 1024 ? count / 1024.0 : 1.0);
        const double r = (double)ctas / num_cu, whole = (double)((ctas + num_cu - 1) / num_cu);
        return r + (whole - r) * (2.0 - longest);
    };
    const double t16 = bh * groups > 2 * num_cu ? (double)(bh * groups) / (2 * num_cu) : 1.0;
    const double t128 = 2.4 * rounds(bh * ((rows + 127) / 128));
    const double t256 = 3.85 * rounds(bh * ((rows + 255) / 256));
    if (t16 <= t128 && t16 <= t256) return 0;
    return t128 < t256 ? 128 : 256;
}

hipError_t launch_attn_prefill_rows(int rows, const AttnCache& kv, const uint16_t* Q, const int32_t* positions, const int32_t* counts,
                                    int count, uint16_t* O, int q_heads, float scale, hipStream_t stream)
{
    if (kv.bits == 8)
        return rows == 256 ? launch<8, 8>(kv, Q, positions, counts, count, O, q_heads, scale, stream)
                           : launch<8, 4>(kv, Q, positions, counts, count, O, q_heads, scale, stream);
    return rows == 256 ? launch<4, 8>(kv, Q, positions, counts, count, O, q_heads, scale, stream)
                       : launch<4, 4>(kv, Q, positions, counts, count, O, q_heads, scale, stream);
}

}  // namespace tmw4
