// Norms of heads and their rotation on the device: what the kernel of packed tokens (tm_heads.hip) and the append to pages (tm_paged_append_impl.h) share.
//
//     n = (x - m) * (offset + w) / sqrt(mean((x - m)^2) + eps),    m = 0 or mean(x) over the head,    y = rotate(n)
//
// in 64 bits throughout, like the rotation alone (tm_rope_device.h): a head's sums are then right to the last bits of 53, the result is the fp16 number next to the true one, and a key
// gets the same codes wherever it is normed.  In 32 bits the factor would be off by up to 2^-23, which moves one fp16 value in about 4000 and one 8-bit code in 10^5.
#pragma once
#include "tm_rope_device.h"

namespace tmw4 {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

struct HeadNorm {                        // off: a head's values as they are
    const uint16_t* w;                   // fp16 weights of head 0, nullptr: ones
    long stride;                         // from head to head, 0: all have the same
    double eps, offset, share;           // share: 1 / dimensions of a head
    int on, centred;
};

// What the append does to keys and queries besides turning them by their sequence's positions; NoHeads: nothing.
struct AppendHeads {
    HeadNorm k, q;
    const int32_t* positions;            // [tokens][axes] that turn them, nullptr: those of the sequences on every axis
};
struct NoHeads {
};

// Sum over the LANES neighbouring lanes that hold a head (a power of two up to 16), the same in all of them.
template <int LANES>
__device__ __forceinline__ double lanes_sum(double v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    auto add = [&](auto CTRL) {
        const u32x2 a = __builtin_bit_cast(u32x2, v);
        const u32x2 b = {(uint32_t)__builtin_amdgcn_mov_dpp((int)a[0], decltype(CTRL)::value, 0xf, 0xf, true),
                         (uint32_t)__builtin_amdgcn_mov_dpp((int)a[1], decltype(CTRL)::value, 0xf, 0xf, true)};
        v += __builtin_bit_cast(double, b);
    };
    if constexpr (LANES >= 2) add(std::integral_constant<int, 0xb1>{});      // quad_perm [1, 0, 3, 2]
    if constexpr (LANES >= 4) add(std::integral_constant<int, 0x4e>{});      // quad_perm [2, 3, 0, 1]
    if constexpr (LANES >= 8) add(std::integral_constant<int, 0x141>{});     // row_half_mirror: the other four of eight
    if constexpr (LANES >= 16) add(std::integral_constant<int, 0x140>{});    // row_mirror: the other eight of sixteen
#endif
    return v;
}

// 1 / sqrt(v) for v of at least 1e-300: the hardware's approximation and two steps of Newton's iteration.
__device__ __forceinline__ double inverse_root(double v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    double y = __builtin_amdgcn_rsq(v);
    const double half = 0.5 * v;
#pragma unroll
    for (int i = 0; i < 2; ++i) y = __builtin_fma(y, __builtin_fma(-half * y, y, 0.5), y);
    return v < __builtin_inf() ? y : v != v ? v : 0.0;       // (the steps make an infinity times zero)
#else
    return v;
#endif
}

// Mean (0 unless CENTRED) and factor of a head, of which this lane holds x[0 .. N - 1]: the first half if `any`, the second if `whole`.
template <int LANES, bool CENTRED, int N>
__device__ __forceinline__ void head_norm(const double (&x)[N], bool any, bool whole, const HeadNorm& n, double& mean, double& factor)
{
    auto sum = [&](auto f) {
        double a = 0.0, b = 0.0;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) a = f(x[i], a), b = f(x[N / 2 + i], b);
        return lanes_sum<LANES>((any ? a : 0.0) + (whole ? b : 0.0)) * n.share;
    };
    mean = 0.0;
    if constexpr (CENTRED) {
        mean = sum([](double v, double s) { return s + v; });
        mean = n.centred ? mean : 0.0;
    }
    factor = inverse_root(sum([&](double v, double s) {
                              const double d = CENTRED ? v - mean : v;
                              return __builtin_fma(d, d, s);
                          }) +
                          n.eps);
}

// (offset + w) * factor; least: offset * factor, finite as either is at most 1e150.  (Where offset and w cancel, 2^-53 of `least` is left: a normed value is at most the root of a head's
// dimensions, so nothing that fp16 has.)
__device__ __forceinline__ double weight_of(_Float16 w, double factor, double least) { return __builtin_fma((double)(float)w, factor, least); }

__device__ __forceinline__ f16x8 head_weights(const HeadNorm& n, int head, int d)
{
    f16x8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (_Float16)1.0f;
    if (n.w) w = *(const f16x8*)(n.w + head * n.stride + d);
    return w;
}

// Sixteen dimensions of a head, which a lane holds in two vectors.  INTERLEAVED: one of each half of the lanes' dimensions, so that lanes lie next to each other and all have their share of
// what is turned; otherwise the eight pairs of one stretch of the rotated part, or a stretch that is not turned, which may end after eight.
template <int LANES, bool INTERLEAVED>
struct HeadPart {
    int d0, d1;
    bool turned, turned1, any, whole;    // the vectors are turned, and are there
    __device__ __forceinline__ HeadPart(int u, int dim, const RopePlan& r)
    {
        if constexpr (INTERLEAVED) {
            any = 8 * u < dim;
            whole = 8 * (u + LANES) < dim;
            turned = 8 * u < r.rot;
            turned1 = 8 * (u + LANES) < r.rot;
            d0 = any ? 8 * u : 0;
            d1 = whole ? 8 * (u + LANES) : d0;
        } else {
            any = 16 * u < dim;
            whole = 16 * u + 8 < dim;
            turned = turned1 = 16 * u < r.rot;
            d0 = !any ? 0 : turned ? 8 * u : 16 * u;
            d1 = !any ? 0 : turned ? 8 * u + r.rot / 2 : whole ? 16 * u + 8 : d0;
        }
    }
};

// Norms of the heads of a launch: none, those without a mean, any.
constexpr int kNoNorm = 0, kPlainNorm = 1, kAnyNorm = 2;

// Cosines and sines in LDS: eight pairs, which a lane reads (or two lanes), begin 144 bytes behind the eight before them, so that the lanes of a head meet no banks of each other's.
__device__ __forceinline__ int turn_at(int pair) { return pair + pair / 8; }
constexpr int turns_of(int pairs) { return pairs + pairs / 8; }

// A lane's sixteen values in fp32.  They are what the next heads' vectors leave of these: loaded into registers of their own, the conversion being the copy.
struct Sixteen {
    float v[16];
    __device__ __forceinline__ void of(const f16x8& a, const f16x8& b)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)a[i], v[8 + i] = (float)b[i];
    }
};

// from: the part's vectors, w: their weights, a, b: where the results go (kNoNorm: the vectors themselves, which stay where they are not turned); cs: cosines and sines of the
// token.  Every lane of a head takes part.
template <int LANES, int MODE, bool INTERLEAVED>
__device__ __forceinline__ void head_turn(f16x8& a, f16x8& b, const Sixteen& from, const Sixteen& w, const HeadPart<LANES, INTERLEAVED>& p, const HeadNorm& n, const CosSin* cs)
{
    if (MODE == kNoNorm && !p.turned) return;                // (nor is the second vector then)
    double x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = (double)from.v[i];
    if constexpr (MODE != kNoNorm) {                         // a side without a norm is multiplied by ones, which changes nothing: a branch around this costs a copy of x
        double mean, factor;
        head_norm<LANES, MODE == kAnyNorm>(x, p.any, p.whole, n, mean, factor);
        factor = n.on ? factor : 1.0;
        const double least = n.offset * factor;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = (MODE == kAnyNorm ? x[i] - mean : x[i]) * __builtin_fma((double)w.v[i], factor, least);
    }
    // (rounded on either side of a branch: eight registers meet behind it, not thirty-two)
    if constexpr (INTERLEAVED) {
        auto vector = [&](f16x8& out, const double* v, bool turned, int d) {
            if (turned) {
                const CosSin* const t = cs + turn_at(d / 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    out[2 * i] = rope_round(v[2 * i] * t[i].c - v[2 * i + 1] * t[i].s);
                    out[2 * i + 1] = rope_round(v[2 * i + 1] * t[i].c + v[2 * i] * t[i].s);
                }
            } else if (MODE != kNoNorm) {
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = rope_round(v[i]);
            }
        };
        vector(a, x, p.turned, p.d0);
        vector(b, x + 8, p.turned1, p.d1);
    } else if (p.turned) {
        const CosSin* const t = cs + turn_at(p.d0);
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = rope_round(x[i] * t[i].c - x[8 + i] * t[i].s), b[i] = rope_round(x[8 + i] * t[i].c + x[i] * t[i].s);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = rope_round(x[i]), b[i] = rope_round(x[8 + i]);
    }
}

// Heads of a token as a buffer: what lies behind them is read as zeros and not stored, so that no branch stands around a load or a store.  With nothing in flight before a loop over
// heads (wait_for_loads), its wait for the next ones, which are requested first, leaves the stores behind them in flight; across a branch the compiler would wait for those too.
constexpr int kBehind = 1 << 26;         // values: behind any token's heads
__device__ __forceinline__ f16x8 load8(__amdgpu_buffer_rsrc_t at, int value)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(f16x8, __builtin_amdgcn_raw_buffer_load_b128(at, value * 2, 0, 0));
#else
    return f16x8{};
#endif
}
__device__ __forceinline__ void store8(__amdgpu_buffer_rsrc_t at, f16x8 v, int value)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), at, value * 2, 0, 0);
#endif
}

__device__ __forceinline__ void wait_for_loads()
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_s_waitcnt(0x0f70);                      // vmcnt(0)
#endif
}

// Heads h0 .. h1 - 1 of 128 dimensions of one token, by one wave; x and y (of all of it) may be the same; cs as turn_at() has it.
template <int MODE, bool INTERLEAVED>
__device__ __forceinline__ void turn_heads(const uint16_t* x, uint16_t* y, int h0, int h1, const HeadNorm& n, const RopePlan& r, const CosSin* cs, int lane)
{
    const HeadPart<8, INTERLEAVED> part(lane & 7, 128, r);
    f16x8 a, b, wa, wb;
    const __amdgpu_buffer_rsrc_t from_row = make_rsrc(x, (uint32_t)h1 * 256u), to_row = make_rsrc(y, (uint32_t)h1 * 256u);
    auto request = [&](int at) {
        const int h = at + (lane >> 3), there = min(h, h1 - 1);
        if (n.stride || at == h0) wa = head_weights(n, there, part.d0), wb = head_weights(n, there, part.d1);
        a = load8(from_row, h * 128 + part.d0);
        b = load8(from_row, h * 128 + part.d1);
    };
    request(h0);
    wait_for_loads();
    Sixteen weights;
    for (int at = h0; at < h1; at += 8) {
        f16x8 y0, y1;
        Sixteen from;
        from.of(a, b);
        if (n.stride || at == h0) weights.of(wa, wb);
        if (at + 8 < h1) request(at + 8);
        head_turn<8, MODE, INTERLEAVED>(y0, y1, from, weights, part, n, cs);
        const int h = at + (lane >> 3);
        store8(to_row, y0, h * 128 + part.d0);
        store8(to_row, y1, h * 128 + part.d1);
    }
}
__device__ __forceinline__ void turn_heads(const uint16_t* x, uint16_t* y, int h0, int h1, const HeadNorm& n, const RopePlan& r, const CosSin* cs, int lane)
{
    if (!n.centred && r.interleaved) turn_heads<kPlainNorm, true>(x, y, h0, h1, n, r, cs, lane);
    else if (!n.centred) turn_heads<kPlainNorm, false>(x, y, h0, h1, n, r, cs, lane);
    else if (r.interleaved) turn_heads<kAnyNorm, true>(x, y, h0, h1, n, r, cs, lane);
    else turn_heads<kAnyNorm, false>(x, y, h0, h1, n, r, cs, lane);
}

// Sixteen neighbouring lanes hold a head of 128 dimensions, a lane eight of them.  Where two lanes hold the halves of eight pairs, each takes four of the pairs, so that every value is normed
// once: dimensions d1 .. d1 + 3 and d2 .. d2 + 3.
struct Sixteenth {
    int sub, half, d1, d2;               // half: vectors of eight in half of the rotated part
    bool turned, swap, low;
    __device__ __forceinline__ Sixteenth(const RopePlan& r, int lane) : sub(lane & 15), half(r.rot / 16)
    {
        turned = 8 * sub < r.rot;
        swap = turned && !r.interleaved;
        low = sub < half;
        d1 = !swap || low ? 8 * sub : 8 * (sub - half) + 4;
        d2 = !swap ? d1 + 4 : d1 + r.rot / 2;
    }
};
struct SixteenthWeights {
    f16x4 w1, w2;
};
__device__ __forceinline__ SixteenthWeights sixteenth_weights(const HeadNorm& n, int h, const Sixteenth& s)
{
    SixteenthWeights w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w.w1[i] = w.w2[i] = (_Float16)1.0f;
    if (n.w) {
        w.w1 = *(const f16x4*)(n.w + h * n.stride + s.d1);
        w.w2 = *(const f16x4*)(n.w + h * n.stride + s.d2);
    }
    return w;
}

// What a lane keeps of the norm of a head's sixteenth; nothing where heads are not normed.
template <class Heads>
struct SixteenthNorm {
    __device__ __forceinline__ SixteenthNorm(const RopePlan&, int) {}
};
template <>
struct SixteenthNorm<AppendHeads> {
    Sixteenth at;
    SixteenthWeights w;
    __device__ __forceinline__ SixteenthNorm(const RopePlan& r, int lane) : at(r, lane), w{} {}
    __device__ __forceinline__ void request(const HeadNorm& n, int h) { w = sixteenth_weights(n, h, at); }
};

// The lane's dimensions 8 * sub ..; cs without gaps.
__device__ __forceinline__ u32x4 head_sixteenth(u32x4 raw, const SixteenthWeights& w, const Sixteenth& s, const HeadNorm& n, const RopePlan& r, const CosSin* cs, int lane)
{
    if (!n.on) return r.rot ? rope_sixteenth(raw, r, cs, lane) : raw;
    const bool turned = s.turned, swap = s.swap, low = s.low;
    const int partner = swap ? (lane & ~15) | (low ? s.sub + s.half : s.sub - s.half) : lane;
    u32x2 first = {raw[0], raw[1]}, second = {raw[2], raw[3]};
    if (r.rot && !r.interleaved) {                           // (uniform)
        const u32x2 out = low ? second : first;
        const u32x2 in = {(uint32_t)__shfl((int)out[0], partner), (uint32_t)__shfl((int)out[1], partner)};
        if (swap && low) second = in;
        if (swap && !low) first = in;
    }
    const f16x4 a = __builtin_bit_cast(f16x4, first), b = __builtin_bit_cast(f16x4, second);
    double x[8], mean, factor;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (double)(float)a[i], x[4 + i] = (double)(float)b[i];
    if (n.centred) head_norm<16, true>(x, true, true, n, mean, factor);
    else head_norm<16, false>(x, true, true, n, mean, factor);
    const double least = n.offset * factor;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (x[i] - mean) * weight_of(i < 4 ? w.w1[i & 3] : w.w2[i & 3], factor, least);
    if (turned) {
        const CosSin* const mine = cs + (r.interleaved ? 4 * s.sub : s.d1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const CosSin c = mine[i];
            if (r.interleaved) {
                const double u = x[2 * i], v = x[2 * i + 1];
                x[2 * i] = u * c.c - v * c.s;
                x[2 * i + 1] = v * c.c + u * c.s;
            } else {
                const double u = x[i], v = x[4 + i];
                x[i] = u * c.c - v * c.s;
                x[4 + i] = v * c.c + u * c.s;
            }
        }
    }
    f16x4 y1, y2;
#pragma unroll
    for (int i = 0; i < 4; ++i) y1[i] = rope_round(x[i]), y2[i] = rope_round(x[4 + i]);
    first = __builtin_bit_cast(u32x2, y1), second = __builtin_bit_cast(u32x2, y2);
    if (r.rot && !r.interleaved) {
        const u32x2 out = low ? second : first;
        const u32x2 in = {(uint32_t)__shfl((int)out[0], partner), (uint32_t)__shfl((int)out[1], partner)};
        if (swap && low) second = in;
        if (swap && !low) first = in;
    }
    return u32x4{first[0], first[1], second[0], second[1]};
}

}  // namespace tmw4
