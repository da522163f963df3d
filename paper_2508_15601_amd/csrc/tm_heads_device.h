// Norms of heads and their rotation on the device: what the kernel of packed tokens (tm_heads.hip) and the append to pages (tm_paged_append_impl.h) share.
//
//     n = (x - m) * (offset + w) / sqrt(mean((x - m)^2) + eps),    m = 0 or mean(x) over the head,    y = rotate(n)
//
// in 64 bits throughout, like the rotation alone (tm_rope_device.h): a head's sums are then right to the last bits of 53, the result is the fp16 number next to the true one, and a key
// gets the same codes wherever it is normed.  In 32 bits the factor would be off by up to 2^-23, which moves one fp16 value in about 4000 and one 8-bit code in 10^5.
#pragma once
#include "tm_rope_device.h"

namespace tmw4 {

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

__device__ __forceinline__ f16x8 head_weights(const HeadNorm& n, int head, int d)
{
    f16x8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (_Float16)1.0f;
    if (n.w) w = *(const f16x8*)(n.w + head * n.stride + d);
    return w;
}

// Sixteen dimensions of a head, which a lane holds in two vectors: the eight pairs of one stretch of the rotated part, or a stretch that is not turned, which may
// end after eight.
struct HeadPart {
    int d0, d1;
    bool turned, any, whole;             // whole: the second vector is there too
    __device__ __forceinline__ HeadPart(int u, int dim, const RopePlan& r)
    {
        any = 16 * u < dim;
        whole = 16 * u + 8 < dim;
        turned = 16 * u < r.rot;
        d0 = !any ? 0 : turned && !r.interleaved ? 8 * u : 16 * u;
        d1 = !any ? 0 : turned && !r.interleaved ? 8 * u + r.rot / 2 : whole ? 16 * u + 8 : d0;
    }
};

// Norms of the heads of a launch: none, those without a mean, any.
constexpr int kNoNorm = 0, kPlainNorm = 1, kAnyNorm = 2;

// Cosines and sines in LDS: eight pairs, which a lane reads, begin 144 bytes behind the eight before them, so that the lanes of a head meet no banks of each other's.
__device__ __forceinline__ int turn_at(int pair) { return pair + pair / 8; }
constexpr int turns_of(int pairs) { return pairs + pairs / 8; }

// a, b: the part's vectors, wa, wb: their weights; cs: cosines and sines of the part's pairs.  Every lane of a head takes part.
template <int LANES, int MODE, bool INTERLEAVED>
__device__ __forceinline__ void head_turn(f16x8& a, f16x8& b, const f16x8& wa, const f16x8& wb, const HeadPart& p, const HeadNorm& n, const CosSin* cs)
{
    constexpr int STEP = INTERLEAVED ? 2 : 1, OTHER = INTERLEAVED ? 1 : 8;           // of a pair's values
    if ((MODE == kNoNorm || !n.on) && !p.turned) return;
    double x[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (double)(float)a[i], x[8 + i] = (double)(float)b[i];
    if (MODE != kNoNorm && n.on) {
        double mean, factor;
        head_norm<LANES, MODE == kAnyNorm>(x, p.any, p.whole, n, mean, factor);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = (MODE == kAnyNorm ? x[i] - mean : x[i]) * (factor * (n.offset + (double)(float)(i < 8 ? wa[i & 7] : wb[i & 7])));
    }
    if (p.turned) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const CosSin t = cs[i];
            const double u = x[STEP * i], v = x[STEP * i + OTHER];
            x[STEP * i] = u * t.c - v * t.s;
            x[STEP * i + OTHER] = v * t.c + u * t.s;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = rope_round(x[i]), b[i] = rope_round(x[8 + i]);
}

// Heads h0 .. h1 - 1 of 128 dimensions of one token, by one wave; x and y may be the same; cs as turn_at() has it.
template <int MODE, bool INTERLEAVED>
__device__ __forceinline__ void turn_heads(const uint16_t* x, uint16_t* y, int h0, int h1, const HeadNorm& n, const RopePlan& r, const CosSin* cs, int lane)
{
    const HeadPart part(lane & 7, 128, r);
    for (int at = h0; at < h1; at += 8) {
        const int h = min(at + (lane >> 3), h1 - 1);
        const uint16_t* const from = x + (size_t)h * 128;
        f16x8 a = *(const f16x8*)(from + part.d0), b = *(const f16x8*)(from + part.d1);
        head_turn<8, MODE, INTERLEAVED>(a, b, head_weights(n, h, part.d0), head_weights(n, h, part.d1), part, n, cs + turn_at(8 * (lane & 7)));
        if (at + (lane >> 3) >= h1) continue;
        *(f16x8*)(y + (size_t)h * 128 + part.d0) = a;
        *(f16x8*)(y + (size_t)h * 128 + part.d1) = b;
    }
}
__device__ __forceinline__ void turn_heads(const uint16_t* x, uint16_t* y, int h0, int h1, const HeadNorm& n, const RopePlan& r, const CosSin* cs, int lane)
{
    if (!n.centred && r.interleaved) turn_heads<kPlainNorm, true>(x, y, h0, h1, n, r, cs, lane);
    else if (!n.centred) turn_heads<kPlainNorm, false>(x, y, h0, h1, n, r, cs, lane);
    else if (r.interleaved) turn_heads<kAnyNorm, true>(x, y, h0, h1, n, r, cs, lane);
    else turn_heads<kAnyNorm, false>(x, y, h0, h1, n, r, cs, lane);
}

// A lane's eight dimensions 8 * sub .. of head h of 128 dimensions that sixteen neighbouring lanes hold.
__device__ __forceinline__ u32x4 head_sixteenth(u32x4 raw, int h, const HeadNorm& n, const RopePlan& r, const CosSin* cs, int lane)
{
    if (!n.on) return r.rot ? rope_sixteenth(raw, r, cs, lane) : raw;
    const int sub = lane & 15, half = r.rot / 16;            // vectors of eight in half of the rotated part
    const bool turned = 8 * sub < r.rot, low = sub < half;
    const int partner = r.interleaved || !turned ? sub : low ? sub + half : sub - half;
    u32x4 other = raw;
    if (r.rot && !r.interleaved) {                           // (uniform)
#pragma unroll
        for (int i = 0; i < 4; ++i) other[i] = (uint32_t)__shfl((int)raw[i], (lane & ~15) | partner);
    }
    const f16x8 a = __builtin_bit_cast(f16x8, raw), b = __builtin_bit_cast(f16x8, other), wa = head_weights(n, h, 8 * sub), wb = head_weights(n, h, 8 * partner);
    double x[8], mean, factor;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (double)(float)a[i];
    head_norm<16, true>(x, true, true, n, mean, factor);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (x[i] - mean) * (factor * (n.offset + (double)(float)wa[i]));
    f16x8 y;
    if (turned && r.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const CosSin c = cs[4 * sub + i];
            y[2 * i] = rope_round(x[2 * i] * c.c - x[2 * i + 1] * c.s);
            y[2 * i + 1] = rope_round(x[2 * i + 1] * c.c + x[2 * i] * c.s);
        }
    } else if (turned) {
        const CosSin* const mine = cs + 8 * (low ? sub : sub - half);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double z = ((double)(float)b[i] - mean) * (factor * (n.offset + (double)(float)wb[i]));
            y[i] = rope_round(x[i] * mine[i].c + (low ? -z : z) * mine[i].s);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = rope_round(x[i]);
    }
    return __builtin_bit_cast(u32x4, y);
}

}  // namespace tmw4
