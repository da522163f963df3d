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
    double eps, offset;
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

// Mean (0 unless centred) and factor of a head of dim values, `count` of them this lane's.
template <int LANES, int N>
__device__ __forceinline__ void head_norm(const double (&x)[N], int count, const HeadNorm& n, int dim, double& mean, double& factor)
{
    const bool full = dim == LANES * N;                      // (uniform) every lane has N
    const double share = 1.0 / dim;
    mean = 0.0;
    double s = 0.0;
    if (n.centred) {
#pragma unroll
        for (int i = 0; i < N; ++i) s += full || i < count ? x[i] : 0.0;
        mean = lanes_sum<LANES>(s) * share;
        s = 0.0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const double d = x[i] - mean;
            s += full || i < count ? d * d : 0.0;
        }
    } else if (full) {
#pragma unroll
        for (int i = 0; i < N; ++i) s = __builtin_fma(x[i], x[i], s);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) s += i < count ? x[i] * x[i] : 0.0;
    }
    factor = inverse_root(__builtin_fma(lanes_sum<LANES>(s), share, n.eps));
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

// a, b: the part's vectors, wa, wb: their weights; cs: cosines and sines of the token's pairs.  Every lane of a head takes part.
template <int LANES, bool NORM, bool INTERLEAVED>
__device__ __forceinline__ void head_turn(f16x8& a, f16x8& b, const f16x8& wa, const f16x8& wb, const HeadPart& p, const HeadNorm& n, int dim, const CosSin (&cs)[8])
{
    double x[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (double)(float)a[i], x[8 + i] = (double)(float)b[i];
    if constexpr (NORM) {
        double mean, factor;
        head_norm<LANES>(x, !p.any ? 0 : p.whole ? 16 : 8, n, dim, mean, factor);
        if (n.centred) {                                     // (uniform)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] -= mean;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= factor * (n.offset + (double)(float)(i < 8 ? wa[i] : wb[i - 8]));
    }
    if (p.turned) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            constexpr int STEP = INTERLEAVED ? 2 : 1, OTHER = INTERLEAVED ? 1 : 8;
            const double u = x[STEP * i], v = x[STEP * i + OTHER];
            x[STEP * i] = u * cs[i].c - v * cs[i].s;
            x[STEP * i + OTHER] = v * cs[i].c + u * cs[i].s;
        }
    } else if (!NORM) {
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = rope_round(x[i]), b[i] = rope_round(x[8 + i]);
}

// Heads h0 .. h1 - 1 of 128 dimensions of one token, by one wave; x and y may be the same.
template <bool NORM, bool INTERLEAVED>
__device__ __forceinline__ void turn_heads(const uint16_t* x, uint16_t* y, int h0, int h1, const HeadNorm& n, const HeadPart& part, const CosSin (&c)[8], int lane)
{
    f16x8 wa = head_weights(n, h0, part.d0), wb = head_weights(n, h0, part.d1);
    for (int at = h0; at < h1; at += 8) {
        const int h = min(at + (lane >> 3), h1 - 1);
        const uint16_t* const from = x + (size_t)h * 128;
        f16x8 a = *(const f16x8*)(from + part.d0), b = *(const f16x8*)(from + part.d1);
        if (n.stride) wa = head_weights(n, h, part.d0), wb = head_weights(n, h, part.d1);
        head_turn<8, NORM, INTERLEAVED>(a, b, wa, wb, part, n, 128, c);
        if (at + (lane >> 3) >= h1) continue;
        *(f16x8*)(y + (size_t)h * 128 + part.d0) = a;
        *(f16x8*)(y + (size_t)h * 128 + part.d1) = b;
    }
}
__device__ __forceinline__ void turn_heads(const uint16_t* x, uint16_t* y, int h0, int h1, const HeadNorm& n, const RopePlan& r, const CosSin* cs, int lane)
{
    const HeadPart part(lane & 7, 128, r);
    CosSin c[8] = {};
    if (part.turned) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = cs[8 * (lane & 7) + i];
    }
    if (n.on && r.interleaved) turn_heads<true, true>(x, y, h0, h1, n, part, c, lane);
    else if (n.on) turn_heads<true, false>(x, y, h0, h1, n, part, c, lane);
    else if (r.interleaved) turn_heads<false, true>(x, y, h0, h1, n, part, c, lane);
    else turn_heads<false, false>(x, y, h0, h1, n, part, c, lane);
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
    head_norm<16>(x, 8, n, 128, mean, factor);
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
