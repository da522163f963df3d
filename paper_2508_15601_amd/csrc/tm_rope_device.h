// Rotary positions on the device: angles without loss at any position, and the rotation of a pair.
//
// An angle pos * f is kept in turns.  Of a frequency the whole turns a position are left out on the host and the rest F is held to 96 bits: pos * F less its whole turns is the
// angle, and the integer multiplication, whose upper bits run over, does the argument reduction that a floating-point sine has to do.  At 2^31 an F of 64 bits would be
// off by up to 7e-10 radians, this one by less than 1e-18: the product is kept to 2^-64 of a turn.
// Sine and cosine are their power series on an eighth of a turn to either side of the nearest quarter (largest error 7e-12), in 64 bits: this
// chip adds and multiplies 64-bit floats at the rate of 32-bit ones.  A rotated value is then the fp16 number next to the true one (as good as always),
// which matters where it is quantised afterwards: an error of 2^-24 moves one code in about 3 million.
#pragma once
#include "tm_w4_device.h"

namespace tmw4 {

constexpr int kRopeMaxPairs = 128;       // head dimensions up to 256

struct RopeTurn {                        // a fraction of a turn
    uint64_t high;                       // in units of 2^-64
    uint32_t low;                        // and of 2^-96
};

struct RopePlan {
    const RopeTurn* turns;               // [rot / 2] F of every pair (device)
    double amp;                          // factor of the rotated values
    int rot;                             // dimensions that are rotated, a multiple of 16
    int interleaved;                     // pairs are (2i, 2i + 1); otherwise (i, i + rot / 2)
};

struct CosSin {
    double c, s;
};

__device__ __forceinline__ CosSin rope_angle(const RopePlan& r, int pos, const RopeTurn& turn)
{
    const uint64_t phase = (uint64_t)(int64_t)pos * turn.high + (uint64_t)(((int64_t)pos * (int64_t)turn.low) >> 32);
    const uint32_t quarter = (uint32_t)((phase + (1ull << 61)) >> 62) & 3u;           // nearest quarter turn
    const int64_t rest = (int64_t)(phase - ((uint64_t)quarter << 62));                // within 2^61 of it
    const double x = ((double)(int32_t)(rest >> 32) * 4294967296.0 + (double)(uint32_t)rest) * 0x1.921fb54442d18p-62;      // 2 pi / 2^64
    const double y = x * x;
    // sum of (-1)^n y^n / (2n + 1)! and of (-1)^n y^n / (2n)!
    const double sin_x = x * (1.0 + y * (-1.0 / 6 + y * (1.0 / 120 + y * (-1.0 / 5040 + y * (1.0 / 362880 + y * (-1.0 / 39916800))))));
    const double cos_x = 1.0 + y * (-1.0 / 2 + y * (1.0 / 24 + y * (-1.0 / 720 + y * (1.0 / 40320 + y * (-1.0 / 3628800 + y * (1.0 / 479001600))))));
    const double a = quarter & 1u ? sin_x : cos_x, b = quarter & 1u ? cos_x : sin_x;
    return CosSin{r.amp * (quarter == 1u || quarter == 2u ? -a : a), r.amp * (quarter & 2u ? -b : b)};
}

// To fp16 through fp32, on every path alike.  (Left to itself the compiler rounds some of them directly, which differs where the fp32 value is a tie
// of fp16: one value in 2^14.  The same key has to give the same codes wherever it is rotated.)
__device__ __forceinline__ _Float16 rope_round(double x)
{
    float f = (float)x;
    asm("" : "+v"(f));
    return (_Float16)f;
}

// Rotates the pairs (a[i], b[i]) of eight values each by cs[i].
__device__ __forceinline__ void rope_pairs(f16x8& a, f16x8& b, const CosSin (&cs)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double x = (double)(float)a[i], y = (double)(float)b[i];
        a[i] = rope_round(x * cs[i].c - y * cs[i].s);
        b[i] = rope_round(y * cs[i].c + x * cs[i].s);
    }
}

// Cosines and sines of a token's pairs, by one wave.
__device__ __forceinline__ void rope_angles(CosSin* cs, const RopePlan& r, int pos, int lane)
{
    for (int i = lane; i < r.rot / 2; i += 64) cs[i] = rope_angle(r, pos, r.turns[i]);
}

// Heads h0 .. h1 - 1 of one token, by one wave: x -> y (which may be the same).  A lane takes sixteen dimensions at a time: the eight pairs of
// two vectors of eight, or a stretch that is copied; sixteen-byte accesses throughout.
__device__ __forceinline__ void rope_heads(const uint16_t* x, uint16_t* y, int h0, int h1, int dim, const RopePlan& r, const CosSin* cs, int lane)
{
    const int per = (dim + 15) / 16, turned = r.rot / 16;
    for (int at = lane; at < (h1 - h0) * per; at += 64) {
        const int h = at / per, u = at - h * per;
        const size_t head = (size_t)(h0 + h) * dim;
        const bool whole = u * 16 + 8 < dim;                 // the copied stretch may end after eight dimensions
        const int d0 = u < turned && !r.interleaved ? 8 * u : 16 * u;
        const int d1 = u < turned && !r.interleaved ? 8 * u + r.rot / 2 : whole ? 16 * u + 8 : d0;
        f16x8 a = *(const f16x8*)(x + head + d0), b = *(const f16x8*)(x + head + d1);
        if (u < turned) {
            CosSin c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = cs[8 * u + i];
            if (r.interleaved) {
                f16x8 even = {a[0], a[2], a[4], a[6], b[0], b[2], b[4], b[6]}, odd = {a[1], a[3], a[5], a[7], b[1], b[3], b[5], b[7]};
                rope_pairs(even, odd, c);
                a = f16x8{even[0], odd[0], even[1], odd[1], even[2], odd[2], even[3], odd[3]};
                b = f16x8{even[4], odd[4], even[5], odd[5], even[6], odd[6], even[7], odd[7]};
            } else {
                rope_pairs(a, b, c);
            }
        }
        *(f16x8*)(y + head + d0) = a;
        if (whole) *(f16x8*)(y + head + d1) = b;
    }
}

// A lane's eight dimensions 8 * sub .. of a 128-dimensional head that sixteen neighbouring lanes hold.
__device__ __forceinline__ u32x4 rope_sixteenth(u32x4 raw, const RopePlan& r, const CosSin* cs, int lane)
{
    const int sub = lane & 15, half = r.rot / 16;            // vectors of eight in half of the rotated part
    const f16x8 x = __builtin_bit_cast(f16x8, raw);
    f16x8 y;
    if (r.interleaved) {
        if (8 * sub >= r.rot) return raw;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const CosSin c = cs[4 * sub + i];
            const double a = (double)(float)x[2 * i], b = (double)(float)x[2 * i + 1];
            y[2 * i] = rope_round(a * c.c - b * c.s);
            y[2 * i + 1] = rope_round(b * c.c + a * c.s);
        }
        return __builtin_bit_cast(u32x4, y);
    }
    const bool low = sub < half;
    const int partner = (lane & ~15) | (sub >= 2 * half ? sub : low ? sub + half : sub - half);
    u32x4 other;
#pragma unroll
    for (int i = 0; i < 4; ++i) other[i] = (uint32_t)__shfl((int)raw[i], partner);
    if (sub >= 2 * half) return raw;
    const f16x8 z = __builtin_bit_cast(f16x8, other);
    const CosSin* const mine = cs + 8 * (low ? sub : sub - half);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double a = (double)(float)x[i], b = (double)(float)z[i];
        y[i] = rope_round(a * mine[i].c + (low ? -b : b) * mine[i].s);
    }
    return __builtin_bit_cast(u32x4, y);
}

}  // namespace tmw4
