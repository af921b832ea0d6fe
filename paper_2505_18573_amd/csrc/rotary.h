// Rotary positions: pair i of a head's columns is turned by theta_i = (position on the pair's axis) * f_i.
//
//   y1 = x1 cos theta - x2 sin theta,   y2 = x2 cos theta + x1 sin theta;   the gradient: by -theta.
//
// Angles: positions reach millions and f_0 is 1, so 32 bits would leave nothing of the angle behind the comma.  In turns
// (theta / 2 pi) the whole part drops out, and the product is taken in 64 bits with its own rounding error (fused
// multiply-add), so a position below 2^52 loses nothing; what is left, at most an eighth of a turn after the quadrant is
// taken off, goes into the Taylor polynomials of sine and cosine (degree 9 and 10: the next terms are below 2^-29 of the
// result).  Their leading terms are taken in 64 bits and the others, at most a tenth of those, in 32, so that either is off by little
// more than its own rounding to fp32.
// Keys on their way into the cache are turned in 64 bits throughout and rounded once: in eight bits an element that lies next to
// the border of two codes is a sixteenth larger or smaller by an error of one bit of fp32.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv_cache.h"

namespace e3 {

struct Rotary {
    const double* freqs;              // [rot / 2] radians per position
    const uint8_t* axis;              // [rot / 2] or nullptr: axis 0
    const int64_t* positions;         // [axes][tokens], rows `stride` apart
    int64_t stride;
    int32_t rot, axes;
    bool neighbours;                  // pairs (2 i, 2 i + 1) instead of (i, i + rot / 2)
    float sign;                       // -1: by the opposite angles
};

// Queries (or any rows of heads) that are turned: [tokens][heads][dim], columns next to each other.
struct TurnArgs {
    TokenRows x;
    void* out;
    int64_t out_token_stride, out_head_stride;
    int64_t tokens;
    int32_t heads, dim;
};

hipError_t launch_rotate(const TurnArgs& a, const Rotary& r, bool bf16, hipStream_t stream);
// keys turned and values as they are into the cache, and, where q.heads > 0, queries turned
hipError_t launch_cache_append_rotated(const CacheView& c, const TokenRows& k, const TokenRows& v, const TurnArgs& q, const Rotary& r,
                                       bool in_bf16, const int64_t* slots, int64_t tokens, hipStream_t stream);

// What the angle of pair i at a token is made of.  is: false where the pair goes by no axis and stays as it is.
struct Place {
    double at, freq;
    bool is;
};
__device__ __forceinline__ Place place_of(const Rotary& r, int64_t token, int i)
{
    const int axis = r.axis == nullptr ? 0 : r.axis[i];
    const bool is = axis < r.axes;
    return Place{(double)r.positions[(is ? axis : 0) * r.stride + token], r.freqs[i], is};
}
// The angle: quarter turns taken off, at most pi / 4 left.
__device__ __forceinline__ double angle_of(const Place& p, int* quarters)
{
    constexpr double kHi = 0.15915494309189533577, kLo = -9.839338337591243e-18;    // 1 / (2 pi) in two parts
    const double g = p.freq * kHi, g_rest = fma(p.freq, kHi, -g) + p.freq * kLo;
    const double x = p.at * g, x_rest = fma(p.at, g, -x) + p.at * g_rest;
    const double turn = (x - rint(x)) + x_rest;                   // in [-1/2, 1/2], and x_rest
    const double quarter = rint(turn * 4.0);
    *quarters = (int)quarter;
    return (turn - quarter * 0.25) * 6.28318530717958647693;
}
template <typename T>
__device__ __forceinline__ void by_quarters(int q, float sign, T& c, T& s)
{
    const T cs = (q & 1) ? s : c, sn = (q & 1) ? c : s;
    c = ((q + 1) & 2) ? -cs : cs;
    s = ((q & 2) ? -sn : sn) * (T)sign;
}

// (cos, sin) at a place, in 32 bits
__device__ __forceinline__ float2 turn_of(const Place& p, float sign)
{
    if (!p.is) return float2{1.0f, 0.0f};
    int quarters;
    const double angle = angle_of(p, &quarters);
    const float z = (float)angle, z2 = z * z;
    float p_s = 1.0f / 362880.0f, p_c = -1.0f / 3628800.0f;
    p_s = fmaf(p_s, z2, -1.0f / 5040.0f);
    p_s = fmaf(p_s, z2, 1.0f / 120.0f);
    p_s = fmaf(p_s, z2, -1.0f / 6.0f);
    p_c = fmaf(p_c, z2, 1.0f / 40320.0f);
    p_c = fmaf(p_c, z2, -1.0f / 720.0f);
    p_c = fmaf(p_c, z2, 1.0f / 24.0f);
    float s = (float)(angle + (double)(z2 * z * p_s));
    float c = (float)(fma(angle * angle, -0.5, 1.0) + (double)(z2 * z2 * p_c));
    by_quarters(quarters, sign, c, s);
    return float2{c, s};
}

// The same in 64 bits (series up to z^15 and z^16: the next terms are below 2^-54).
__device__ __forceinline__ double2 turn64_of(const Place& p, float sign)
{
    if (!p.is) return double2{1.0, 0.0};
    int quarters;
    const double z = angle_of(p, &quarters);
    const double z2 = z * z;
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
    s = fma(s, z2, 1.0 / 6227020800.0);
    c = fma(c, z2, -1.0 / 87178291200.0);
    s = fma(s, z2, -1.0 / 39916800.0);
    c = fma(c, z2, 1.0 / 479001600.0);
    s = fma(s, z2, 1.0 / 362880.0);
    c = fma(c, z2, -1.0 / 3628800.0);
    s = fma(s, z2, -1.0 / 5040.0);
    c = fma(c, z2, 1.0 / 40320.0);
    s = fma(s, z2, 1.0 / 120.0);
    c = fma(c, z2, -1.0 / 720.0);
    s = fma(s, z2, -1.0 / 6.0);
    c = fma(c, z2, 1.0 / 24.0);
    s = fma(s * z2, z, z);
    c = fma(c, z2, -0.5);
    c = fma(c, z2, 1.0);
    by_quarters(quarters, sign, c, s);
    return double2{c, s};
}

// x in fp32 such that rounding it on to fewer bits gives what rounding x itself would: towards zero, and odd where that was not exact.
__device__ __forceinline__ float sticky(double x)
{
    const float f = (float)x;
    const double back = (double)f;
    uint32_t bits = __float_as_uint(f);
    if (back != x && fabsf(f) < INFINITY) {                       // (NaN differs from itself, and keeps its bits)
        if (fabs(back) > fabs(x)) bits -= 1;
        bits |= 1u;
    }
    return __uint_as_float(bits);
}

// A unit: up to 16 columns of one token and head, in two vectors of eight; those that are turned hold pairs 8 u .. 8 u + 7.
template <bool kBf16>
struct Eight {
    float x[8];
    __device__ __forceinline__ void load(const char* p)
    {
        if (kBf16) {
            const uint4 w = *reinterpret_cast<const uint4*>(p);
            const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(v[j] << 16); x[2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u); }
        } else {
            const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 16);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        }
    }
    __device__ __forceinline__ void store(char* p) const
    {
        if (kBf16) {
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                typedef __bf16 pair __attribute__((ext_vector_type(2)));
                const pair w = {(__bf16)x[2 * j], (__bf16)x[2 * j + 1]};
                v[j] = __builtin_bit_cast(uint32_t, w);
            }
            *reinterpret_cast<uint4*>(p) = uint4{v[0], v[1], v[2], v[3]};
        } else {
            *reinterpret_cast<float4*>(p) = float4{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<float4*>(p + 16) = float4{x[4], x[5], x[6], x[7]};
        }
    }
};

__host__ __device__ __forceinline__ int units_of(int rot, int dim) { return rot / 16 + (dim - rot + 15) / 16; }

// Unit u of (token, head), as it comes; `by`: (cos, sin) of pairs 8 u .. 8 u + 7 (any, where the unit is not turned).
template <bool kBf16>
struct Unit {
    Eight<kBf16> v, w;
    static __device__ __forceinline__ void columns(const Rotary& r, int u, int* first, int* second)
    {
        const int turned = r.rot / 16;
        const bool pairs = u < turned && !r.neighbours;           // two vectors half the turned columns apart, else next to each other
        *first = pairs ? 8 * u : u < turned ? 16 * u : r.rot + (u - turned) * 16;
        *second = pairs ? *first + r.rot / 2 : *first + 8;
    }
    __device__ __forceinline__ void load(const TurnArgs& a, const Rotary& r, int64_t token, int head, int u)
    {
        constexpr int kSize = kBf16 ? 2 : 4;
        const char* x = static_cast<const char*>(a.x.base) + (token * a.x.token_stride + head * a.x.head_stride) * kSize;
        int first, second;
        columns(r, u, &first, &second);
        v.load(x + first * kSize);
        if (second < a.dim) w.load(x + second * kSize);
    }
    __device__ __forceinline__ void store(const TurnArgs& a, const Rotary& r, int64_t token, int head, int u, const float2 by[8])
    {
        constexpr int kSize = kBf16 ? 2 : 4;
        char* out = static_cast<char*>(a.out) + (token * a.out_token_stride + head * a.out_head_stride) * kSize;
        int first, second;
        columns(r, u, &first, &second);
        if (u < r.rot / 16) {
            if (r.neighbours) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 t = by[j], s = by[4 + j];
                    const float v0 = v.x[2 * j], w0 = w.x[2 * j];
                    v.x[2 * j] = v0 * t.x - v.x[2 * j + 1] * t.y;
                    v.x[2 * j + 1] = v.x[2 * j + 1] * t.x + v0 * t.y;
                    w.x[2 * j] = w0 * s.x - w.x[2 * j + 1] * s.y;
                    w.x[2 * j + 1] = w.x[2 * j + 1] * s.x + w0 * s.y;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 t = by[j];
                    const float v0 = v.x[j];
                    v.x[j] = v0 * t.x - w.x[j] * t.y;
                    w.x[j] = w.x[j] * t.x + v0 * t.y;
                }
            }
        }
        v.store(out + first * kSize);
        if (second < a.dim) w.store(out + second * kSize);
    }
};

}  // namespace e3
