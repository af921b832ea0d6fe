// What the attention kernels share: a step of 32 tokens as a wave takes it from the cache, and small helpers.
#pragma once
#include "kv_cache.h"
#include "vocab_common.h"

namespace e3 {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kStep = 32;                       // tokens of a wave's step
constexpr float kNoScore = -3.0e38f;            // running maximum before any score
constexpr float kSlack = 8.0f;                  // scores may pass the running maximum by this (2^8) before it moves

__device__ __forceinline__ int clamp_len(int n, int64_t most) { return n < 0 ? 0 : n > most ? (int)most : n; }
// tokens that a table of `width` pages can name
__device__ __forceinline__ int64_t table_tokens(int width, int page_size)
{
    const int64_t n = (int64_t)width * page_size;
    return n > 0x7F000000 ? 0x7F000000 : n;                                    // steps beyond it stay in 32 bits
}

// The same in every lane: kept in scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v)
{
    return (int64_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v);
}

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// eight e4m3 codes as bf16 (exact)
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// One step of 32 tokens as it comes from memory.  Lane (m, g) = (lane & 15, lane >> 4).
template <int D, bool kFp8>
struct StepData {
    static constexpr int kLoads = kFp8 ? D / 64 : D / 32;              // of 16 bytes, per row of K
    static constexpr int kVLoads = kFp8 ? D / 32 : D / 16;
    u32x4 k[2][kLoads];
    u32x4 v[kVLoads];
    u32x2 ks, vs;                                                       // scale bytes of tokens 8 g .. 8 g + 7

    // `row`: index of the step's first token among the rows of D elements
    __device__ __forceinline__ void load_keys(const CacheView& c, int64_t row, int lane)
    {
        const int m = lane & 15, g = lane >> 4;
        constexpr int kElem = kFp8 ? 1 : 2;
        const char* kp = static_cast<const char*>(c.k) + row * (D * kElem) + (8 * (m >> 2) + (m & 3)) * (D * kElem) + g * 16;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) k[t][i] = (*reinterpret_cast<const u32x4*>(kp + t * 4 * (D * kElem) + i * 64));
        if (kFp8) ks = *reinterpret_cast<const u32x2*>(c.k_scale + row + g * 8);
    }
    __device__ __forceinline__ void load_values(const CacheView& c, int64_t row, int lane)
    {
        const int m = lane & 15, g = lane >> 4;
        constexpr int kElem = kFp8 ? 1 : 2;
        const char* vp = static_cast<const char*>(c.v) + row * (D * kElem) + g * (8 * D * kElem) + m * 16;
#pragma unroll
        for (int i = 0; i < kVLoads; ++i) v[i] = (*reinterpret_cast<const u32x4*>(vp + i * 256));
        if (kFp8) vs = *reinterpret_cast<const u32x2*>(c.v_scale + row + g * 8);
    }
    // A step in LDS: every lane's registers as they are, 64 lanes next to each other, and the factors of its tokens in fp32 (made
    // once for the four waves that read them: with the bytes 512 rows of five tokens take 13 us longer).
    static constexpr int kImage = (2 * kLoads + kVLoads) * 64 * 16 + (kFp8 ? 2 * kStep * 4 : 0);         // bytes
    __device__ __forceinline__ void put(char* to, float c, int lane) const
    {
        u32x4* w = reinterpret_cast<u32x4*>(to) + lane;
#pragma unroll
        for (int i = 0; i < 2 * kLoads; ++i) w[i * 64] = k[i / kLoads][i % kLoads];
#pragma unroll
        for (int i = 0; i < kVLoads; ++i) w[(2 * kLoads + i) * 64] = v[i];
        if (kFp8) {
            float* e = reinterpret_cast<float*>(to + (2 * kLoads + kVLoads) * 1024) + (lane >> 4) * 8;
            if ((lane & 15) == 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    e[j] = c * k_factor(j);
                    e[kStep + j] = v_factor(j);
                }
            }
        }
    }
    __device__ __forceinline__ void take(const char* from, int lane)
    {
        const u32x4* w = reinterpret_cast<const u32x4*>(from) + lane;
#pragma unroll
        for (int i = 0; i < 2 * kLoads; ++i) k[i / kLoads][i % kLoads] = w[i * 64];
#pragma unroll
        for (int i = 0; i < kVLoads; ++i) v[i] = w[(2 * kLoads + i) * 64];
    }
    // of a step in LDS
    static __device__ __forceinline__ const float* factors(const char* from, int lane)
    {
        return reinterpret_cast<const float*>(from + (2 * kLoads + kVLoads) * 1024) + (lane >> 4) * 8;
    }
    // K of score tile t, columns of k-step s
    __device__ __forceinline__ bf16x8 key(int t, int s) const
    {
        if (kFp8) {
            const u32x4 w = k[t][s >> 1];
            return (s & 1) ? widen(w.z, w.w) : widen(w.x, w.y);
        }
        return __builtin_bit_cast(bf16x8, k[t][s]);
    }
    // V^T of block b of 16 columns: which column row m of the block is, see column()
    __device__ __forceinline__ bf16x8 value(int b) const
    {
        if (kFp8) {
            const u32x4 w = v[b >> 1];
            return (b & 1) ? widen(w.z, w.w) : widen(w.x, w.y);
        }
        return __builtin_bit_cast(bf16x8, v[b]);
    }
    static __device__ __forceinline__ int key_column(int s, int g) { return kFp8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8; }
    static __device__ __forceinline__ int column(int b, int m) { return kFp8 ? (b >> 1) * 32 + 2 * m + (b & 1) : b * 16 + m; }

    // tokens of the lane's eight from the n-th on become zeros, in V and in both scales
    __device__ __forceinline__ void clear_from(int n)
    {
        if (kFp8) {
            const uint32_t lo = n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
            const uint32_t hi = n >= 8 ? 0xFFFFFFFFu : n <= 4 ? 0u : (1u << (8 * (n - 4))) - 1u;
#pragma unroll
            for (int i = 0; i < kVLoads; ++i) v[i] &= u32x4{lo, hi, lo, hi};
            ks &= u32x2{lo, hi};
            vs &= u32x2{lo, hi};
        } else {
            u32x4 mask;
#pragma unroll
            for (int j = 0; j < 4; ++j) mask[j] = n >= 2 * j + 2 ? 0xFFFFFFFFu : n == 2 * j + 1 ? 0xFFFFu : 0u;
#pragma unroll
            for (int i = 0; i < kVLoads; ++i) v[i] &= mask;
        }
    }
    // all bits of the elements of two (bf16) or four (codes) that are no finite number
    static __device__ __forceinline__ uint32_t unbounded_in(uint32_t w)
    {
        if (kFp8) return (((w & 0x7F7F7F7Fu) + 0x01010101u) >> 7 & 0x01010101u) * 0xFFu;   // 0x7F, 0xFF: the sum carries
        const uint32_t top = exponents_full(w);
        return (top - (top >> 15)) | top;
    }
    // the highest bit of each bf16 whose exponent is all ones (the addition carries into it)
    static __device__ __forceinline__ uint32_t exponents_full(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
    // whether the lane holds a value that is no finite number
    __device__ __forceinline__ bool unbounded() const
    {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < kVLoads; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) bad |= kFp8 ? unbounded_in(v[i][j]) : exponents_full(v[i][j]);
        return bad != 0;
    }
    // such values of `from` as ones, all others as zeros; they are zeros in `from` afterwards
    __device__ __forceinline__ void take_unbounded(StepData& from)
    {
#pragma unroll
        for (int i = 0; i < kVLoads; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t bad = unbounded_in(from.v[i][j]);
                v[i][j] = bad & (kFp8 ? 0x38383838u : 0x3F803F80u);
                from.v[i][j] &= ~bad;
            }
    }
    __device__ __forceinline__ float k_factor(int j) const { return __uint_as_float(((ks[j >> 2] >> (8 * (j & 3))) & 0xFFu) << 23); }
    __device__ __forceinline__ float v_factor(int j) const { return __uint_as_float(((vs[j >> 2] >> (8 * (j & 3))) & 0xFFu) << 23); }
};

}  // namespace e3
