// Writing keys and values into the paged cache and reading them back (layout: kv_cache.h).
//
// 8-bit form, per token, head and tensor, x the D elements:
//   a = largest finite |x|,  e = the smallest integer in [-126, 127] with a <= 448 * 2^e,
//   code = x * 2^-e rounded to e4m3 (nearest, ties to even),  value = code * 2^e.
// The scale is a power of two, because an arbitrary one would gain nothing (e4m3 is a floating-point format: a factor
// within a binade moves no value closer) and would cost a rounding on either side; this way scaling is exact, a value
// that is read back and written again keeps its bits, and the attention may apply the scale to sums instead of
// elements.  448 is e4m3's largest value, so nothing saturates.  Elements that are not finite become the NaN code and
// leave the scale of the others alone.
//
// One wave takes eight successive tokens of the call ("window") and one head (two heads where D = 64): lane
// (half, part) holds four columns of tokens 4 half .. 4 half + 3, so a token's row is 256 contiguous bytes of bf16 and
// its maximum is a reduction over 32 (16) lanes.  Keys are written row by row.  Values go eight tokens to a block: where
// eight tokens of the call fill a block (a prompt does that all along, wherever it starts in the call), the wave
// in whose window they start has their values transposed in registers and writes the block whole; a token whose
// block is not filled by its neighbours is written element by element.
//
// What bounds it: memory for prompts (60,001 tokens x 4 heads of 128: 123 MB of bf16 into 62 MB of codes 42 us, 4.4 TB/s; back
// 31 us, 6.0 TB/s, part of the codes still in the memory-side cache), the launch and its chain of two loads (slot, row) for a step's
// tokens (512: 5.4 us in, 4.3 us back).
#include "kv_cache.h"
#include "vocab_common.h"
#include "vocab_pass.h"

namespace e3 {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kBlockTokens = 8;
constexpr int kCacheWaves = 2;                  // of a workgroup at most

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const bf16x2 p = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, p);
}

// four successive elements as fp32
template <bool kBf16>
__device__ __forceinline__ void load4(const char* p, float x[4])
{
    if (kBf16) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(p);
        x[0] = __uint_as_float(w.x << 16); x[1] = __uint_as_float(w.x & 0xFFFF0000u);
        x[2] = __uint_as_float(w.y << 16); x[3] = __uint_as_float(w.y & 0xFFFF0000u);
    } else {
        const float4 w = *reinterpret_cast<const float4*>(p);
        x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w;
    }
}

// maximum over the lanes that hold one token's row: 16 lanes for D = 64, 32 for D = 128; in each of them
template <int D>
__device__ __forceinline__ float row_max(float v)
{
    v = fmaxf(v, dpp_f<kDppXor1>(v, v));
    v = fmaxf(v, dpp_f<kDppXor2>(v, v));
    v = fmaxf(v, dpp_f<kDppHalfMirror>(v, v));
    v = fmaxf(v, dpp_f<kDppMirror>(v, v));
    if (D == 128) v = fmaxf(v, __shfl_xor(v, 16));
    return v;
}

// e of a row whose largest finite magnitude is a: a = 1.m * 2^k; 448 = 1.75 * 2^8.
__device__ __forceinline__ int exponent_for(float a)
{
    const uint32_t bits = __float_as_uint(a);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e < -126 ? -126 : e;                                   // a < 2^128: e <= 120
}

struct Window {
    int64_t slot;           // of token `first - 7 + lane`, -1: none (out of the call, out of the cache)
    uint32_t whole;         // bit i: the block of window token i is filled by tokens of the call
    int start;              // window token whose block starts and is filled here, -1: none
};

// What the wave needs to know about its window: the slots of 7 tokens before it, its own 8 and 7 after it, and from
// them which blocks are filled.  (Block starts lie at least eight tokens apart: a window holds one at most.)
__device__ __forceinline__ Window look_at(const int64_t* slots, int64_t first, int64_t tokens, int64_t capacity, int lane)
{
    Window w;
    const int64_t at = first - 7 + lane;
    w.slot = -1;
    if (lane < 22 && at >= 0 && at < tokens) {
        const int64_t s = slots[at];
        w.slot = s >= 0 && s < capacity ? s : -1;
    }
    const int64_t next = __shfl_down(w.slot, 1);
    const uint32_t follows = (uint32_t)__ballot(lane < 21 && w.slot >= 0 && next == w.slot + 1);
    const uint32_t aligned = (uint32_t)__ballot(lane < 22 && w.slot >= 0 && (w.slot & 7) == 0);
    uint32_t starts = aligned;
#pragma unroll
    for (int i = 0; i < 7; ++i) starts &= follows >> i;           // followed by seven successive slots
    starts &= 0x7FFFu;                                            // lanes 0 .. 14: seven before the window to its last
    uint32_t covered = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) covered |= starts << i;
    w.whole = (covered >> 7) & 0xFFu;
    const uint32_t here = (starts >> 7) & 0xFFu;
    w.start = here ? (int)__builtin_ctz(here) : -1;
    return w;
}

__device__ __forceinline__ int64_t slot_of(const Window& w, int lane_of_token)
{
    const int lo = __shfl((int)(uint32_t)w.slot, lane_of_token), hi = __shfl((int)(w.slot >> 32), lane_of_token);
    return ((int64_t)hi << 32) | (uint32_t)lo;
}

// index of (slot, head) among the rows of D elements
__device__ __forceinline__ int64_t row_index(const CacheView& c, int64_t slot, int head)
{
    return ((slot >> c.page_shift) * c.heads + head) * c.page_size + (slot & (c.page_size - 1));
}

// four fp32 to codes, given the row's exponent
__device__ __forceinline__ uint32_t to_codes(const float x[4], int e)
{
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23); // 2^-e, e in [-126, 120]
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
    return (uint32_t)w;
}

__device__ __forceinline__ float finite_or_nan(float x) { return fabsf(x) < INFINITY ? x : __builtin_nanf(""); }

// 4 x 4 bytes: word i of the result holds byte i of each of the four words
__device__ __forceinline__ void transpose4(const uint32_t a[4], uint32_t t[4])
{
    const uint32_t lo01 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), hi01 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u);
    const uint32_t lo23 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u), hi23 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
    t[0] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u);
    t[1] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
    t[2] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u);
    t[3] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
}

// Codes of values whose block is not written whole go into memory one by one, eight bytes apart.  So that a row's lanes store next to
// each other, lane `part` takes columns part, part + D / 4, ... for its own four: 30,000 tokens x 4 heads of 128, each to a slot
// anywhere, 43 us, 62 before (23 as whole blocks).
template <int D>
__device__ __forceinline__ uint32_t deal(uint32_t w, int lane)
{
    constexpr int L = D / 4;
    const int part = lane & (L - 1), base = lane & ~(L - 1);
    uint32_t out = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) out |= (((uint32_t)__shfl((int)w, base + (part >> 2) + L / 4 * j) >> (8 * (part & 3))) & 0xFFu) << (8 * j);
    return out;
}
template <int D, bool kFp8, bool kBf16>
__global__ __launch_bounds__(64 * kCacheWaves)
void cache_append_kernel(CacheView c, TokenRows k, TokenRows v, const int64_t* slots, int64_t tokens, int64_t items)
{
    constexpr int kHeads = 128 / D;                               // heads of a wave
    constexpr int kIn = kBf16 ? 2 : 4;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6);
    if (item >= items) return;
    const int per = (c.heads + kHeads - 1) / kHeads;
    const int64_t first = item / per * kBlockTokens;
    const int half = lane >> 5, part = lane & (D / 4 - 1), col = part * 4;
    const int head = (int)(item % per) * kHeads + ((lane & 31) >> (D == 128 ? 5 : 4));
    const bool live = head < c.heads;
    const int safe_head = live ? head : 0;
    auto load = [&](const TokenRows& t, int64_t token, float x[4]) {
        const int64_t safe = token < tokens ? token : tokens - 1;
        load4<kBf16>(static_cast<const char*>(t.base) + (safe * t.token_stride + safe_head * t.head_stride + col) * kIn, x);
    };
    // rows of the window: keys, and values for those whose block is not filled.  Requested before the slots are known.
    float xk[4][4], xv[4][4], xb[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) load(k, first + 4 * half + i, xk[i]);
#pragma unroll
    for (int i = 0; i < 4; ++i) load(v, first + 4 * half + i, xv[i]);
    const Window w = look_at(slots, first, tokens, c.num_pages * c.page_size, lane);
    // codes of four rows, and their scale bytes into the cache
    auto quantise = [&](float x[4][4], const int64_t row[4], const bool ok[4], uint8_t* scales, uint32_t code[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[i][j] = finite_or_nan(x[i][j]);
                a = fmaxf(a, fabsf(x[i][j]));                     // NaN is passed over
            }
            const int e = exponent_for(row_max<D>(a));
            code[i] = to_codes(x[i], e);
            if (part == 0 && live && ok[i]) scales[row[i]] = (uint8_t)(e + 127);
        }
    };

    int64_t row[4], brow[4];
    bool ok[4], single[4], all[4] = {true, true, true, true};
    const bool some_single = ((~w.whole) & 0xFFu) != 0;
    if (w.start > 0) {                                            // a block that starts with the window is the window
#pragma unroll
        for (int i = 0; i < 4; ++i) load(v, first + w.start + 4 * half + i, xb[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) xb[i][j] = xv[i][j];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t slot = slot_of(w, 7 + 4 * half + i);
        ok[i] = slot >= 0;
        row[i] = ok[i] ? row_index(c, slot, safe_head) : 0;
        single[i] = ok[i] && !((w.whole >> (4 * half + i)) & 1u);
    }

    if (kFp8) {
        uint8_t* kc = static_cast<uint8_t*>(c.k);
        uint8_t* vc = static_cast<uint8_t*>(c.v);
        uint32_t code[4];
        quantise(xk, row, ok, c.k_scale, code);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (ok[i] && live) *reinterpret_cast<uint32_t*>(kc + row[i] * D + col) = code[i];
        if (some_single) {
            quantise(xv, row, single, c.v_scale, code);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t dealt = deal<D>(code[i], lane);
                if (!single[i] || !live) continue;
                uint8_t* p = vc + (row[i] & ~7ll) * D + part * 8 + (row[i] & 7);
#pragma unroll
                for (int j = 0; j < 4; ++j) p[j * (2 * D)] = (uint8_t)(dealt >> (8 * j));
            }
        }
        if (w.start >= 0) {
            const int64_t block = row_index(c, slot_of(w, 7 + w.start), safe_head);
#pragma unroll
            for (int i = 0; i < 4; ++i) brow[i] = block + 4 * half + i;
            quantise(xb, brow, all, c.v_scale, code);
            // word j: tokens 4 half .. 4 half + 3 of column col + j; the halves trade, so that each holds two whole
            // columns (the lower half the first two)
            uint32_t t[4];
            transpose4(code, t);
            const uint32_t give0 = half ? t[0] : t[2], give1 = half ? t[1] : t[3];
            const uint32_t got0 = __shfl_xor(give0, 32), got1 = __shfl_xor(give1, 32);
            const u32x4 out = half ? u32x4{got0, t[2], got1, t[3]} : u32x4{t[0], got0, t[1], got1};
            if (live) *reinterpret_cast<u32x4*>(vc + block * D + (col + 2 * half) * 8) = out;
        }
    } else {
        uint16_t* kc = static_cast<uint16_t*>(c.k);
        uint16_t* vc = static_cast<uint16_t*>(c.v);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (ok[i] && live)
                *reinterpret_cast<u32x2*>(kc + row[i] * D + col) = u32x2{pack_bf16(xk[i][0], xk[i][1]), pack_bf16(xk[i][2], xk[i][3])};
        if (some_single) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!single[i] || !live) continue;
                uint16_t* p = vc + (row[i] & ~7ll) * D + col * 8 + (row[i] & 7);
#pragma unroll
                for (int j = 0; j < 4; ++j) p[j * 8] = (uint16_t)pack_bf16(xv[i][j], 0.0f);
            }
        }
        if (w.start >= 0 && live) {
            const int64_t block = row_index(c, slot_of(w, 7 + w.start), safe_head);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<u32x2*>(vc + block * D + (col + j) * 8 + 4 * half) =
                    u32x2{pack_bf16(xb[0][j], xb[1][j]), pack_bf16(xb[2][j], xb[3][j])};
        }
    }
}

// Reading back: the same windows.  A token whose slot is not in the cache reads as zeros.
template <bool kBf16>
__device__ __forceinline__ void store4(char* p, const float x[4])
{
    if (kBf16) *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    else *reinterpret_cast<float4*>(p) = float4{x[0], x[1], x[2], x[3]};
}

__device__ __forceinline__ void from_codes(uint32_t w, uint8_t scale, float x[4])
{
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    const float s = __uint_as_float((uint32_t)scale << 23);
    x[0] = a.x * s; x[1] = a.y * s; x[2] = b.x * s; x[3] = b.y * s;
}

template <int D, bool kFp8, bool kBf16>
__global__ __launch_bounds__(64 * kCacheWaves)
void cache_read_kernel(CacheView c, const int64_t* slots, int64_t tokens, int64_t items, char* k_out, char* v_out)
{
    constexpr int kHeads = 128 / D;
    constexpr int kOut = kBf16 ? 2 : 4;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6);
    if (item >= items) return;
    const int per = (c.heads + kHeads - 1) / kHeads;
    const int64_t first = item / per * kBlockTokens;
    const int half = lane >> 5, part = lane & (D / 4 - 1), col = part * 4;
    const int head = (int)(item % per) * kHeads + ((lane & 31) >> (D == 128 ? 5 : 4));
    const bool live = head < c.heads;
    const int safe_head = live ? head : 0;
    const Window w = look_at(slots, first, tokens, c.num_pages * c.page_size, lane);

    float x[4];
    auto put = [&](char* out, int64_t token, const float v[4]) {
        if (live && token < tokens) store4<kBf16>(out + ((token * c.heads + safe_head) * D + col) * kOut, v);
    };
    const uint8_t* kc = static_cast<const uint8_t*>(c.k);
    const uint8_t* vc = static_cast<const uint8_t*>(c.v);
    constexpr int kElem = kFp8 ? 1 : 2;
    int64_t row[4];
    bool ok[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t slot = slot_of(w, 7 + 4 * half + i);
        ok[i] = slot >= 0;
        row[i] = ok[i] ? row_index(c, slot, safe_head) : 0;
    }
    // requests first, then what is made of them
    uint32_t kw[4][2] = {}, vw[4][4] = {};
    uint8_t ks[4] = {}, vs[4] = {};
    const bool some_single = ((~w.whole) & 0xFFu) != 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(kc + (row[i] * D + col) * kElem);
        kw[i][0] = p[0];
        if (kFp8) ks[i] = c.k_scale[row[i]];
        else kw[i][1] = p[1];
    }
    if (some_single) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint8_t* p = vc + ((row[i] & ~7ll) * D + col * 8 + (row[i] & 7)) * kElem;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                vw[i][j] = kFp8 ? (uint32_t)p[j * 8] : (uint32_t)*reinterpret_cast<const uint16_t*>(p + j * 16);
            if (kFp8) vs[i] = c.v_scale[row[i]];
        }
    }
    u32x4 blk{};
    u32x2 blk16[4]{};
    uint8_t bs[4] = {};
    if (w.start >= 0) {
        const int64_t block = row_index(c, slot_of(w, 7 + w.start), safe_head);
        if (kFp8) {
            blk = *reinterpret_cast<const u32x4*>(vc + block * D + (col + 2 * half) * 8);
#pragma unroll
            for (int i = 0; i < 4; ++i) bs[i] = c.v_scale[block + 4 * half + i];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                blk16[j] = *reinterpret_cast<const u32x2*>(vc + (block * D + (col + j) * 8 + 4 * half) * 2);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (kFp8) {
            from_codes(kw[i][0], ks[i], x);
        } else {
            x[0] = __uint_as_float(kw[i][0] << 16); x[1] = __uint_as_float(kw[i][0] & 0xFFFF0000u);
            x[2] = __uint_as_float(kw[i][1] << 16); x[3] = __uint_as_float(kw[i][1] & 0xFFFF0000u);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = ok[i] ? x[j] : 0.0f;
        put(k_out, first + 4 * half + i, x);
    }
    if (some_single) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (kFp8) {
                from_codes(vw[i][0] | vw[i][1] << 8 | vw[i][2] << 16 | vw[i][3] << 24, vs[i], x);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(vw[i][j] << 16);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = ok[i] ? x[j] : 0.0f;
            if (!((w.whole >> (4 * half + i)) & 1u)) put(v_out, first + 4 * half + i, x);
        }
    }
    if (w.start >= 0) {
        if (kFp8) {
            // the reverse of the exchange above: two whole columns -> four columns of the half's four tokens
            const uint32_t give0 = half ? blk.x : blk.y, give1 = half ? blk.z : blk.w;
            const uint32_t got0 = __shfl_xor(give0, 32), got1 = __shfl_xor(give1, 32);
            const uint32_t t[4] = {half ? got0 : blk.x, half ? got1 : blk.z, half ? blk.y : got0, half ? blk.w : got1};
            uint32_t code[4];
            transpose4(t, code);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                from_codes(code[i], bs[i], x);
                put(v_out, first + w.start + 4 * half + i, x);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t pair = i < 2 ? blk16[j].x : blk16[j].y;
                    x[j] = __uint_as_float((i & 1) ? pair & 0xFFFF0000u : pair << 16);
                }
                put(v_out, first + w.start + 4 * half + i, x);
            }
        }
    }
}

template <typename F>
static hipError_t by_shape(const CacheView& c, bool io_bf16, F f)
{
    auto with = [&](auto d, auto fp8) {
        if (io_bf16) f(d, fp8, std::true_type{});
        else f(d, fp8, std::false_type{});
    };
    auto of_dim = [&](auto d) {
        if (c.fp8) with(d, std::true_type{});
        else with(d, std::false_type{});
    };
    if (c.dim == 128) of_dim(std::integral_constant<int, 128>{});
    else of_dim(std::integral_constant<int, 64>{});
    return hipGetLastError();
}

static int64_t cache_items(const CacheView& c, int64_t tokens)
{
    const int per = (c.heads + 128 / c.dim - 1) / (128 / c.dim);
    return (tokens + kBlockTokens - 1) / kBlockTokens * per;
}

// Waves of a workgroup: one while there are at most sixteen of them per compute unit, which spreads a decode step's few waves over
// all units (512 tokens x 4 heads of 128 written and read back: 9.2 us with one, 10.1 with two, 12.1 with four), two beyond (60,001
// tokens: 81.8, 80.0, 80.6).
static int cache_waves(int64_t items) { return items <= (int64_t)compute_units() * 16 ? 1 : kCacheWaves; }

hipError_t launch_cache_append(const CacheView& c, const TokenRows& k, const TokenRows& v, bool in_bf16,
                               const int64_t* slots, int64_t tokens, hipStream_t stream)
{
    const int64_t items = cache_items(c, tokens);
    const int waves = cache_waves(items);
    const dim3 grid((uint32_t)((items + waves - 1) / waves));
    return by_shape(c, in_bf16, [&](auto d, auto fp8, auto bf16) {
        cache_append_kernel<decltype(d)::value, decltype(fp8)::value, decltype(bf16)::value>
            <<<grid, 64 * waves, 0, stream>>>(c, k, v, slots, tokens, items);
    });
}

hipError_t launch_cache_read(const CacheView& c, const int64_t* slots, int64_t tokens, void* k_out, void* v_out,
                             bool out_bf16, hipStream_t stream)
{
    const int64_t items = cache_items(c, tokens);
    const int waves = cache_waves(items);
    const dim3 grid((uint32_t)((items + waves - 1) / waves));
    return by_shape(c, out_bf16, [&](auto d, auto fp8, auto bf16) {
        cache_read_kernel<decltype(d)::value, decltype(fp8)::value, decltype(bf16)::value>
            <<<grid, 64 * waves, 0, stream>>>(c, slots, tokens, items, static_cast<char*>(k_out), static_cast<char*>(v_out));
    });
}

}  // namespace e3
