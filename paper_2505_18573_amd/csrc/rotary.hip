// Turning rows of heads by their tokens' positions (formulas: rotary.h).
//
// A workgroup takes a few tokens with all their heads: sine and cosine of every (token, pair) are made once, by one thread each,
// and lie in LDS; then a thread keeps those of eight pairs of its token and takes units of two 16-byte vectors (bf16) from head after
// head.  Each element is read and written once, in place where the caller likes, since a unit's two
// vectors are read before either is written.
//
// Bound by memory: 16,384 tokens x 28 heads of 128 in bf16 take 44.1 us, 5.3 TB/s read and written (a copy of 2 GiB: 4.85); 5003
// tokens x 16 heads of 80 in fp32 with three axes 12.4 us, 4.1 TB/s, the start and the first chain of loads among them.  Asking for the next
// head's unit before this one is stored was slower: other waves of a compute unit cover the wait, and it costs registers.
#include "rotary.h"
#include "vocab_pass.h"

namespace e3 {

constexpr int kTurnThreads = 256;
constexpr int kTurnMostTokens = 16;             // of a workgroup
constexpr int kTurnUnits = kTurnThreads / 2;    // it has at least so many units, where there are many tokens

template <bool kBf16>
__global__ __launch_bounds__(kTurnThreads)
void rotate_kernel(TurnArgs a, Rotary r, int tokens_each, int heads_each)
{
    extern __shared__ float2 turns[];                             // [tokens_each][rot / 2]
    const int64_t first = (int64_t)blockIdx.x * tokens_each;
    const int here = a.tokens - first < tokens_each ? (int)(a.tokens - first) : tokens_each;
    const int pairs = r.rot / 2, units = units_of(r.rot, a.dim);
    const int u = threadIdx.x % units, t = threadIdx.x / units % tokens_each;
    int h = threadIdx.x / (units * tokens_each);
    const bool is = h < heads_each && t < here;
    const int64_t token = first + (is ? t : 0);
    Unit<kBf16> now;
    if (is) now.load(a, r, token, h < a.heads ? h : 0, u);
    for (int i = threadIdx.x; i < here * pairs; i += kTurnThreads) turns[i] = turn_of(place_of(r, first + i / pairs, i % pairs), r.sign);
    __syncthreads();
    if (h >= a.heads || !is) return;
    float2 by[8];
    if (u < r.rot / 16) {
#pragma unroll
        for (int j = 0; j < 8; ++j) by[j] = turns[t * pairs + 8 * u + j];
    }
    now.store(a, r, token, h, u, by);
    for (h += heads_each; h < a.heads; h += heads_each) {
        now.load(a, r, token, h, u);
        now.store(a, r, token, h, u, by);
    }
}

hipError_t launch_rotate(const TurnArgs& a, const Rotary& r, bool bf16, hipStream_t stream)
{
    const int units = units_of(r.rot, a.dim);
    // One token a workgroup while nearly all of those are on the card at once (28 heads of 128, bf16: 512 tokens 3.7 us, with two a workgroup
    // 4.3, with four 5.2; 1024 tokens 5.0, 5.4, 5.8).  Beyond that as many as give half of the threads a unit; more tokens make
    // fewer, longer workgroups (16,384 tokens of 28 heads: one 44.1 us, two 45.3, four 46.4; 30,000 of 16 heads of 80 in fp32: two
    // 58.6, four 68.5; though 5003 of these: two 12.4, four 11.6).
    const int64_t of_token = (int64_t)units * a.heads;
    int each = a.tokens <= 4 * (int64_t)compute_units() ? 1 : (int)((kTurnUnits + of_token - 1) / of_token);
    if (each > kTurnMostTokens) each = kTurnMostTokens;
    const int least = (int)((a.tokens + (1 << 23) - 1) >> 23);                // threads of a launch below 2^32; 4 at most
    if (each < least) each = least;
    if (each > kTurnThreads / units) each = kTurnThreads / units;
    const int heads_each = kTurnThreads / (each * units);
    const dim3 grid((uint32_t)((a.tokens + each - 1) / each));
    const size_t lds = (size_t)each * (r.rot / 2) * sizeof(float2);
    if (bf16) rotate_kernel<true><<<grid, kTurnThreads, lds, stream>>>(a, r, each, heads_each);
    else rotate_kernel<false><<<grid, kTurnThreads, lds, stream>>>(a, r, each, heads_each);
    return hipGetLastError();
}

}  // namespace e3
