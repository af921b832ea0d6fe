// Beam search: the best continuations over beams and vocabulary, and the beams' pages after them.
//
//   score(b, v) = s_b + z_bv / tau - ln sum_i exp(z_bi / tau),   the `keep` largest of a sequence, ties to the lowest (b, v).
//
// Two launches.
//   stream   Every wave takes a segment of a row, eight 16-byte loads a lane, and leaves sum exp2 (fp32 in a lane, fp64 over the
//            lanes) relative to its largest logit, and the largest logit of every chunk of 512 columns.  The logits are read once; that is what bounds the call.
//   select   A workgroup per sequence.  No element outside the `keep` best chunks can be among the `keep` best: each of those
//            chunks holds one that comes before it (chunks are runs of columns, so this is also right for equal values, where the
//            lower index comes first).  So the chunks' maxima are ranked first and only `keep` chunks are read again, 1 KB each.
// Scores are compared in fp64, as differences of logits: base_b + (z - largest z) / tau.  Sums taken in fp32 leave ln sum exp off by 1e-7
// as a rule (4e-7 the most of 27,648 beams: tau 0.02 to 3, logits around 0 to +-4000, 1000 to 151,936 columns), the same for all tokens
// of a beam, so only the order between beams is in question: where two neighbours of different beams among the results, or one that is
// kept and one that is left out, are within 2e-6 of each other, the beams' sums are taken again in fp64, by the sequence's
// workgroup, and the selection is made once more.  (One sequence in some hundreds; V = 151,936 takes 19 us for a beam.)
//
// Measured: 64 sequences x 8 beams, V = 151,936, bf16, keep 16: 36.5 us; the stream 27.3 (5.7 TB/s), the selection 9.7, a chain of phases with
// barriers between (the beams' sums 1.8, the bound 2, chunks in order 1, their elements 1.8, these in order and out 1.2).  One sequence x 4, V
// = 32,000, fp32: 10.6 us, two launches of latency.  A selection by the stream's last workgroup would need counters that start at zero.
#include "beam.h"
#include "vocab_common.h"
#include "vocab_pass.h"

namespace e3 {

constexpr int kChunkCols = 512;
constexpr int kVecs = 8;                        // 16-byte vectors of a lane in a segment
constexpr int kStreamWaves = 4;
constexpr int kSelectWaves = 16, kSelectThreads = 64 * kSelectWaves;
constexpr float kNoLogit = -1e30f;              // at or below: no probability
constexpr double kNear = 2e-6;
constexpr double kNone = -INFINITY;

template <bool kBf16> struct Segment { static constexpr int kCols = kVecs * 64 * (kBf16 ? 8 : 4), kChunks = kCols / kChunkCols; };

struct Partial { double ref, sum; };            // the largest logit, and the sum of 2^((z - ref) c), c = log2(e) / tau

struct BeamShape {
    int64_t chunks, segments;                   // of a row (segments: of the narrower type)
    uint32_t per_chunk;                         // ceil(2^32 / chunks): x * per_chunk >> 32 = x / chunks for x * chunks < 2^32 (chunks > 1)
    int64_t at_partials, bytes;
};
static BeamShape beam_shape(int64_t rows, int64_t V, bool bf16)
{
    BeamShape s;
    const int64_t cols = bf16 ? Segment<true>::kCols : Segment<false>::kCols;
    s.chunks = (V + kChunkCols - 1) / kChunkCols;
    s.segments = (V + cols - 1) / cols;
    s.per_chunk = s.chunks > 1 ? (uint32_t)((((uint64_t)1 << 32) + s.chunks - 1) / s.chunks) : 0;
    s.at_partials = (rows * s.chunks * 4 + 255) / 256 * 256;
    s.bytes = s.at_partials + rows * s.segments * (int64_t)sizeof(Partial);
    return s;
}

size_t beam_workspace_bytes(int64_t seqs, int32_t beams, int64_t V)
{
    const BeamShape s = beam_shape(seqs * beams, V, false);
    // a wave per segment, a workgroup of 1024 threads per sequence: threads of the launches below 2^32
    return seqs < 1 << 22 && seqs * beams * s.segments < (int64_t)1 << 25 ? (size_t)s.bytes : 0;
}

__device__ __forceinline__ const char* row_of(const BeamArgs& a, int64_t row, int size)
{
    return static_cast<const char*>(a.logits) + (row / a.beams * a.seq_stride + row % a.beams * a.beam_stride) * size;
}
__device__ __forceinline__ bool takes_part(float score) { return fabsf(score) < INFINITY; }

// ---------------------------------------------------------------- stream
// kFlat: log2(e) / tau is so small (kFlatBelow) that a logit of kNoLogit would count, which has no probability whatever tau makes of it.
// A kernel of its own: with the comparison as a branch of this one the compiler holds the logits unpacked for both, 64 x 8 beams
// 41.6 to 48.7 us for 36.6.
constexpr float kFlatBelow = 1e-20f;
template <bool kBf16, bool kFlat>
__global__ __launch_bounds__(64 * kStreamWaves)
void beam_stream_kernel(BeamArgs a, BeamShape s, float c, char* ws)
{
    constexpr int kPer = kBf16 ? 8 : 4, kCols = Segment<kBf16>::kCols, kChunks = Segment<kBf16>::kChunks, kOf = kVecs / kChunks;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * kStreamWaves + (threadIdx.x >> 6);
    if (item >= a.seqs * a.beams * s.segments) return;
    const int64_t row = item / s.segments, segment = item % s.segments;
    if (!takes_part(a.scores[row]) || (a.finished && a.finished[row])) return;
    const char* p = row_of(a, row, kBf16 ? 2 : 4);
    const int64_t first = segment * kCols + lane * kPer;
    const bool tail = (segment + 1) * kCols > a.V;                            // uniform
    u32x4 w[kVecs];
    if (!tail) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) w[i] = stream_load(reinterpret_cast<const u32x4*>(p + (first + (int64_t)i * 64 * kPer) * (kBf16 ? 2 : 4)));
    } else {                                                                   // nothing behind the row is read
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int64_t col = first + (int64_t)i * 64 * kPer;
            constexpr uint32_t kLow = kBf16 ? 0xFF80FF80u : 0xFF800000u;       // -inf
            w[i] = u32x4{kLow, kLow, kLow, kLow};
            if (col + kPer <= a.V) {
                w[i] = stream_load(reinterpret_cast<const u32x4*>(p + col * (kBf16 ? 2 : 4)));
            } else {
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if (col + j < a.V) {
                        if (kBf16) {
                            const uint32_t x = reinterpret_cast<const uint16_t*>(p)[col + j];
                            w[i][j >> 1] = (j & 1) ? (w[i][j >> 1] & 0xFFFFu) | x << 16 : (w[i][j >> 1] & 0xFFFF0000u) | x;
                        } else {
                            w[i][j & 3] = reinterpret_cast<const uint32_t*>(p)[col + j];
                        }
                    }
            }
        }
    }
    auto logit = [&](int i, int j) {
        return kBf16 ? __uint_as_float((j & 1) ? w[i][j >> 1] & 0xFFFF0000u : w[i][j >> 1] << 16) : __uint_as_float(w[i][j & 3]);
    };
    float top[kChunks];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        float m = fmaxf(logit(i, 0), logit(i, 1));
#pragma unroll
        for (int j = 2; j < kPer; j += 2) m = fmax3(m, logit(i, j), logit(i, j + 1));
        top[i / kOf] = i % kOf == 0 ? m : fmaxf(top[i / kOf], m);
    }
    float most = top[0];
#pragma unroll
    for (int i = 1; i < kChunks; ++i) most = fmaxf(most, top[i]);
    const float ref = fmaxf(most, kNoLogit);
    auto add_up = [&](auto term) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            float part[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) part[j] = __builtin_amdgcn_exp2f(term(logit(i, j)));
#pragma unroll
            for (int d = 1; d < kPer; d <<= 1)
#pragma unroll
                for (int j = 0; j < kPer; j += 2 * d) part[j] += part[j + d];
            sum += part[0];
        }
        return sum;
    };
    // One multiply-add a term: the lane's reference is rounded once, in the scaled domain, and by how much (fused: exactly) is made up
    // for in the lane's factor, so that everything is relative to a logit: c is off by 2^-25 of itself, and only differences of logits may see
    // that.  Not where the reference is large (masks of -1e9 throughout): its rounding there is more than the exponent holds.
    const float most_ref = wave_max(ref), below = ref - most_ref;
    float sum, off = 0.0f;
    if (kFlat) {
        sum = add_up([&](float z) { return z <= kNoLogit ? -INFINITY : (z - ref) * c; });         // (NaN stays)
    } else if (!__any(fabsf(ref) > 4096.0f) && c < 1024.0f) {
        const float scaled = ref * c;
        off = fmaf(ref, c, -scaled);
        sum = add_up([&](float z) { return fmaf(z, c, -scaled); });
    } else {
        sum = add_up([&](float z) { return (z - ref) * c; });
    }
    const double all = wave_sum((double)sum * (double)__builtin_amdgcn_exp2f(fmaf(below, c, -off)));
    // The chunks' maxima over the wave: halves trade two chunks each and keep one, rows of sixteen lanes again; what is left is a row's.
    float* tops = reinterpret_cast<float*>(ws) + row * s.chunks + segment * kChunks;
    float in_half[kChunks / 2], in_row[kChunks / 4];
#pragma unroll
    for (int i = 0; i < kChunks / 2; ++i) {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top[i]), __float_as_uint(top[i + kChunks / 2]), false, false);
        in_half[i] = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));      // lower half: chunk i, upper: i + kChunks / 2
    }
#pragma unroll
    for (int i = 0; i < kChunks / 4; ++i) {
        const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(in_half[i]), __float_as_uint(in_half[i + kChunks / 4]), false, false);
        float m = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));         // row r: chunk i + (r & 1) kChunks / 4 + (r >> 1) kChunks / 2
        m = fmaxf(m, dpp_f<kDppXor1>(m, m));
        m = fmaxf(m, dpp_f<kDppXor2>(m, m));
        m = fmaxf(m, dpp_f<kDppHalfMirror>(m, m));
        in_row[i] = fmaxf(m, dpp_f<kDppMirror>(m, m));
    }
#pragma unroll
    for (int i = 0; i < kChunks / 4; ++i) {
        const int chunk = i + ((lane >> 4) & 1) * (kChunks / 4) + (lane >> 5) * (kChunks / 2);
        if ((lane & 15) == i && segment * kChunks + chunk < s.chunks) tops[chunk] = in_row[i];
    }
    if (lane == 0) reinterpret_cast<Partial*>(ws + s.at_partials)[row * s.segments + segment] = Partial{(double)most_ref, all};
}

// ---------------------------------------------------------------- select
// A candidate or a chunk's best one: larger keys come first, of equal ones the lower index.
struct Entry { double key; int index; };

// The lane that holds the wave's first entry, -1 if there is none (all keys -inf).  Rounding to fp32 keeps the order, so only lanes
// that are equal there are looked at one by one.
__device__ __forceinline__ int first_of(const Entry& e)
{
    const float f = (float)e.key;
    const float top = wave_max(f);
    if (!(top > -INFINITY)) return -1;
    unsigned long long tied = __ballot(f == top);
    int best = (int)__builtin_ctzll(tied);
    tied &= tied - 1;
    if (tied != 0) {
        double key = read_lane(e.key, best);
        int index = __builtin_amdgcn_readlane(e.index, best);
        for (; tied != 0; tied &= tied - 1) {
            const int l = (int)__builtin_ctzll(tied);
            const double k = read_lane(e.key, l);
            const int i = __builtin_amdgcn_readlane(e.index, l);
            if (k > key || (k == key && i < index)) { best = l; key = k; index = i; }
        }
    }
    return best;
}

// 2^x for -1000 < x < 1000 in fp64: the fraction's exponential series, whose next term is below 1e-14.
__device__ __forceinline__ double exp2_of(double x)
{
    const double n = rint(x), t = (x - n) * kLn2;
    double p = 1.0 / 39916800.0;
    p = fma(p, t, 1.0 / 3628800.0);
    p = fma(p, t, 1.0 / 362880.0);
    p = fma(p, t, 1.0 / 40320.0);
    p = fma(p, t, 1.0 / 5040.0);
    p = fma(p, t, 1.0 / 720.0);
    p = fma(p, t, 1.0 / 120.0);
    p = fma(p, t, 1.0 / 24.0);
    p = fma(p, t, 1.0 / 6.0);
    p = fma(p, t, 0.5);
    p = fma(p, t, 1.0);
    p = fma(p, t, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)n);
}

template <bool kBf16>
__device__ __forceinline__ float logit_at(const char* row, int64_t col)
{
    return kBf16 ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[col] << 16) : reinterpret_cast<const float*>(row)[col];
}

// Whether a comes before b.
__device__ __forceinline__ bool before(const Entry& a, const Entry& b) { return a.key > b.key || (a.key == b.key && a.index < b.index); }

constexpr int kGroups = kSelectThreads / 8;     // of eight lanes, whose maxima bound what is kept
constexpr int kRoom = 256;                      // chunks above the bound
constexpr int kElements = kMaxKeep * (kMaxKeep + 1) / 2;          // of the r-th best chunk at most keep - r elements
struct SelectLds {
    // score(b, v) = base + (z - top) / tau: relative to the beam's largest logit, or logits far from zero would cost the score its last digits
    double base[kMaxBeams];                     // s_b - ln sum exp((z - top) / tau), a finished beam's s_b, -inf: the beam offers nothing
    double top[kMaxBeams];
    double log2_sum[kMaxBeams];
    double sums[kSelectWaves];
    int ends[kMaxBeams];                        // a finished beam
    alignas(16) float group[kGroups];
    float bound;
    int found, elements, chunks_found;
    uint32_t near;                              // beams whose sums decide
    Entry chunk[kMaxKeep + 2];                  // the best ones, in order
    Entry some[kRoom + kMaxKeep + 2];           // chunks above the bound
    Entry element[kElements];
    Entry best[kMaxKeep + 2];
    Entry of_wave[kSelectWaves + 1][kMaxKeep + 2];
};

__device__ __forceinline__ int sum_of_eight(int x)              // over eight lanes
{
    x += dpp_i<kDppXor1>(x, x);
    x += dpp_i<kDppXor2>(x, x);
    return x + dpp_i<kDppHalfMirror>(x, x);
}

// to[r] = the r-th of n entries in order, r < most, by counting how many come before each: eight lanes an entry.
__device__ __forceinline__ void in_order(const Entry* from, int n, Entry* to, int most)
{
    const int part = threadIdx.x & 7;
    for (int i0 = 0; i0 < n; i0 += kSelectThreads / 8) {
        const int i = i0 + (int)(threadIdx.x >> 3);
        const Entry mine = from[i < n ? i : 0];
        int rank = 0;
#pragma unroll 4
        for (int j = part; j < n; j += 8) rank += before(from[j], mine) ? 1 : 0;
        rank = sum_of_eight(rank);
        if (part == 0 && i < n && rank < most) to[rank] = mine;
    }
}

template <bool kBf16>
__global__ __launch_bounds__(kSelectThreads)
void beam_select_kernel(BeamArgs a, BeamShape s, double per_logit, const char* ws)
{
    __shared__ SelectLds lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t seq = blockIdx.x, row0 = seq * a.beams;
    const float* tops = reinterpret_cast<const float*>(ws) + row0 * s.chunks;
    const double c = kLog2e * per_logit;                                       // per_logit = 1 / tau
    const int keep = a.keep, need = keep + 1, most = (int)s.chunks;
    // Chunks a thread holds.  A pass over 1024 times as many costs 2.5 us, instructions that are not used cost their fetch: 16 beams of 297
    // chunks 18.2 us with five, 20.6 with four, 18.3 with eight; 4 beams of 63 11.7, 11.6, 12.3.
    constexpr int kEach = 5;
    const int entries = a.beams * most;
    float z[kEach];                                                            // asked for before the sums are
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int e = i * kSelectThreads + (int)threadIdx.x;
        z[i] = e < entries ? tops[e] : 0.0f;
    }

    for (int b = wave; b < a.beams; b += kSelectWaves) {
        // (what a beam that takes no part has left is asked for as well, and not used)
        const Partial* parts = reinterpret_cast<const Partial*>(ws + s.at_partials) + (row0 + b) * s.segments;
        const Partial mine = parts[lane < s.segments ? lane : 0];
        const float score = a.scores[row0 + b];
        const bool ends = a.finished && a.finished[row0 + b];
        double base = kNone, total = 0.0, up = 0.0;
        if (takes_part(score)) {
            if (ends) {
                base = score;
            } else {
                up = lane < s.segments ? mine.ref : -INFINITY;
                for (int64_t i = lane + 64; i < s.segments; i += 64) up = fmax(up, parts[i].ref);
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) up = fmax(up, __shfl_xor(up, d));
                double sum = lane < s.segments ? mine.sum * exp2_of(fmax((mine.ref - up) * c, -1000.0)) : 0.0;
                for (int64_t i = lane + 64; i < s.segments; i += 64) sum += parts[i].sum * exp2_of(fmax((parts[i].ref - up) * c, -1000.0));
                sum = wave_sum(sum);
                total = log2(sum);
                // NaN and +inf make the sum no number; a row without any probability has none
                if (sum > 0.0 && sum < INFINITY && fabs(up) < INFINITY) base = score - total * kLn2;
            }
        }
        if (lane == 0) { lds.base[b] = base; lds.top[b] = up; lds.log2_sum[b] = total; lds.ends[b] = ends; }
    }
    if (threadIdx.x == 0) lds.near = 0;
    __syncthreads();

    for (int round = 0; round < 2; ++round) {
        // ---- the best keep + 1 chunks: thread t's are entries t, t + 1024, ... of eight times as many at a time
        int known = 0;                                                         // in lds.chunk
        for (int from = 0; from < entries; from += kEach * kSelectThreads) {
            double key[kEach];
            Entry mine{kNone, 0};
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                key[i] = kNone;
                if (from + i * kSelectThreads >= entries) continue;            // uniform
                const int e = from + i * kSelectThreads + (int)threadIdx.x;
                if (e < entries) {
                    if (from > 0 || round > 0) z[i] = tops[e];
                    const int b = most > 1 ? (int)__umulhi((uint32_t)e, s.per_chunk) : e;     // e / most
                    const double base = lds.base[b], top = lds.top[b];
                    const bool ends = lds.ends[b] != 0;
                    if (base > kNone && (ends ? e - b * most == a.eos / kChunkCols : z[i] > kNoLogit)) key[i] = ends ? base : base + ((double)z[i] - top) * per_logit;
                }
                if (key[i] > mine.key) mine = Entry{key[i], e};
            }
            // A bound that at least `need` of them reach if so many are there: the need-th of the maxima of eight lanes.  (Rounding to fp32
            // keeps the order.)
            float g = (float)mine.key;
            g = fmaxf(g, dpp_f<kDppXor1>(g, g));
            g = fmaxf(g, dpp_f<kDppXor2>(g, g));
            g = fmaxf(g, dpp_f<kDppHalfMirror>(g, g));
            if ((lane & 7) == 0) lds.group[threadIdx.x >> 3] = g;
            if (threadIdx.x == 0) { lds.bound = -INFINITY; lds.found = known; }
            if (wave == 0)
                for (int i = lane; i < known; i += 64) lds.some[i] = lds.chunk[i];
            __syncthreads();
            {                                                                  // eight lanes a group
                const int part = threadIdx.x & 7;
                const float x = lds.group[threadIdx.x >> 3];
                int above = 0, equal = 0;
#pragma unroll
                for (int j = 4 * part; j < kGroups; j += 32) {
                    const float4 y = *reinterpret_cast<const float4*>(&lds.group[j]);
                    above += (y.x > x) + (y.y > x) + (y.z > x) + (y.w > x);
                    equal += (y.x == x) + (y.y == x) + (y.z == x) + (y.w == x);
                }
                above = sum_of_eight(above);
                equal = sum_of_eight(equal);
                if (part == 0 && above < need && above + equal >= need) lds.bound = x;          // equal ones store the same
            }
            __syncthreads();
            const float bound = lds.bound;
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (key[i] > kNone && (float)key[i] >= bound) {
                    const int at = atomicAdd(&lds.found, 1);
                    if (at < kRoom + known) lds.some[at] = Entry{key[i], from + i * kSelectThreads + (int)threadIdx.x};
                }
            __syncthreads();
            const int found = lds.found;
            if (found <= kRoom + known) {                                      // in any order there, in order afterwards
                in_order(lds.some, found, lds.chunk, need);
                known = found < need ? found : need;
                __syncthreads();
                continue;
            }
            // Hundreds of equal ones: one after the other, a list for each wave, then the lists.
            int n = 0;
            for (; n <= keep; ++n) {
                const int l = first_of(mine);
                if (l < 0) break;
                if (lane == l) {
                    lds.of_wave[wave][n] = mine;
                    const int taken = mine.index;
                    mine = Entry{kNone, 0};
#pragma unroll
                    for (int i = 0; i < kEach; ++i) {
                        const int e = from + i * kSelectThreads + (int)threadIdx.x;
                        if (e == taken) key[i] = kNone;
                        if (key[i] > mine.key) mine = Entry{key[i], e};
                    }
                }
            }
            if (lane == 0) lds.of_wave[wave][n] = Entry{kNone, 0};
            if (wave == 0)
                for (int i = lane; i <= known; i += 64) lds.of_wave[kSelectWaves][i] = i < known ? lds.chunk[i] : Entry{kNone, 0};
            __syncthreads();
            if (wave == 0) {
                int at = 0, out = 0;
                Entry head = lane <= kSelectWaves ? lds.of_wave[lane][0] : Entry{kNone, 0};
                for (; out <= keep; ++out) {
                    const int l = first_of(head);
                    if (l < 0) break;
                    if (lane == l) {
                        lds.chunk[out] = head;
                        head = lds.of_wave[lane][++at];
                    }
                }
                if (lane == 0) lds.chunks_found = out;
            }
            __syncthreads();
            known = lds.chunks_found;
        }
        // ---- their elements
        const int chunks = known < keep ? known : keep;
        // `keep` candidates reach the last of these chunks' best; those a little below it tell where beams are near each other
        const double border = chunks == keep ? lds.chunk[keep - 1].key - kNear : kNone;
        if (threadIdx.x == 0) lds.elements = 0;
        __syncthreads();
        for (int r = wave; r < chunks; r += kSelectWaves) {
            const Entry of = lds.chunk[r];
            const int b = of.index / most, chunk = of.index % most, room = keep - r;
            if (lds.ends[b]) {
                if (lane == 0) lds.element[atomicAdd(&lds.elements, 1)] = Entry{of.key, b * (int)a.V + a.eos};
                continue;
            }
            const char* row = row_of(a, row0 + b, kBf16 ? 2 : 4);
            const int64_t first = (int64_t)chunk * kChunkCols + lane * 8;
            const double base = lds.base[b], top_logit = lds.top[b];
            const auto key_of = [&](float z) { return base + ((double)z - top_logit) * per_logit; };
            float x[8];
            if (first + 8 <= a.V) {
                const u32x4* p = reinterpret_cast<const u32x4*>(row + first * (kBf16 ? 2 : 4));
                const u32x4 w0 = p[0], w1 = kBf16 ? w0 : p[1];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[j] = kBf16 ? __uint_as_float((j & 1) ? w0[j >> 1] & 0xFFFF0000u : w0[j >> 1] << 16) : __uint_as_float(j < 4 ? w0[j & 3] : w1[j & 3]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = first + j < a.V ? logit_at<kBf16>(row, first + j) : -INFINITY;
            }
            int n = 0;
            unsigned long long reach[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                reach[j] = __ballot(x[j] > kNoLogit && key_of(x[j]) >= border);
                n += (int)__popcll(reach[j]);
            }
            if (n <= room) {
                int at = 0;
                if (lane == 0) at = atomicAdd(&lds.elements, n);
                at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if ((reach[j] >> lane) & 1ull)
                        lds.element[at + (int)__popcll(reach[j] & ((1ull << lane) - 1ull))] = Entry{key_of(x[j]), b * (int)a.V + (int)first + j};
                    at += (int)__popcll(reach[j]);
                }
                continue;
            }
            // more than can be kept (equal values): the first ones, one after the other
            int at = 0;
            if (lane == 0) at = atomicAdd(&lds.elements, room);
            at = __builtin_amdgcn_readfirstlane(at);
            for (n = 0; n < room; ++n) {
                float best = x[0];
                int j0 = 0;
#pragma unroll
                for (int j = 1; j < 8; ++j)
                    if (x[j] > best) { best = x[j]; j0 = j; }
                const float top = wave_max(best);
                const int l = (int)__builtin_ctzll(__ballot(best == top));
                if (lane == l) {
                    lds.element[at + n] = Entry{key_of(top), b * (int)a.V + (int)first + j0};
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j == j0) x[j] = -INFINITY;
                }
            }
        }
        __syncthreads();
        // ---- in order
        const int n = lds.elements, kept = n < keep ? n : keep;
        in_order(lds.element, n, lds.best, keep);
        __syncthreads();
        if (round == 0) {
            const auto beam_of = [&](int i) { return lds.best[i].index / (int)a.V; };
            if ((int)threadIdx.x + 1 < kept) {
                const int x = beam_of(threadIdx.x), y = beam_of(threadIdx.x + 1);
                if (x != y && lds.best[threadIdx.x].key - lds.best[threadIdx.x + 1].key < kNear) atomicOr(&lds.near, 1u << x | 1u << y);
            }
            // a candidate that is left out, or the best of a chunk that is, against the last ones that are kept
            const Entry last = lds.best[keep - 1];                             // (of `keep` chunks there are `keep` candidates)
            const auto left_out = [&](double key, int beam) {
                for (int i = keep - 1; i >= 0 && lds.best[i].key - key < kNear; --i)
                    if (beam_of(i) != beam) atomicOr(&lds.near, 1u << beam_of(i) | 1u << beam);
            };
            if (kept == keep) {
                for (int i = (int)threadIdx.x; i < n; i += kSelectThreads) {
                    const Entry e = lds.element[i];
                    if (last.key - e.key < kNear && before(last, e)) left_out(e.key, e.index / (int)a.V);
                }
                if (known > keep && last.key - lds.chunk[keep].key < kNear) {
                    const Entry border_chunk = lds.chunk[keep - 1];
                    for (int e = (int)threadIdx.x; e < entries; e += kSelectThreads) {
                        const int b = e / most;
                        const double base = lds.base[b];
                        const bool ends = lds.ends[b] != 0;
                        if (!(base > kNone) || (ends && e - b * most != a.eos / kChunkCols)) continue;
                        const Entry of{ends ? base : base + ((double)tops[e] - lds.top[b]) * per_logit, e};
                        if (last.key - of.key < kNear && before(border_chunk, of)) left_out(of.key, b);
                    }
                }
            }
        }
        __syncthreads();
        const uint32_t near = round == 0 ? lds.near : 0u;
        if (near == 0) {
            if ((int)threadIdx.x < keep) {
                const Entry x = (int)threadIdx.x < kept ? lds.best[threadIdx.x] : Entry{kNone, 0};
                const int64_t at = seq * keep + threadIdx.x;
                a.parent_out[at] = (int)threadIdx.x < kept ? x.index / (int)a.V : -1;
                a.token_out[at] = (int)threadIdx.x < kept ? x.index % (int)a.V : -1;
                a.score_out[at] = (float)x.key;
            }
            return;
        }
        for (int b = 0; b < a.beams; ++b) {                                    // uniform
            if (((near >> b) & 1u) == 0 || lds.ends[b]) continue;
            const char* row = row_of(a, row0 + b, kBf16 ? 2 : 4);
            const double total = lds.log2_sum[b], top = lds.top[b];
            double sum = 0.0;
            for (int64_t col = threadIdx.x; col < a.V; col += kSelectThreads) {
                const float z = logit_at<kBf16>(row, col);
                const double x = fma((double)z - top, c, -total);
                if (x > -1000.0 && z > kNoLogit) sum += exp2_of(x);
            }
            sum = wave_sum(sum);
            if (lane == 0) lds.sums[wave] = sum;
            __syncthreads();
            if (threadIdx.x == 0) {
                double all = 0.0;
                for (int i = 0; i < kSelectWaves; ++i) all += lds.sums[i];
                lds.base[b] -= log(all);
            }
            __syncthreads();
        }
    }
}

hipError_t launch_beam_select(const BeamArgs& a, bool bf16, void* workspace, hipStream_t stream)
{
    const BeamShape s = beam_shape(a.seqs * a.beams, a.V, bf16);
    char* ws = static_cast<char*>(workspace);
    const float c = (float)(kLog2e / (double)a.tau);
    const int64_t items = a.seqs * a.beams * s.segments;
    const dim3 grid((uint32_t)((items + kStreamWaves - 1) / kStreamWaves));
    const auto stream_kernel = bf16 ? (c < kFlatBelow ? beam_stream_kernel<true, true> : beam_stream_kernel<true, false>)
                                    : (c < kFlatBelow ? beam_stream_kernel<false, true> : beam_stream_kernel<false, false>);
    stream_kernel<<<grid, 64 * kStreamWaves, 0, stream>>>(a, s, c, ws);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    if (bf16) beam_select_kernel<true><<<(uint32_t)a.seqs, kSelectThreads, 0, stream>>>(a, s, 1.0 / (double)a.tau, ws);
    else beam_select_kernel<false><<<(uint32_t)a.seqs, kSelectThreads, 0, stream>>>(a, s, 1.0 / (double)a.tau, ws);
    return hipGetLastError();
}

// ---------------------------------------------------------------- the beams' pages
// The first child of a beam goes on in its last page; every other child takes the last page of a beam without children (there are as
// many) and needs a copy of what its parent's holds.
__global__ __launch_bounds__(256)
void beam_reorder_kernel(ReorderArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t row0 = (int64_t)blockIdx.x * a.beams;
    int parent = -1, donor = -1, at = 0, len = 0, own = -1;
    if (lane < a.beams) {
        parent = a.parent[row0 + lane];
        if (parent < 0 || parent >= a.beams) parent = lane;
        len = a.row_lens[row0 + lane];
        len = len < 0 ? 0 : len;
        at = len / a.page_size;
        own = at < a.width ? a.row_pages[(row0 + lane) * a.width + at] : -1;   // the page that the row's next token goes to
    }
    uint32_t childless = 0, first = 0;
    for (int p = 0; p < a.beams; ++p) {
        const uint32_t children = (uint32_t)__ballot(parent == p);
        if (children != 0) first |= children & (0u - children);
        else childless |= 1u << p;
    }
    const bool other = lane < a.beams && ((first >> lane) & 1u) == 0;
    const uint32_t others = (uint32_t)__ballot(other);
    if (other) {                                                               // the j-th of them takes the j-th childless beam's
        uint32_t left = childless;
        for (int j = __builtin_popcount(others & ((1u << lane) - 1u)); j > 0; --j) left &= left - 1u;
        donor = __builtin_ctz(left);
    }
    const int from = lane < a.beams ? parent : 0;
    const int page = __shfl(own, other ? donor : from);                        // of the new row
    const int source = __shfl(own, from), parent_at = __shfl(at, from), parent_len = __shfl(len, from);
    if (threadIdx.x < 64 && lane < a.beams) {
        const int count = parent_len % a.page_size;
        const bool copy = other && count > 0 && page >= 0 && source >= 0;
        a.lens_out[row0 + lane] = parent_len;
        a.src_out[row0 + lane] = copy ? source : -1;
        a.dst_out[row0 + lane] = copy ? page : -1;
        a.counts_out[row0 + lane] = copy ? count : 0;
    }
    for (int r = threadIdx.x >> 6; r < a.beams; r += 4) {
        const int p = __builtin_amdgcn_readlane(parent, r), e = __builtin_amdgcn_readlane(parent_at, r), last = __builtin_amdgcn_readlane(page, r);
        const int32_t* in = a.row_pages + (row0 + p) * a.width;
        int32_t* out = a.pages_out + (row0 + r) * a.width;
        for (int i = lane; i < a.width; i += 64) out[i] = i == e ? last : in[i];
    }
}

hipError_t launch_beam_reorder(const ReorderArgs& a, hipStream_t stream)
{
    beam_reorder_kernel<<<(uint32_t)a.seqs, 256, 0, stream>>>(a);
    return hipGetLastError();
}

// A workgroup per page and head: its keys, values and scale bytes are four runs next to each other each.  (64 sequences x 8 beams, 4 heads of 128
// in 16 bits: 7.4 us for 23 MB in and out, in 8 bits 5.1 for 11.6, the tables before it 3.5; what bounds both is the start and a chain of two
// loads.)
__global__ __launch_bounds__(256)
void cache_copy_kernel(CacheView c, const int32_t* src, const int32_t* dst, const int32_t* counts)
{
    const int64_t i = blockIdx.x / (uint32_t)c.heads;
    const int head = (int)(blockIdx.x % (uint32_t)c.heads);
    const int from = src[i], to = dst[i];
    if (from == to || (uint32_t)from >= (uint64_t)c.num_pages || (uint32_t)to >= (uint64_t)c.num_pages) return;
    int n = counts[i];
    n = n < 0 ? 0 : n > c.page_size ? c.page_size : (n + 7) & ~7;
    const int64_t a = ((int64_t)from * c.heads + head) * c.page_size, b = ((int64_t)to * c.heads + head) * c.page_size;
    const int row = c.dim * (c.fp8 ? 1 : 2);
    const int64_t vectors = (int64_t)n * row / 16;
    const u32x4* k0 = reinterpret_cast<const u32x4*>(static_cast<const char*>(c.k) + a * row);
    const u32x4* v0 = reinterpret_cast<const u32x4*>(static_cast<const char*>(c.v) + a * row);
    u32x4* k1 = reinterpret_cast<u32x4*>(static_cast<char*>(c.k) + b * row);
    u32x4* v1 = reinterpret_cast<u32x4*>(static_cast<char*>(c.v) + b * row);
    for (int64_t j = threadIdx.x; j < vectors; j += 256) {
        const u32x4 x = k0[j], y = v0[j];
        k1[j] = x;
        v1[j] = y;
    }
    if (c.fp8)
        for (int j = threadIdx.x; j < n; j += 256) {
            c.k_scale[b + j] = c.k_scale[a + j];
            c.v_scale[b + j] = c.v_scale[a + j];
        }
}

hipError_t launch_cache_copy(const CacheView& c, const int32_t* src, const int32_t* dst, const int32_t* counts, int64_t n, hipStream_t stream)
{
    cache_copy_kernel<<<(uint32_t)(n * c.heads), 256, 0, stream>>>(c, src, dst, counts);
    return hipGetLastError();
}

}  // namespace e3
