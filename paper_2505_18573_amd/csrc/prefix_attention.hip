// Attention of a decode step for groups of rows that share a prefix (the rollouts of one question share its prompt).
//
//   row r of group g, query t of T, query head h:  keys = prefix of g ++ the first row_len - (T - 1 - t) own tokens,
//   s_j = scale q . k_j,   out = sum_j e^{s_j - m} v_j / l,   l = sum_j e^{s_j - m},   lse = m + ln l.
//
// The softmax's maximum and sum are running ones, and partial results (m, l, O) over disjoint sets of keys join exactly
// (O scaled by 2^{m - m'}), so the keys may be cut anywhere: into prefix and own tokens, and either into runs.  A
// prefix is read once for all rows of its group, whose queries form the columns of one product.
//
// Two launches:
//   attend   workgroups of four waves, as many as are resident together.  Each looks at all lengths first (device
//            memory: they change with every step).  A prefix or a row's own tokens ("unit"), a key head and a tile of
//            queries are an item.  Items of at most 16 queries are one wave's work, larger ones (64 queries at most) a
//            workgroup's, whose waves bring the keys into LDS for each other.  Items of either kind lie behind one another
//            on a line, measured in a wave's steps of 32 tokens and a few more for the item itself.  The workgroups are
//            divided between the two lines, and every wave (workgroup) takes an equal stretch of its line, whichever items it
//            falls into.  What it has of an item, (m, l, O), stays in registers and is left in the workspace as one partial
//            result.  (Runs of one length dealt round robin before: rows of 1 to 6000 tokens gave the busiest workgroup 1.6
//            times the mean.)
//   join     a workgroup per row and key head joins the partial results of its prefix and its own tokens.
//
// Registers instead of LDS: S^T = K Q^T puts the queries on the matrix instruction's columns, so a lane holds one
// query's scores and the softmax needs hardly any exchange; and since a sum over tokens may be taken in any order, row
// 4 g + i of the t-th 16 x 16 score tile is given token 8 g + 4 t + i of the step.  The eight scores of a lane are then
// tokens 8 g .. 8 g + 7, exactly the eight a lane has to hold of P^T as operand of O^T = V^T P^T.  The cache keeps eight
// tokens of a column together (kv_cache.h), so V^T comes from memory in that form too.
//
// An 8-bit cache is widened to bf16 (exactly) and its powers of two are applied to the scores and to P, both in fp32.
// P enters its product as the sum of three bf16 numbers, which hold all 24 bits of an fp32 weight, so everything between the
// loads and the output's own rounding is fp32.  Two of them (sixteen bits) would leave up to 2^-18 of each weight, visible where
// the terms of an output cancel; the third product costs nothing where memory is what the kernel waits for (512 rows
// below: 332.7 us, 333.0 with two), and 8 % where it is not (512 rows x 5 tokens: 329 us, 305 with two).
//
// What bounds it: reading keys and values, 5.1 TB/s at 512 rows x 28 heads of 128 over 4 key heads with prefixes of 100 to 1000 and 1 to
// 6000 own tokens (1.63 GB, 322 us; leaving out all products and exponentials changed nothing).  Small batches wait
// for chains of loads: 2.5 us for the lengths, about 8 us into and out of an item, 5 us for the join.  With several tokens a row
// the workgroups' line does more work per byte: 512 rows x 5 tokens with 500 + 5 to 2000 take 329 us at 1.9 TB/s, the vector
// units busy for half of the waves' time (64 of a step's 270 instructions widen codes), the rest of it barriers and LDS.
#include "kv_cache.h"
#include "stretch.h"
#include "vocab_common.h"
#include "vocab_pass.h"

namespace e3 {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kStep = 32;                       // tokens of a wave's step
constexpr int kAttendWaves = 4;
// What an item costs besides its steps, in steps (a chain of loads to its page, its keys and its queries).  16 rollouts x 8 with drafts
// 55.1 us with 2, 53.4 with 4, 55.8 with 8; 512 rows 336.0, 332.5, 335.6.
constexpr int kItemCost = 4;
// What a step of the workgroups' line costs against one of the waves' line, which waits for more memory.  512 rows 331.6 to 333.4 us with
// 0.5 to 0.7, 335.7 with 1 and 455 with 0.3, where the few workgroups of the prefixes end last; batches with hardly any work on one of the
// lines take the same with any of them (12 rows with a prefix of 32,771 tokens 50.9 to 52.5).
constexpr float kSharedCost = 0.6f;
// Steps of a stretch at least, on average: with more the join has fewer parts, with fewer the few steps of a small batch are taken side
// by side.  One row with 150 + 77 tokens (32 steps) 13.0 us with 1, 13.6 with 2, 15.1 with 4; with 8192 tokens (1048 steps) 24.2,
// 20.0 and 18.4.
__device__ __forceinline__ int least_stretch(int64_t steps) { return steps < 512 ? 1 : steps < 1024 ? 2 : 4; }
constexpr int kWaveQueries = 16;                // an item of so many is a wave's
constexpr float kNoScore = -3.0e38f;            // running maximum before any score
constexpr float kSlack = 8.0f;                  // scores may pass the running maximum by this (2^8) before it moves

enum { kByGroup = 0, kByWave = 1 };             // the two lines

// What the host fixes of a call; the workspace's parts lie behind one another.
struct AttendShape {
    int32_t R, M;                               // query heads per key head; queries of a row and key head (T * R)
    int32_t units;                              // groups, then rows
    int32_t slot[2];                            // queries that an item of either line leaves results of, at most
    int64_t slots[2];                           // places for its partial results
    int64_t at_items, at_ml, at_o, bytes;       // byte offsets (at_items: Parts; at_o: fp32 [results][D])
};

// Where the partial results of an item lie: `first` and the places behind it.
struct Parts { int32_t first, count; };

static int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Tiles of 16 queries that the waves of a workgroup share: as many as a unit's queries fill, up to one per wave.
__host__ __device__ __forceinline__ int query_waves(int64_t queries) { return queries <= 16 ? 1 : queries <= 32 ? 2 : 4; }
__host__ __device__ __forceinline__ int64_t query_tiles(int64_t queries)
{
    const int per = 16 * query_waves(queries);
    return (queries + per - 1) / per;
}

// The unit's first item in the list of items: rows first, a fixed number of tiles each; a group of n rows has n * M / 64 tiles or
// one more.  The key heads of a tile lie next to each other.
__device__ __forceinline__ int64_t first_item(const AttendShape& s, int rows, int heads, bool prefix, int group, int row0)
{
    const int64_t of_rows = query_tiles(s.M);
    return heads * (prefix ? rows * of_rows + (int64_t)row0 * s.M / 64 + group : row0 * of_rows);
}

// Workgroups per compute unit, which are waves per SIMD, that the registers allow.
constexpr int attend_occupancy(int64_t D) { return D == 64 ? 3 : 2; }

static bool attend_shape(int64_t rows, int64_t T, int64_t q_heads, int64_t heads, int64_t D, int64_t groups, AttendShape& s)
{
    s.R = (int32_t)(q_heads / heads);
    const int64_t M = T * s.R;
    if (M > (1 << 16) || rows * heads >= (1 << 24)) return false;              // threads of the join: below 2^32
    s.M = (int32_t)M;
    s.units = (int32_t)(groups + rows);
    // an item, or a part of it, per place: no more parts than items and workers together
    const int64_t workgroups = compute_units() * attend_occupancy(D);
    const int64_t most = groups > 0 ? rows * M : M;               // queries of a unit
    s.slot[kByGroup] = (int32_t)(most < 64 ? most : 64);
    s.slot[kByWave] = (int32_t)(most < 16 ? most : 16);
    s.slots[kByGroup] = most > kWaveQueries
        ? workgroups + heads * ((M > kWaveQueries ? rows * query_tiles(M) : 0) + (groups > 0 ? rows * M / 64 + groups : 0)) : 0;
    s.slots[kByWave] = workgroups * kAttendWaves + heads * ((M > kWaveQueries ? 0 : rows) + groups);
    const int64_t places = s.slots[0] * s.slot[0] + s.slots[1] * s.slot[1];
    if (s.slots[0] + s.slots[1] > (int64_t)1 << 30 || places > ((int64_t)1 << 31) - 1) return false;
    s.at_items = 0;
    s.at_ml = up(heads * (rows * query_tiles(M) + (groups > 0 ? rows * M / 64 + groups : 0)) * (int64_t)sizeof(Parts), 256);
    s.at_o = up(s.at_ml + places * 8, 256);
    s.bytes = up(s.at_o + places * D * 4, 256);
    return true;
}

size_t prefix_attention_workspace_bytes(int64_t rows, int64_t T, int64_t q_heads, int64_t heads, int64_t dim, int64_t groups)
{
    AttendShape s;
    return attend_shape(rows, T, q_heads, heads, dim, groups, s) ? (size_t)s.bytes : 0;
}

// ---------------------------------------------------------------- plan
constexpr int kPlanThreads = 64 * kAttendWaves;

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

// A group's prefix or a row's own tokens.
struct Unit {
    int len, row0;                              // tokens; the first row that sees them
    int64_t queries;                            // per key head
    int items, steps;                           // (tile, key head) pairs, and a wave's steps in each with kItemCost; 0: nothing to do
    int line;
};
__device__ __forceinline__ int round_tokens(int64_t queries) { return queries <= kWaveQueries ? kStep : kStep * kAttendWaves / query_waves(queries); }
__device__ __forceinline__ Unit unit_at(const AttentionArgs& a, const AttendShape& s, int heads, int page_size, int u)
{
    Unit x;
    if (u < a.groups) {
        x.row0 = clamp_len(a.group_offsets[u], a.rows);
        const int n = clamp_len(a.group_offsets[u + 1], a.rows) - x.row0;
        x.len = n > 0 ? clamp_len(a.prefix_lens[u], table_tokens(a.prefix_width, page_size)) : 0;
        x.queries = (int64_t)(n > 0 ? n : 0) * s.M;
    } else {
        x.row0 = u - a.groups;
        x.len = clamp_len(a.row_lens[x.row0], table_tokens(a.row_width, page_size));
        x.queries = s.M;
    }
    const int apart = round_tokens(x.queries);
    x.line = x.queries <= kWaveQueries ? kByWave : kByGroup;
    x.items = x.len > 0 ? (int)(query_tiles(x.queries) * heads) : 0;
    x.steps = x.len > 0 ? (int)(((int64_t)x.len + apart - 1) / apart) + kItemCost : 0;
    return x;
}
__device__ __forceinline__ Unit uniform(const Unit& x)
{
    return Unit{uniform(x.len), uniform(x.row0), uniform(x.queries), uniform(x.items), uniform(x.steps), uniform(x.line)};
}

// Every thread sums up a share of successive units; `first` gets each share's first step and item on either line.
struct Plan {
    int share;                                  // units of a share
    int64_t steps[2];
    int groups;                                 // workgroups that work on the line of workgroups
    int parts[2];                               // stretches
};
struct PlanLds {
    int64_t first[2][kPlanThreads];
    int first_item[2][kPlanThreads];
    int64_t sums[kAttendWaves][3];
};
__device__ __forceinline__ Plan make_plan(const AttentionArgs& a, const AttendShape& s, int heads, int page_size, PlanLds& lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Plan p;
    p.share = (s.units + kPlanThreads - 1) / kPlanThreads;
    const int u0 = (int)threadIdx.x * p.share;
    const int u1 = u0 + p.share < s.units ? u0 + p.share : s.units;
    int64_t own[3] = {0, 0, 0};                                                // steps of both lines; items, those of waves in the upper half
    for (int u = u0; u < u1; ++u) {
        const Unit x = unit_at(a, s, heads, page_size, u);
        const int64_t steps = (int64_t)x.items * x.steps;
        own[0] += x.line == kByGroup ? steps : 0;
        own[1] += x.line == kByWave ? steps : 0;
        own[2] += x.line == kByWave ? (int64_t)x.items << 32 : x.items;
    }
    int64_t sum[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        sum[k] = own[k];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t y = __shfl_up(sum[k], d);
            if (lane >= d) sum[k] += y;
        }
        if (lane == 63) lds.sums[wave][k] = sum[k];
        sum[k] -= own[k];
    }
    __syncthreads();
    int64_t all[3] = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < kAttendWaves; ++i)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            if (i < wave) sum[k] += lds.sums[i][k];
            all[k] += lds.sums[i][k];
        }
    lds.first[0][threadIdx.x] = sum[0];
    lds.first[1][threadIdx.x] = sum[1];
    lds.first_item[0][threadIdx.x] = (int)(uint32_t)sum[2];
    lds.first_item[1][threadIdx.x] = (int)(sum[2] >> 32);
    p.steps[0] = uniform(all[0]);
    p.steps[1] = uniform(all[1]);
    // the workgroups are divided by what the lines cost; four waves of one take four steps of the waves' line at a time
    const float of_groups = (float)p.steps[kByGroup] * kSharedCost, of_waves = (float)p.steps[kByWave] * (1.0f / kAttendWaves);
    const int n = (int)gridDim.x;
    int share = (int)(of_groups / (of_groups + of_waves) * (float)n + 0.5f);
    if (p.steps[kByWave] > 0 && share > n - 1) share = n - 1;
    if (p.steps[kByGroup] > 0 && share < 1) share = 1;
    p.groups = p.steps[kByGroup] == 0 ? 0 : uniform(share);
    const int64_t waves = (int64_t)(n - p.groups) * kAttendWaves;
    const int64_t most[2] = {p.groups, waves};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int least = least_stretch(p.steps[k]);
        const int64_t enough = (p.steps[k] + least - 1) / least;
        p.parts[k] = (int)(enough < most[k] ? enough : most[k]);
    }
    __syncthreads();
    return p;
}
// The unit that holds a step of a line, with the unit's first step and item; uniform.
struct Place {
    int unit, item;
    int64_t step;
    Unit of;
};
__device__ __forceinline__ Place place_of(const AttentionArgs& a, const AttendShape& s, int heads, int page_size, const Plan& p,
                                          const PlanLds& lds, int line, int64_t step)
{
    const int lane = threadIdx.x & 63;
    // the last share that begins at or before the step
    int below = 0;
#pragma unroll
    for (int k = 0; k < kPlanThreads / 64; ++k) below += (int)__popcll(__ballot(lds.first[line][k * 64 + lane] <= step));
    const int share = uniform(below) - 1;
    Place r{};
    r.unit = -1;
    r.step = uniform(lds.first[line][share]);
    r.item = uniform(lds.first_item[line][share]);
    for (int u0 = share * p.share; u0 < s.units && u0 < (share + 1) * p.share; u0 += 64) {
        const int u = u0 + lane;
        Unit x{};
        if (u < s.units && u < (share + 1) * p.share) x = unit_at(a, s, heads, page_size, u);
        int items = x.line == line ? x.items : 0;
        const int own_items = items;
        const int64_t own = (int64_t)items * x.steps;
        int64_t sum = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t y = __shfl_up(sum, d);
            const int z = __shfl_up(items, d);
            if (lane >= d) { sum += y; items += z; }
        }
        const unsigned long long behind = __ballot(r.step + sum > step);
        const int l = behind != 0ull ? (int)__builtin_ctzll(behind) : 63;
        r.step += uniform(__shfl(sum, l));
        r.item += __builtin_amdgcn_readlane(items, l);
        if (behind != 0ull) {
            r.unit = u0 + l;
            r.step -= uniform(__shfl(own, l));
            r.item -= __builtin_amdgcn_readlane(own_items, l);
            r.of.len = __builtin_amdgcn_readlane(x.len, l);
            r.of.row0 = __builtin_amdgcn_readlane(x.row0, l);
            r.of.queries = uniform(__shfl(x.queries, l));
            r.of.items = __builtin_amdgcn_readlane(x.items, l);
            r.of.steps = __builtin_amdgcn_readlane(x.steps, l);
            r.of.line = line;
            break;
        }
    }
    return r;
}

struct Task {
    int unit, head, tile, from, to;             // tokens [from, to)
    Unit of;
};

// ---------------------------------------------------------------- attend
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
        return ((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
    }
    // whether the lane holds a value that is no finite number
    __device__ __forceinline__ bool unbounded() const
    {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < kVLoads; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) bad |= unbounded_in(v[i][j]);
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

template <int D, bool kFp8>
struct Attend {
    using Data = StepData<D, kFp8>;
    static constexpr int kBlocks = D / 16, kSteps = D / 32;
    bf16x8 q[kSteps];
    f32x4 o[kBlocks];
    float m, l;
    int limit;                                  // tokens the lane's query sees (of the prefix, of the row)

    // One step.  `at`: its first token; every query sees at least `sure` tokens, none more than `most`, and the tokens from there
    // on are cleared.  key_factor, value_factor: what a token's score and weight are multiplied by.  The keys' registers
    // are free for the next step's (next_keys) as soon as the scores are there, the values' (next_values) at the end.
    template <typename KeyFactor, typename ValueFactor, typename Keys, typename Values>
    __device__ __forceinline__ void step(Data& d, int at, int sure, int most, int lane, KeyFactor key_factor, ValueFactor value_factor,
                                         Keys next_keys, Values next_values)
    {
        const int g = lane >> 4;
        const bool tail = at + kStep > sure;                              // uniform
        const int see = limit < most ? limit : most;
        f32x4 s[2] = {f32x4{0.0f, 0.0f, 0.0f, 0.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = mfma(d.key(t, i), q[i], s[t]);
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = s[j >> 2][j & 3] * key_factor(j);
            if (tail) x[j] = at + 8 * g + j < see ? x[j] : -INFINITY;
        }
        next_keys();
        float top = fmax3(fmax3(x[0], x[1], x[2]), fmax3(x[3], x[4], x[5]), fmaxf(x[6], x[7]));
        if (__any(top > m + kSlack)) {
            // the queries' maxima over the four lanes that hold their scores
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float to = fmaxf(m, top);
            const float f = __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) o[b] *= f;
        }
        bf16x8 p, rest, last;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = __builtin_amdgcn_exp2f(x[j] - m);
            l += e;
            const float w = kFp8 ? e * value_factor(j) : e;
            p[j] = (__bf16)w;
            const float left = w - (float)p[j];
            rest[j] = (__bf16)left;
            last[j] = (__bf16)(left - (float)rest[j]);
        }
        // Tokens that some queries see and others do not: a weight of zero keeps them out, unless the value is no
        // finite number.  Such values leave the product, and one more counts those that a query sees.
        if (__builtin_expect(tail && sure < most && __any(d.unbounded()), 0)) {
            bf16x8 seen;
#pragma unroll
            for (int j = 0; j < 8; ++j) seen[j] = (__bf16)(at + 8 * g + j < see ? 1.0f : 0.0f);
            Data ones;
            ones.take_unbounded(d);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                const f32x4 count = mfma(ones.value(b), seen, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
                for (int k = 0; k < 4; ++k) o[b][k] = count[k] > 0.0f ? __builtin_nanf("") : o[b][k];
            }
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const bf16x8 value = d.value(b);
            o[b] = mfma(value, last, mfma(value, rest, mfma(value, p, o[b])));
        }
        next_values();
    }

    // The queries of a wave: column n is query first + n of the unit.
    __device__ __forceinline__ void begin(const AttentionArgs& a, const AttendShape& sh, const Task& task, int first, int lane)
    {
        const int col = lane & 15, g = lane >> 4;
        const int qi = first + col;
        const bool is = qi < task.of.queries;
        const int row = task.of.row0 + (is ? qi / sh.M : 0), in_row = is ? qi % sh.M : 0;
        const int t = in_row / sh.R, h = task.head * sh.R + in_row % sh.R;
        const uint16_t* qp = a.q + row * a.q_row_stride + t * a.q_token_stride + h * a.q_head_stride;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            u32x4 w = *reinterpret_cast<const u32x4*>(qp + Data::key_column(s, g));
            if (!is) w = u32x4{0, 0, 0, 0};
            q[s] = __builtin_bit_cast(bf16x8, w);
        }
        const int own = task.of.len - (a.T - 1 - t);
        limit = task.unit < a.groups ? task.of.len : own > 0 ? own : 0;
        m = kNoScore;
        l = 0.0f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) o[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // The partial result: l is spread over the four lanes of a query until here.
    __device__ __forceinline__ void leave(int queries, float2* ml_out, float* o_out, int lane)
    {
        const int col = lane & 15, g = lane >> 4;
        if (col >= queries) return;
        if (g == 0) ml_out[col] = float2{m, l};
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int k = 0; k < 4; ++k) o_out[(int64_t)col * D + Data::column(b, 4 * g + k)] = o[b][k];
    }
    // every query of the unit sees so many of its tokens
    static __device__ __forceinline__ int seen_by_all(const AttentionArgs& a, const Task& task)
    {
        const int n = task.of.len - (a.T - 1);
        return task.unit < a.groups ? task.of.len : n > 0 ? n : 0;
    }
    static __device__ __forceinline__ const int32_t* pages_of(const AttentionArgs& a, const Task& task)
    {
        return task.unit < a.groups ? a.prefix_pages + (int64_t)task.unit * a.prefix_width
                                    : a.row_pages + (int64_t)task.of.row0 * a.row_width;
    }
    // Where the step at token `at` lies.  A page that the cache does not have is not seen; page 0 is read in its place.
    static __device__ __forceinline__ int64_t row_of(const CacheView& c, const Task& task, int page, int at)
    {
        const int64_t p = (uint32_t)page < (uint64_t)c.num_pages ? page : 0;
        return (p * c.heads + task.head) * c.page_size + (at & (c.page_size - 1));
    }

    // A wave's task: all of the unit's queries, steps one after the other.
    __device__ __forceinline__ void direct(const CacheView& c, const AttentionArgs& a, const AttendShape& sh, const Task& task,
                                           float2* ml_out, float* o_out)
    {
        const int lane = threadIdx.x & 63;
        const int to = task.to, len = task.of.len, sure = seen_by_all(a, task);
        const int32_t* pages = pages_of(a, task);
        auto page_at = [&](int at) { return at < to ? pages[at >> c.page_shift] : -1; };
        int at = task.from;
        Data d;
        int page = page_at(at), page_next = page_at(at + kStep);
        d.load_keys(c, row_of(c, task, page, at), lane);
        d.load_values(c, row_of(c, task, page, at), lane);
        begin(a, sh, task, 0, lane);
        const float scale = a.scale * kLog2eF;
        for (; at < to; at += kStep) {
            const int page_after = page_at(at + 2 * kStep);
            const int64_t next = row_of(c, task, page_next, at + kStep);       // behind the last step: read for nothing
            const bool there = (uint32_t)page < (uint64_t)c.num_pages;
            const int most = there ? len : -1;
            if (at + kStep > (there ? sure : -1)) d.clear_from(most - at - 8 * (lane >> 4));
            step(d, at, there ? sure : -1, most, lane, [&](int j) { return kFp8 ? scale * d.k_factor(j) : scale; },
                 [&](int j) { return d.v_factor(j); }, [&] { d.load_keys(c, next, lane); }, [&] { d.load_values(c, next, lane); });
            page = page_next;
            page_next = page_after;
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        leave((int)task.of.queries, ml_out, o_out, lane);
    }

    // A workgroup's task: a tile of 16 queries per wave, or per two waves, which then take steps in turn.  Each wave brings one
    // step of four into LDS, in registers while the last four are worked on.
    // lds: four steps and whether their pages exist; then (m, l) of all waves and O of two.
    static constexpr int kLds = (kAttendWaves * Data::kImage + 16) > (kAttendWaves * 16 * 8 + 2 * kBlocks * 64 * 16)
                                    ? (kAttendWaves * Data::kImage + 16) : (kAttendWaves * 16 * 8 + 2 * kBlocks * 64 * 16);
    __device__ __forceinline__ void shared(const CacheView& c, const AttentionArgs& a, const AttendShape& sh, const Task& task,
                                           char* lds, float2* ml_out, float* o_out)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int col = lane & 15, g = lane >> 4;
        const int qw = task.of.queries <= 32 ? 2 : 4, qs = qw == 2 ? 1 : 2;
        const int tile = wave & (qw - 1), share = wave >> qs, shares = kAttendWaves >> qs;
        const int first = (task.tile * qw + tile) * 16, queries = (int)task.of.queries;
        const int to = task.to, len = task.of.len, sure = seen_by_all(a, task);
        const int32_t* pages = pages_of(a, task);
        auto page_at = [&](int at) { return at < to ? pages[at >> c.page_shift] : -1; };
        int* there = reinterpret_cast<int*>(lds + kAttendWaves * Data::kImage);
        constexpr int kFour = kAttendWaves * kStep;
        auto nothing = [] {};
        Data mine;
        int own = task.from + wave * kStep;
        int page = page_at(own), page_next = page_at(own + kFour);
        mine.load_keys(c, row_of(c, task, page, own), lane);
        mine.load_values(c, row_of(c, task, page, own), lane);
        begin(a, sh, task, first, lane);
        const float scale = a.scale * kLog2eF;
        for (int at = task.from; at < to; at += kFour, own += kFour) {
            __syncthreads();                                               // the last four (or the last task) are done with
            const bool has = (uint32_t)page < (uint64_t)c.num_pages;
            if (own + kStep > (has ? sure : -1)) mine.clear_from((has ? len : -1) - own - 8 * g);
            mine.put(lds + wave * Data::kImage, scale, lane);
            if (lane == 0) there[wave] = has;
            __syncthreads();
            page = page_next;
            page_next = page_at(own + 2 * kFour);
            if (at + kFour < to) {                                         // uniform: the barriers would wait for loads of nothing
                mine.load_keys(c, row_of(c, task, page, own + kFour), lane);
                mine.load_values(c, row_of(c, task, page, own + kFour), lane);
            }
            if (first < queries) {
                for (int i = share; i < kAttendWaves && at + i * kStep < to; i += shares) {
                    Data d;
                    d.take(lds + i * Data::kImage, lane);
                    const bool is = uniform(there[i]) != 0;
                    const float* factors = Data::factors(lds + i * Data::kImage, lane);
                    step(d, at + i * kStep, is ? sure : -1, is ? len : -1, lane, [&](int j) { return kFp8 ? factors[j] : scale; },
                         [&](int j) { return factors[kStep + j]; }, nothing, nothing);
                }
            }
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (shares > 1) {                                                  // two waves with the same queries
            float2* ml = reinterpret_cast<float2*>(lds);
            f32x4* part = reinterpret_cast<f32x4*>(lds + kAttendWaves * 16 * 8);           // [2][kBlocks][64]
            __syncthreads();
            if (g == 0) ml[wave * 16 + col] = float2{m, l};
            __syncthreads();
            const float2 other = ml[(wave ^ qw) * 16 + col];
            const float all = fmaxf(m, other.x);
            const float f = __builtin_amdgcn_exp2f(m - all);
            l = l * f + other.y * __builtin_amdgcn_exp2f(other.x - all);
            m = all;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                o[b] *= f;
                if (share == 1) part[(tile * kBlocks + b) * 64 + lane] = o[b];
            }
            __syncthreads();
            if (share == 0) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) o[b] += part[(tile * kBlocks + b) * 64 + lane];
            }
        }
        if (share == 0) leave(queries - first, ml_out + tile * 16, o_out + (int64_t)tile * 16 * D, lane);
    }
};

// The stretch of worker `part` on a line: f(task, place of its result).
template <int kLine, typename F>
__device__ __forceinline__ void along_line(const AttentionArgs& a, const AttendShape& s, const CacheView& c, const Plan& plan, const PlanLds& lds,
                                           Parts* items, int part, F f)
{
    if (part >= plan.parts[kLine]) return;
    const int lane = threadIdx.x & 63;
    int64_t at = begin_of(part, plan.steps[kLine], plan.parts[kLine]);
    const int64_t end = begin_of(part + 1, plan.steps[kLine], plan.parts[kLine]);
    Place u = place_of(a, s, c.heads, c.page_size, plan, lds, kLine, at);
    while (at < end && u.unit >= 0) {
        const Piece piece = piece_at(at - u.step, end - at, u.of.steps);
        const int item = piece.item, from = piece.from, n = piece.n;
        const int apart = round_tokens(u.of.queries);
        const int real_from = from > kItemCost ? from - kItemCost : 0, real_to = from + n - kItemCost;
        Task task;
        task.unit = u.unit;
        task.head = item % c.heads;
        task.tile = item / c.heads;
        task.from = real_from * apart;
        task.to = u.of.len < (int64_t)real_to * apart ? u.of.len : real_to * apart;
        task.of = u.of;
        const int64_t place = (int64_t)part + u.item + item;
        if (real_to > 0) {
            // (groups that overlap, against the contract, could exceed the places, or the 32 bits that items are counted in)
            if (from <= kItemCost && lane == 0) {                              // the item's first part
                const int last = part_of(at - from + u.of.steps - 1, plan.steps[kLine], plan.parts[kLine]);
                const int64_t i = first_item(s, a.rows, c.heads, u.unit < a.groups, u.unit, u.of.row0) + item;
                items[i] = Parts{(int)place, place >= 0 && place + (last - part) < s.slots[kLine] ? last - part + 1 : 0};
            }
            if (place >= 0 && place < s.slots[kLine]) f(task, place);
        }
        at += n;
        if (at < end && item + 1 == u.of.items && from + n == u.of.steps) {
            const int next = u.unit + 1;
            Unit x{};
            if (next < s.units) x = uniform(unit_at(a, s, c.heads, c.page_size, next));
            if (x.items > 0 && x.line == kLine) {
                u.step = at;
                u.item += u.of.items;
                u.unit = next;
                u.of = x;
            } else {
                u = place_of(a, s, c.heads, c.page_size, plan, lds, kLine, at);
            }
        }
    }
}

template <int D, bool kFp8>
__global__ __launch_bounds__(64 * kAttendWaves, attend_occupancy(D))
void attend_kernel(CacheView c, AttentionArgs a, AttendShape s, char* ws)
{
    __shared__ __align__(16) char lds[Attend<D, kFp8>::kLds];
    __shared__ PlanLds plan_lds;
    const Plan plan = make_plan(a, s, c.heads, c.page_size, plan_lds);
    Parts* items = reinterpret_cast<Parts*>(ws + s.at_items);
    float2* ml = reinterpret_cast<float2*>(ws + s.at_ml);
    float* o = reinterpret_cast<float*>(ws + s.at_o);
    if ((int)blockIdx.x < plan.groups) {
        along_line<kByGroup>(a, s, c, plan, plan_lds, items, blockIdx.x, [&](const Task& task, int64_t place) {
            const int64_t at = place * s.slot[kByGroup];
            Attend<D, kFp8> x;
            x.shared(c, a, s, task, lds, ml + at, o + at * D);
        });
        return;
    }
    // a workgroup's waves lie far apart on their line: few stretches are spread over all workgroups
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = wave * ((int)gridDim.x - plan.groups) + (int)blockIdx.x - plan.groups;
    along_line<kByWave>(a, s, c, plan, plan_lds, items, part, [&](const Task& task, int64_t place) {
        const int64_t at = s.slots[kByGroup] * s.slot[kByGroup] + place * s.slot[kByWave];
        Attend<D, kFp8> x;
        x.direct(c, a, s, task, ml + at, o + at * D);
    });
}

// ---------------------------------------------------------------- join
// The partial results of a query's prefix and of its row's own tokens become its output.  What bounds it is the chain of loads
// (lengths, list of items, results), so a wave takes several queries at once, D / 4 lanes each with four columns,
// and asks for (m, l) and O of four parts together.
constexpr int join_queries(int D) { return 4 * 256 / D; }          // of a workgroup of 256 at most

struct Merged {
    float m, l;
    f32x4 o;
};
__device__ __forceinline__ void merge(Merged& x, float m, float l, const f32x4& o)
{
    const float up = fmaxf(x.m, m);
    const float f = __builtin_amdgcn_exp2f(x.m - up), g = __builtin_amdgcn_exp2f(m - up);
    x.m = up;
    x.l = x.l * f + l * g;
    x.o = x.o * f + o * g;
}

// (Eight waves per SIMD: 2048 workgroups, those of 512 rows and four key heads, are then resident together.)
template <int D>
__global__ __launch_bounds__(256, 8)
void attend_join_kernel(AttentionArgs a, AttendShape s, int heads, int page_size, int per_group, const char* ws)
{
    constexpr int kLanes4 = D / 4;                                             // lanes of a query
    __shared__ float lds[256 / kLanes4][2 + D];
    const int lane = threadIdx.x & 63;
    const int sub = threadIdx.x / kLanes4, col = (threadIdx.x % kLanes4) * 4;
    const int head = blockIdx.x % heads, row = blockIdx.x / heads;
    const Parts* items = reinterpret_cast<const Parts*>(ws + s.at_items);
    const float2* ml = reinterpret_cast<const float2*>(ws + s.at_ml);
    const float* o = reinterpret_cast<const float*>(ws + s.at_o);
    const int first_query = blockIdx.y * per_group;
    const int end_query = first_query + per_group < s.M ? first_query + per_group : s.M;

    const Unit of_row = uniform(unit_at(a, s, heads, page_size, a.groups + row));
    // The row's group is the last one that begins at or before it.  All lanes look, at a 64th of the groups each until there are no
    // more than 64 left, whose lengths they ask for as well.  (64 after 64 from the first on before: 512 groups of eight rows
    // and four key heads 104 us, now 74.)
    int group = -1, left = a.groups;
    while (left > 64) {
        const int apart = (left + 63) / 64, at = lane * apart;
        const int n = (int)__popcll(__ballot(at < left && a.group_offsets[group + 1 + (at < left ? at : 0)] <= row));
        if (n == 0) { left = 0; break; }                                       // before the first group
        group += (n - 1) * apart;
        left = left - (n - 1) * apart < apart ? left - (n - 1) * apart : apart;
    }
    Unit of_prefix{};
    if (left > 0) {
        const int g = group + 1 + (lane < left ? lane : left - 1);
        const Unit x = unit_at(a, s, heads, page_size, g);
        const int n = (int)__popcll(__ballot(lane < left && a.group_offsets[g] <= row));
        if (n > 0) {
            group += n;
            of_prefix.row0 = __builtin_amdgcn_readlane(x.row0, n - 1);
            of_prefix.queries = __builtin_amdgcn_readlane((int)x.queries, n - 1);
            of_prefix.items = __builtin_amdgcn_readlane(x.items, n - 1);
            of_prefix.line = __builtin_amdgcn_readlane(x.line, n - 1);
        }
    }
    const int prefix_query = (row - of_prefix.row0) * s.M;

    // A query's parts: n1 of the prefix, then the row's.
    struct Found {
        int n1, n, first1, apart1, first2, apart2;
        __device__ __forceinline__ int64_t place(int i) const { return i < n1 ? first1 + (int64_t)i * apart1 : first2 + (int64_t)(i - n1) * apart2; }
    };
    auto find = [&](int in_row) {
        auto of = [&](const Unit& x, bool prefix, int qi, int* first, int* apart) {
            *first = *apart = 0;
            if (x.items == 0 || qi >= x.queries) return 0;
            const int per = 16 * query_waves(x.queries);
            const Parts parts = items[first_item(s, a.rows, heads, prefix, group, x.row0) + (int64_t)(qi / per) * heads + head];
            *apart = x.line == kByWave ? s.slot[kByWave] : s.slot[kByGroup];
            // results of the line of workgroups come first
            *first = (int)((x.line == kByWave ? s.slots[kByGroup] * s.slot[kByGroup] : 0) + (int64_t)parts.first * *apart + qi % per);
            return parts.count;
        };
        Found f;
        const int n2 = of(of_row, false, in_row, &f.first2, &f.apart2);
        f.n1 = of(of_prefix, true, prefix_query + in_row, &f.first1, &f.apart1);
        f.n = f.n1 + n2;
        return f;
    };
    // parts from, from + apart, ... of a query
    auto join = [&](const Found& f, int from, int apart) {
        Merged x{kNoScore, 0.0f, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
        for (int i = from; i < f.n; i += 4 * apart) {
            float2 w[4];
            f32x4 p[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t at = f.place(i + k * apart < f.n ? i + k * apart : i);
                w[k] = ml[at];
                p[k] = *reinterpret_cast<const f32x4*>(o + at * D + col);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k * apart < f.n) merge(x, w[k].x, w[k].y, p[k]);
        }
        return x;
    };
    auto write = [&](const Merged& x, int in_row) {
        const int t = in_row / s.R, h = head * s.R + in_row % s.R;
        const int64_t where = ((int64_t)row * a.T + t) * a.q_heads + h;
        const bool none = x.l == 0.0f && x.m == kNoScore;                      // no key at all
        const float inv = none ? 0.0f : 1.0f / x.l;
        const bf16x2 lo = {(__bf16)(x.o[0] * inv), (__bf16)(x.o[1] * inv)}, hi = {(__bf16)(x.o[2] * inv), (__bf16)(x.o[3] * inv)};
        *reinterpret_cast<u32x2*>(a.out + where * D + col) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
        if (a.lse && col == 0) a.lse[where] = none ? -INFINITY : (x.m + __builtin_amdgcn_logf(x.l)) * (float)kLn2;
    };
    // lanes of as many queries as there are; fewer queries have their parts spread over several lots of lanes
    constexpr int kSubs = 256 / kLanes4;
    const int queries = end_query - first_query, spread = kSubs / queries;     // uniform, at least one
    const int query = sub / spread, in_row = first_query + query;
    Merged x{kNoScore, 0.0f, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
    if (query < queries) x = join(find(in_row), sub % spread, spread);
    if (spread > 1) {
        if (col == 0) { lds[sub][0] = x.m; lds[sub][1] = x.l; }
#pragma unroll
        for (int j = 0; j < 4; ++j) lds[sub][2 + col + j] = x.o[j];
        __syncthreads();
        if (sub % spread != 0) return;
        for (int k = sub + 1; k < sub + spread && k < kSubs; ++k)
            merge(x, lds[k][0], lds[k][1], f32x4{lds[k][2 + col], lds[k][3 + col], lds[k][4 + col], lds[k][5 + col]});
    }
    if (query < queries) write(x, in_row);
}

template <int D, bool kFp8>
static hipError_t launch_attend(const CacheView& c, const AttentionArgs& a, const AttendShape& s, char* ws, hipStream_t stream)
{
    const int workgroups = compute_units() * attend_occupancy(D);
    attend_kernel<D, kFp8><<<workgroups, 64 * kAttendWaves, 0, stream>>>(c, a, s, ws);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    // Queries of a workgroup of the join: fewer where there are few workgroups, whose queries have many parts (12 rows x 8 heads
    // with a prefix of 32,771: the join 8.1 us, and 15.4 with all four queries together).
    int per_group = join_queries(D) < s.M ? join_queries(D) : s.M;
    const int64_t pairs = (int64_t)a.rows * c.heads;
    while (per_group > 1 && pairs * ((s.M + per_group - 1) / per_group) < compute_units() * 2) per_group = (per_group + 1) / 2;
    const dim3 grid((uint32_t)pairs, (uint32_t)((s.M + per_group - 1) / per_group));
    attend_join_kernel<D><<<grid, 256, 0, stream>>>(a, s, c.heads, c.page_size, per_group, ws);
    return hipGetLastError();
}

hipError_t launch_prefix_attention(const CacheView& c, const AttentionArgs& a, void* workspace, hipStream_t stream)
{
    AttendShape s;
    if (!attend_shape(a.rows, a.T, a.q_heads, c.heads, c.dim, a.groups, s)) return hipErrorInvalidValue;
    char* ws = static_cast<char*>(workspace);
    if (c.dim == 128) return c.fp8 ? launch_attend<128, true>(c, a, s, ws, stream) : launch_attend<128, false>(c, a, s, ws, stream);
    return c.fp8 ? launch_attend<64, true>(c, a, s, ws, stream) : launch_attend<64, false>(c, a, s, ws, stream);
}

}  // namespace e3
