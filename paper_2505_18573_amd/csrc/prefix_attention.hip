// Attention of a decode step for groups of rows that share a prefix (the rollouts of one question share its prompt).
//
//   row r of group g, query t of T, query head h:  keys = prefix of g ++ the first row_len - (T - 1 - t) own tokens,
//   s_j = scale q . k_j,   out = sum_j e^{s_j - m} v_j / l,   l = sum_j e^{s_j - m},   lse = m + ln l.
//
// The softmax's maximum and sum are running ones, and partial results (m, l, O) over disjoint sets of keys join exactly
// (O scaled by 2^{m - m'}), so the keys may be cut anywhere: into prefix and own tokens, and either into runs.  A
// prefix is read once for all rows of its group, whose queries form the columns of one product.
//
// Three launches:
//   plan     one workgroup looks at the lengths (device memory: they change with every step) and lists the tasks: a run
//            of tokens of one prefix or one row, a key head, a tile of queries.  Runs are of one length, chosen so that
//            the tasks fill the card some times over.
//   attend   workgroups of four waves take tasks; each wave takes every fourth step of 32 tokens of the run and keeps
//            its own (m, l, O) in registers; the four join through LDS and leave one partial result in the workspace.
//   join     a wave per row, query and head joins the partial results of its prefix and its own tokens.
//
// Registers instead of LDS: S^T = K Q^T puts the queries on the matrix instruction's columns, so a lane holds one
// query's scores and the softmax needs hardly any exchange; and since a sum over tokens may be taken in any order, row
// 4 g + i of the t-th 16 x 16 score tile is given token 8 g + 4 t + i of the step.  The eight scores of a lane are then
// tokens 8 g .. 8 g + 7, exactly the eight a lane has to hold of P^T as operand of O^T = V^T P^T.  The cache keeps eight
// tokens of a column together (kv_cache.h), so V^T comes from memory in that form too.
//
// An 8-bit cache is widened to bf16 (exactly) and its powers of two are applied to the scores and to P, both in fp32.
// P enters its product as the sum of two bf16 numbers (sixteen bits of each weight): one alone (eight bits) would double the
// error that the output's own rounding leaves, and the second product costs nothing where memory is what the kernel
// waits for.  Everything else between the loads and the output is fp32.
#include "kv_cache.h"
#include "vocab_common.h"
#include "vocab_pass.h"

namespace e3 {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kStep = 32;                       // tokens of a wave's step
constexpr int kAttendWaves = 4;
constexpr int kRun = kStep * kAttendWaves;      // a run is a multiple of this
constexpr float kNoScore = -3.0e38f;            // running maximum before any score
constexpr float kSlack = 8.0f;                  // scores may pass the running maximum by this (2^8) before it moves
constexpr int kTargetTasks = 2048;              // tasks that one long run is cut into, all prefixes and rows together

struct Task { int32_t unit, item, from, to; };  // item: key head + heads * query tile; tokens [from, to)

// What the host fixes of a call; the workspace's parts lie behind one another.
struct AttendShape {
    int32_t R, M;                               // query heads per key head; queries of a row and key head (T * R)
    int32_t row_tile, prefix_tile;              // queries of a task (16 or 32 or 64)
    int32_t row_tiles;                          // tiles of a row
    int32_t row_slot;                           // queries a row's task leaves results of
    int64_t max_row_tasks, max_prefix_tasks;
    int64_t at_tasks, at_row, at_prefix, at_group, at_ml, at_o, bytes;     // byte offsets (at_o: fp32 [rows of D])
};

struct PlanHead { int32_t run, prefix_tasks, row_tasks, pad; };

static int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

static bool attend_shape(int64_t rows, int64_t T, int64_t q_heads, int64_t heads, int64_t D, int64_t groups, AttendShape& s)
{
    s.R = (int32_t)(q_heads / heads);
    const int64_t M = T * s.R;
    if (M > (1 << 16)) return false;
    s.M = (int32_t)M;
    // A row's queries in as few tiles as possible, since each reads the row's keys once more; a prefix has the queries
    // of many rows, at least two tiles' worth for one read.
    const int tiles = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    s.row_tile = 16 * tiles;
    s.prefix_tile = 16 * (tiles < 2 ? 2 : tiles);
    s.row_tiles = (int32_t)((M + s.row_tile - 1) / s.row_tile);
    s.row_slot = (int32_t)(M < s.row_tile ? M : s.row_tile);
    s.max_row_tasks = heads * rows * s.row_tiles + kTargetTasks;
    s.max_prefix_tasks = groups > 0 ? heads * (rows * M / s.prefix_tile + groups) + kTargetTasks : 0;
    const int64_t tasks = s.max_row_tasks + s.max_prefix_tasks;
    const int64_t slots = s.max_row_tasks * s.row_slot + s.max_prefix_tasks * s.prefix_tile;
    if (tasks > (int64_t)1 << 30 || slots > ((int64_t)1 << 31) - 1) return false;
    s.at_tasks = 256;
    s.at_row = up(s.at_tasks + tasks * (int64_t)sizeof(Task), 256);
    s.at_prefix = up(s.at_row + rows * 8, 256);
    s.at_group = up(s.at_prefix + groups * 8, 256);
    s.at_ml = up(s.at_group + rows * 4, 256);
    s.at_o = up(s.at_ml + slots * 8, 256);
    s.bytes = up(s.at_o + slots * D * 4, 256);
    return true;
}

size_t prefix_attention_workspace_bytes(int64_t rows, int64_t T, int64_t q_heads, int64_t heads, int64_t dim, int64_t groups)
{
    AttendShape s;
    return attend_shape(rows, T, q_heads, heads, dim, groups, s) ? (size_t)s.bytes : 0;
}

// ---------------------------------------------------------------- plan
constexpr int kPlanThreads = 1024;

// exclusive prefix sums over the workgroup; the total to everyone
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* lds, int64_t* total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t x = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int i = 0; i < kPlanThreads / 64; ++i) {
        if (i < wave) before += lds[i];
        all += lds[i];
    }
    *total = all;
    return before + x - v;
}

__device__ __forceinline__ int clamp_len(int n, int64_t most) { return n < 0 ? 0 : n > most ? (int)most : n; }
// tokens that a table of `width` pages can name
__device__ __forceinline__ int64_t table_tokens(int width, int page_size)
{
    const int64_t n = (int64_t)width * page_size;
    return n > 0x7FFFFF00 ? 0x7FFFFF00 : n;
}

__global__ __launch_bounds__(kPlanThreads)
void attend_plan_kernel(AttentionArgs a, AttendShape s, int heads, int page_size, char* ws)
{
    __shared__ int64_t lds[kPlanThreads / 64];
    const int64_t row_most = table_tokens(a.row_width, page_size), prefix_most = table_tokens(a.prefix_width, page_size);
    auto row_len = [&](int r) { return clamp_len(a.row_lens[r], row_most); };
    auto prefix_len = [&](int g) { return clamp_len(a.prefix_lens[g], prefix_most); };
    auto first_row = [&](int g) { return clamp_len(a.group_offsets[g], a.rows); };
    auto prefix_tiles = [&](int g) {
        const int n = first_row(g + 1) - first_row(g);
        return n > 0 ? (int)(((int64_t)n * s.M + s.prefix_tile - 1) / s.prefix_tile) : 0;
    };
    Task* tasks = reinterpret_cast<Task*>(ws + s.at_tasks);
    int2* row_plan = reinterpret_cast<int2*>(ws + s.at_row);          // first task, runs
    int2* prefix_plan = reinterpret_cast<int2*>(ws + s.at_prefix);
    int32_t* group_of = reinterpret_cast<int32_t*>(ws + s.at_group);

    int64_t mine = 0, total, carry;
    for (int r = threadIdx.x; r < a.rows; r += kPlanThreads) {
        mine += (int64_t)row_len(r) * s.row_tiles;
        group_of[r] = -1;
    }
    for (int g = threadIdx.x; g < a.groups; g += kPlanThreads) mine += (int64_t)prefix_len(g) * prefix_tiles(g);
    block_scan(mine * heads, lds, &total);
    int64_t run = (total / kTargetTasks + kRun) / kRun * kRun;
    if (run > 0x40000000) run = 0x40000000;

    // group_of[] = -1 above is written by the thread that may be overtaken here: same workgroup, barrier in block_scan
    carry = 0;
    for (int g0 = 0; g0 < a.groups; g0 += kPlanThreads) {
        const int g = g0 + (int)threadIdx.x;
        const int len = g < a.groups ? prefix_len(g) : 0, tiles = g < a.groups ? prefix_tiles(g) : 0;
        const int runs = (int)((len + run - 1) / run);
        int64_t at = block_scan((int64_t)runs * tiles * heads, lds, &total) + carry;
        carry += total;
        if (g < a.groups) {
            // (groups that overlap could exceed the list: those beyond it have no prefix)
            const bool fits = at + (int64_t)runs * tiles * heads <= s.max_prefix_tasks;
            prefix_plan[g] = fits ? int2{(int)at, runs} : int2{0, 0};
            for (int item = 0; fits && item < tiles * heads; ++item)
                for (int c = 0; c < runs; ++c, ++at)
                    tasks[at] = Task{-1 - g, item, (int)(c * run), (int)((c + 1) * run < len ? (c + 1) * run : len)};
            for (int r = first_row(g); r < first_row(g + 1); ++r) group_of[r] = g;
        }
    }
    const int64_t prefix_tasks = carry = carry < s.max_prefix_tasks ? carry : s.max_prefix_tasks;
    for (int r0 = 0; r0 < a.rows; r0 += kPlanThreads) {
        const int r = r0 + (int)threadIdx.x;
        const int len = r < a.rows ? row_len(r) : 0;
        const int runs = (int)((len + run - 1) / run);
        int64_t at = block_scan((int64_t)runs * s.row_tiles * heads, lds, &total) + carry;
        carry += total;
        if (r < a.rows) {
            row_plan[r] = int2{(int)(at - prefix_tasks), runs};
            for (int item = 0; item < s.row_tiles * heads; ++item)
                for (int c = 0; c < runs; ++c, ++at)
                    tasks[at] = Task{r, item, (int)(c * run), (int)((c + 1) * run < len ? (c + 1) * run : len)};
        }
    }
    if (threadIdx.x == 0) {
        PlanHead h;
        h.run = (int)run;
        h.prefix_tasks = (int)prefix_tasks;
        h.row_tasks = (int)(carry - prefix_tasks);
        h.pad = 0;
        *reinterpret_cast<PlanHead*>(ws) = h;
    }
}

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
    __device__ __forceinline__ void load(const CacheView& c, int64_t row, int lane)
    {
        const int m = lane & 15, g = lane >> 4;
        constexpr int kElem = kFp8 ? 1 : 2;
        const char* kp = static_cast<const char*>(c.k) + row * (D * kElem) + (8 * (m >> 2) + (m & 3)) * (D * kElem) + g * 16;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) k[t][i] = stream_load(reinterpret_cast<const u32x4*>(kp + t * 4 * (D * kElem) + i * 64));
        const char* vp = static_cast<const char*>(c.v) + row * (D * kElem) + g * (8 * D * kElem) + m * 16;
#pragma unroll
        for (int i = 0; i < kVLoads; ++i) v[i] = stream_load(reinterpret_cast<const u32x4*>(vp + i * 256));
        if (kFp8) {
            ks = *reinterpret_cast<const u32x2*>(c.k_scale + row + g * 8);
            vs = *reinterpret_cast<const u32x2*>(c.v_scale + row + g * 8);
        }
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
    // whether the lane holds a value (or a scale) that is no finite number
    __device__ __forceinline__ bool unbounded() const
    {
        bool bad = false;
        if (kFp8) {
#pragma unroll
            for (int i = 0; i < kVLoads; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)                              // a byte of 0x7F or 0xFF: + 1 carries into its top bit
                    bad |= (((v[i][j] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) bad |= ((vs[j >> 2] >> (8 * (j & 3))) & 0xFFu) == 0xFFu;
        } else {
#pragma unroll
            for (int i = 0; i < kVLoads; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    bad |= (v[i][j] & 0x7F80u) == 0x7F80u || (v[i][j] & 0x7F800000u) == 0x7F800000u;
        }
        return bad;
    }
    __device__ __forceinline__ float k_factor(int j) const { return __uint_as_float(((ks[j >> 2] >> (8 * (j & 3))) & 0xFFu) << 23); }
    __device__ __forceinline__ float v_factor(int j) const { return __uint_as_float(((vs[j >> 2] >> (8 * (j & 3))) & 0xFFu) << 23); }
};

template <int D, bool kFp8, int kTiles>
struct Attend {
    using Data = StepData<D, kFp8>;
    static constexpr int kBlocks = D / 16, kSteps = D / 32;
    bf16x8 q[kTiles][kSteps];
    f32x4 o[kTiles][kBlocks];
    float m[kTiles], l[kTiles];
    int limit[kTiles];                          // tokens the lane's query sees (of the prefix, of the row)

    // One step.  `at`: its first token; every query sees at least `sure` tokens, none more than `most`.
    __device__ __forceinline__ void step(Data& d, int at, int sure, int most, float c, int lane)
    {
        const int g = lane >> 4;
        const bool tail = at + kStep > sure;                              // uniform
        if (tail) d.clear_from(most - at - 8 * g);
        f32x4 s[kTiles][2];
#pragma unroll
        for (int n = 0; n < kTiles; ++n) s[n][0] = s[n][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const bf16x8 key = d.key(t, i);
#pragma unroll
                for (int n = 0; n < kTiles; ++n) s[n][t] = mfma(key, q[n][i], s[n][t]);
            }
        bf16x8 p[kTiles], rest[kTiles];
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = s[n][j >> 2][j & 3] * (kFp8 ? c * d.k_factor(j) : c);
                if (tail) x[j] = at + 8 * g + j < limit[n] ? x[j] : -INFINITY;
            }
            float top = fmax3(fmax3(x[0], x[1], x[2]), fmax3(x[3], x[4], x[5]), fmaxf(x[6], x[7]));
            if (__any(top > m[n] + kSlack)) {
                // the queries' maxima over the four lanes that hold their scores
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float to = fmaxf(m[n], top);
                const float f = __builtin_amdgcn_exp2f(m[n] - to);
                m[n] = to;
                l[n] *= f;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) o[n][b] *= f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float e = __builtin_amdgcn_exp2f(x[j] - m[n]);
                l[n] += e;
                const float w = kFp8 ? e * d.v_factor(j) : e;
                p[n][j] = (__bf16)w;
                rest[n][j] = (__bf16)(w - (float)p[n][j]);
            }
        }
        // Tokens that some queries see and others do not: a weight of zero keeps them out, unless the value is no
        // number.  Then the queries take turns, each with the others' tokens cleared.
        if (__builtin_expect(tail && sure < most && __any(d.unbounded()), 0)) {
            for (int have = sure; have <= most; ++have) {
                Data only = d;
                only.clear_from(have - at - 8 * g);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int n = 0; n < kTiles; ++n) {
                        const f32x4 r = mfma(only.value(b), rest[n], mfma(only.value(b), p[n], o[n][b]));
                        if (limit[n] == have) o[n][b] = r;
                    }
            }
            return;
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const bf16x8 value = d.value(b);
#pragma unroll
            for (int n = 0; n < kTiles; ++n) o[n][b] = mfma(value, rest[n], mfma(value, p[n], o[n][b]));
        }
    }

    // kPrefix: task.unit is -1 - group; otherwise a row.  `head`, `tile` of the task.
    template <bool kPrefix>
    __device__ __forceinline__ void run(const CacheView& c, const AttentionArgs& a, const AttendShape& sh, const Task& task,
                                        float* lds, float2* ml_out, float* o_out, int slot_rows)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int col = lane & 15, g = lane >> 4;
        const int unit = kPrefix ? -1 - task.unit : task.unit;
        const int head = task.item % c.heads, tile = task.item / c.heads;
        int row0 = unit, queries = sh.M, len, sure;
        const int32_t* pages;
        if (kPrefix) {
            row0 = clamp_len(a.group_offsets[unit], a.rows);
            queries *= clamp_len(a.group_offsets[unit + 1], a.rows) - row0;
            pages = a.prefix_pages + (int64_t)unit * a.prefix_width;
            len = sure = clamp_len(a.prefix_lens[unit], table_tokens(a.prefix_width, c.page_size));
        } else {
            pages = a.row_pages + (int64_t)unit * a.row_width;
            len = clamp_len(a.row_lens[unit], table_tokens(a.row_width, c.page_size));
            sure = len - (a.T - 1) > 0 ? len - (a.T - 1) : 0;
        }
        // queries: column n of tile i is query first + 16 i + n
        const int first = tile * (16 * kTiles);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
            const int qi = first + 16 * i + col;
            const bool is = qi < queries;
            const int row = row0 + (is ? qi / sh.M : 0), in_row = is ? qi % sh.M : 0;
            const int t = in_row / sh.R, h = head * sh.R + in_row % sh.R;
            const uint16_t* qp = a.q + row * a.q_row_stride + t * a.q_token_stride + h * a.q_head_stride;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                u32x4 w = *reinterpret_cast<const u32x4*>(qp + Data::key_column(s, g));
                if (!is) w = u32x4{0, 0, 0, 0};
                q[i][s] = __builtin_bit_cast(bf16x8, w);
            }
            const int own = len - (a.T - 1 - t);
            limit[i] = kPrefix ? len : own > 0 ? own : 0;
            m[i] = kNoScore;
            l[i] = 0.0f;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) o[i][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const float scale = a.scale * kLog2eF;

        // tokens [from, to) of the run; the wave's steps are 4 apart.  A page that the cache does not have is not seen.
        const int to = task.to;
        auto page_at = [&](int at) { return at < to ? pages[at >> c.page_shift] : -1; };
        auto row_of = [&](int page, int at) {
            const int64_t p = (uint32_t)page < (uint64_t)c.num_pages ? page : 0;
            return (p * c.heads + head) * c.page_size + (at & (c.page_size - 1));
        };
        int at = task.from + wave * kStep;
        if (at < to) {
            Data cur, next;
            int page = page_at(at), page_next = page_at(at + kRun);
            cur.load(c, row_of(page, at), lane);
            for (; at < to; at += kRun) {
                const int page_after = page_at(at + 2 * kRun);
                if (at + kRun < to) next.load(c, row_of(page_next, at + kRun), lane);
                if ((uint32_t)page < (uint64_t)c.num_pages) step(cur, at, sure, len, scale, lane);
                cur = next;
                page = page_next;
                page_next = page_after;
            }
        }

        // Join the four waves.  l is spread over the four lanes of a query.
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
            l[i] += __shfl_xor(l[i], 16);
            l[i] += __shfl_xor(l[i], 32);
        }
        constexpr int kMl = kAttendWaves * 16 * kTiles;                    // lds: (m, l) of all waves, then O of two waves
        float2* ml = reinterpret_cast<float2*>(lds);
        f32x4* part = reinterpret_cast<f32x4*>(lds + 2 * kMl);             // [2][kTiles * kBlocks][64]
        __syncthreads();                                                   // the last task's results are read
        if (g == 0) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i) ml[wave * 16 * kTiles + 16 * i + col] = float2{m[i], l[i]};
        }
        __syncthreads();
        float all_m[kTiles], all_l[kTiles];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
            float2 w[kAttendWaves];
            all_m[i] = kNoScore;
#pragma unroll
            for (int k = 0; k < kAttendWaves; ++k) {
                w[k] = ml[k * 16 * kTiles + 16 * i + col];
                all_m[i] = fmaxf(all_m[i], w[k].x);
            }
            all_l[i] = 0.0f;
#pragma unroll
            for (int k = 0; k < kAttendWaves; ++k) all_l[i] = fmaf(w[k].y, __builtin_amdgcn_exp2f(w[k].x - all_m[i]), all_l[i]);
            const float f = __builtin_amdgcn_exp2f(m[i] - all_m[i]);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) o[i][b] *= f;
        }
        auto give = [&](int to_slot) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) part[(to_slot * kTiles * kBlocks + i * kBlocks + b) * 64 + lane] = o[i][b];
        };
        auto take = [&](int from_slot) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) o[i][b] += part[(from_slot * kTiles * kBlocks + i * kBlocks + b) * 64 + lane];
        };
        if (wave >= 2) give(wave - 2);
        __syncthreads();
        if (wave < 2) take(wave);
        __syncthreads();
        if (wave == 1) give(0);
        __syncthreads();
        if (wave == 0) {
            take(0);
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                const int slot = 16 * i + col;
                if (first + slot >= queries || slot >= slot_rows) continue;
                if (g == 0) ml_out[slot] = float2{all_m[i], all_l[i]};
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o_out[(int64_t)slot * D + Data::column(b, 4 * g + k)] = o[i][b][k];
            }
        }
    }
};

template <int D, int kTiles>
constexpr int attend_lds_floats() { return 2 * kAttendWaves * 16 * kTiles + 2 * kTiles * (D / 16) * 64 * 4; }

template <int D, bool kFp8, int kRowTiles, int kPrefixTiles>
__global__ __launch_bounds__(64 * kAttendWaves)
void attend_kernel(CacheView c, AttentionArgs a, AttendShape s, char* ws)
{
    __shared__ __align__(16) float lds[attend_lds_floats<D, kPrefixTiles>()];
    const PlanHead head = *reinterpret_cast<const PlanHead*>(ws);
    const Task* tasks = reinterpret_cast<const Task*>(ws + s.at_tasks);
    float2* ml = reinterpret_cast<float2*>(ws + s.at_ml);
    float* o = reinterpret_cast<float*>(ws + s.at_o);
    for (int i = blockIdx.x; i < head.prefix_tasks + head.row_tasks; i += gridDim.x) {
        const Task task = tasks[i];
        if (i < head.prefix_tasks) {
            const int64_t slot = s.max_row_tasks * s.row_slot + (int64_t)i * s.prefix_tile;
            Attend<D, kFp8, kPrefixTiles> x;
            x.template run<true>(c, a, s, task, lds, ml + slot, o + slot * D, s.prefix_tile);
        } else {
            const int64_t slot = (int64_t)(i - head.prefix_tasks) * s.row_slot;
            Attend<D, kFp8, kRowTiles> x;
            x.template run<false>(c, a, s, task, lds, ml + slot, o + slot * D, s.row_slot);
        }
    }
}

// ---------------------------------------------------------------- join
// A wave per (row, key head, query): the partial results of the prefix's runs, then those of the row's.
template <int D>
__global__ __launch_bounds__(256)
void attend_join_kernel(AttentionArgs a, AttendShape s, int heads, const char* ws)
{
    constexpr int kCols = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= (int64_t)a.rows * heads * s.M) return;
    const int in_row = (int)(at % s.M), head = (int)(at / s.M % heads), row = (int)(at / s.M / heads);
    const int2* row_plan = reinterpret_cast<const int2*>(ws + s.at_row);
    const int2* prefix_plan = reinterpret_cast<const int2*>(ws + s.at_prefix);
    const int group = reinterpret_cast<const int32_t*>(ws + s.at_group)[row];
    const float2* ml = reinterpret_cast<const float2*>(ws + s.at_ml);
    const float* o = reinterpret_cast<const float*>(ws + s.at_o);

    float m = kNoScore, l = 0.0f, acc[kCols] = {};
    // results at slots first + i * apart, i < n
    auto join = [&](int64_t first, int64_t apart, int n) {
        for (int i0 = 0; i0 < n; i0 += 64) {
            const int many = n - i0 < 64 ? n - i0 : 64;
            float2 mine = lane < many ? ml[first + (i0 + lane) * apart] : float2{kNoScore, 0.0f};
            const float top = wave_max(mine.x);
            const float to = fmaxf(m, top);
            const float f = __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int j = 0; j < kCols; ++j) acc[j] *= f;
            const float w = __builtin_amdgcn_exp2f(mine.x - to);           // 0 beyond `many` once any score is there
            l += (float)wave_sum((double)(mine.y * w));
            for (int i = 0; i < many; ++i) {
                const float wi = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), i));
                const float* p = o + (first + (i0 + i) * apart) * D + lane * kCols;
#pragma unroll
                for (int j = 0; j < kCols; ++j) acc[j] = fmaf(wi, p[j], acc[j]);
            }
        }
    };
    if (group >= 0) {
        const int2 plan = prefix_plan[group];
        const int qi = (row - clamp_len(a.group_offsets[group], a.rows)) * s.M + in_row;
        const int64_t item = (int64_t)(qi / s.prefix_tile) * heads + head;
        join(s.max_row_tasks * s.row_slot + (plan.x + item * plan.y) * s.prefix_tile + qi % s.prefix_tile, s.prefix_tile, plan.y);
    }
    {
        const int2 plan = row_plan[row];
        const int64_t item = (int64_t)(in_row / s.row_tile) * heads + head;
        join((plan.x + item * plan.y) * s.row_slot + in_row % s.row_tile, s.row_slot, plan.y);
    }
    const int t = in_row / s.R, h = head * s.R + in_row % s.R;
    const int64_t where = ((int64_t)row * a.T + t) * a.q_heads + h;
    const bool none = l == 0.0f && m == kNoScore;                          // no key at all
    const float inv = none ? 0.0f : 1.0f / l;
    uint32_t packed = 0;
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
        const __bf16 b = (__bf16)(none ? 0.0f : acc[j] * inv);
        packed |= (uint32_t)__builtin_bit_cast(uint16_t, b) << (16 * j);
    }
    if (kCols == 2) reinterpret_cast<uint32_t*>(a.out + where * D)[lane] = packed;
    else a.out[where * D + lane] = (uint16_t)packed;
    if (a.lse && lane == 0) a.lse[where] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * (float)kLn2;
}

template <int D, bool kFp8, int kRowTiles, int kPrefixTiles>
static hipError_t launch_attend(const CacheView& c, const AttentionArgs& a, const AttendShape& s, char* ws, hipStream_t stream)
{
    attend_plan_kernel<<<1, kPlanThreads, 0, stream>>>(a, s, c.heads, c.page_size, ws);
    const int64_t most = s.max_row_tasks + s.max_prefix_tasks;
    const int64_t groups = (int64_t)compute_units() * 2;
    attend_kernel<D, kFp8, kRowTiles, kPrefixTiles><<<(uint32_t)(most < groups ? most : groups), 64 * kAttendWaves, 0, stream>>>(c, a, s, ws);
    const int64_t waves = (int64_t)a.rows * c.heads * s.M;
    attend_join_kernel<D><<<(uint32_t)((waves + 3) / 4), 256, 0, stream>>>(a, s, c.heads, ws);
    return hipGetLastError();
}

hipError_t launch_prefix_attention(const CacheView& c, const AttentionArgs& a, void* workspace, hipStream_t stream)
{
    AttendShape s;
    if (!attend_shape(a.rows, a.T, a.q_heads, c.heads, c.dim, a.groups, s)) return hipErrorInvalidValue;
    char* ws = static_cast<char*>(workspace);
    auto by_tiles = [&](auto d, auto fp8) {
        constexpr int D = decltype(d)::value;
        constexpr bool kFp8 = decltype(fp8)::value;
        if (s.row_tile == 16) return launch_attend<D, kFp8, 1, 2>(c, a, s, ws, stream);
        if (s.row_tile == 32) return launch_attend<D, kFp8, 2, 2>(c, a, s, ws, stream);
        return launch_attend<D, kFp8, 4, 4>(c, a, s, ws, stream);
    };
    auto by_type = [&](auto d) { return c.fp8 ? by_tiles(d, std::true_type{}) : by_tiles(d, std::false_type{}); };
    return c.dim == 128 ? by_type(std::integral_constant<int, 128>{}) : by_type(std::integral_constant<int, 64>{});
}

}  // namespace e3
