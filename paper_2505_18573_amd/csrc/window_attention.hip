// Attention over the paged cache with a sliding window and first tokens that stay visible.
//
//   row r brings n_r queries, the last n_r of its len_r tokens; the one at position p sees
//   { j <= p : j > p - window or j < sinks },   s_j = scale q . k_j,   out = sum e^{s_j - m} v_j / l,   lse = m + ln l.
//
// The softmax's maximum and sum are running ones, and partial results (m, l, O) over disjoint sets of keys join exactly, so the
// work may be cut anywhere.  Three launches, two for few rows:
//   plan     one workgroup makes the list of work: lengths and numbers of queries are device memory.  A row's queries of one key
//            head (tokens x query heads) are cut into tiles; a tile and a key head are an item, measured in steps of tokens that
//            any of its queries sees (pages that none sees are never touched) and a little for the item itself.  For few rows
//            every workgroup of the next launch does that for itself.
//   attend   Items of at most 32 queries are a wave's work: a new token's or a few drafted ones', bound by reading the keys, which go from
//            memory straight into operand registers.  Larger ones, tiles of 128 queries of prompts, are a workgroup's: bound by
//            the matrix instructions, the keys pass through LDS once for four waves of 32 queries.  Either kind lies on a line, cut into as
//            many equal stretches as there are workers, whichever items they fall into.  An item that lies in one
//            stretch is written out; of one that is cut every worker leaves its part in the workspace.
//   join     the parts of cut items.
//
// Weights times values.  For few queries the weights enter as three bf16 numbers, all 24 bits of an fp32 weight, as memory is what
// is waited for.  For tiles of prompts they enter as two, 16 bits and more: a weight is off by 2^-17 of itself at most, far below the output's own
// rounding (2^-9 at best) unless an output's terms cancel to less than a hundredth, while one number alone (2^-9)
// would add as much error as the output's rounding (prompts 392 us for 465); the third product would cost a quarter more time.
//
// Measured, with the plan where there is one and the join: 512 rows of one query, 28 heads over 4 of 128, 8 bits, window 4096 of up to 7000
// tokens 303 us, 5.1 TB/s: memory.  Prompts of 1000 to 4001 tokens, the same heads, 16 bits, window 1024: 434 to 467 us from card to card, 234
// GFLOP of scores and values, 350 with the second bf16 number of the weights, so 0.8 PFLOP/s (a large product of the library: 1.26):
// the matrix instructions of the two waves on a SIMD are half of the time, the vector instructions the other half, at the 1.6 to 1.8
// GHz that were measured under this load.  A mixed batch of 33 rows of 1 to 300 queries, 12 heads over 2 of 64: 33.9 us; a workgroup has
// 1.3 items and 7 steps, 5 us pass before the first item, 1.5 in a step, 3.5 into and out of an item, 8 in the join.  One row: 10.3
// us, two launches.  (The figures at the constants below compare builds that differ in nothing else, on these four.)
#include "attention_step.h"
#include "stretch.h"
#include "vocab_common.h"
#include "vocab_pass.h"
#include "window_attention.h"

namespace e3 {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4;                       // of a workgroup
constexpr int kFewQueries = 32;                 // an item of so many is a wave's
constexpr int kTile = 128;                      // queries of a workgroup's item
constexpr int kBlock = 64;                      // tokens of a workgroup's step
// What an item costs besides its steps, in steps of either kind (prompts 465 us; with 1: 496, with 4: 456; 512 rows 303.2, 307.5, 302.9;
// mixed 35.5, 36.5, 36.6).
constexpr int kCost = 2;
constexpr int kPerUnit = 2;                     // workgroups per compute unit, as registers and LDS allow
constexpr float kBlockCost = 1.0f;              // a workgroup's step against four steps of its waves (mixed 35.5 us; 0.7: 37.4, 1.4: 35.6)

enum { kOfGroups = 0, kOfWaves = 1 };           // the two lines

// A tile of a row's queries, all key heads: its place on its line is in steps.
struct Work {
    int64_t first;
    int32_t row, tile, offset, n, len, cost;    // offset, n: the row's queries; cost: steps of one key head, kCost among them
};
struct Totals {
    int64_t steps[2];
    int32_t count[2];
};
// The item that a worker's stretch begins inside of, if the item's first part is the worker's before: parts worker - 1 .. last are joined.
struct Cut {
    int32_t row, tile, offset, n, len, head, last, unused;         // row: -1 where there is none
};

struct WindowShape {
    int32_t R;                                  // query heads per key head
    int64_t most[2];                            // records of either line
    int32_t workgroups, workers[2];             // workers: at most
    int64_t steps, most_cost;                   // of either line, of an item at most
    int64_t at_list[2], at_cuts, at_ml, at_o[2], bytes;
};

static int64_t up(int64_t x) { return (x + 255) / 256 * 256; }

// `visible`: tokens that any query can see at most, for a workspace that serves every call as many as there are.
static bool window_shape(int64_t rows, int64_t tokens, int64_t q_heads, int64_t heads, int64_t D, int64_t visible, WindowShape& s)
{
    s.R = (int32_t)(q_heads / heads);
    if (rows * heads >= (1 << 24) || tokens * q_heads > 0x7FFFFFFF) return false;
    const int64_t groups = compute_units() * kPerUnit;
    const int64_t queries = tokens * s.R;
    s.most[kOfGroups] = queries > kFewQueries ? queries / kTile + rows : 0;
    s.most[kOfWaves] = rows;
    // No more workgroups than steps, half as many where there may be tiles, whose workgroups are four workers each of the other line too: a
    // small call's launches are small (3 rows of 2 to 8 queries, 8 heads of 128: 14.8 us in kernels, with all workgroups 19.7).
    s.most_cost = visible / kStep + 4 + kCost;
    s.steps = (queries / kTile + rows) * heads * s.most_cost;
    const int64_t enough = s.most[kOfGroups] == 0 ? s.steps : s.steps / 2 + 2;
    s.workgroups = (int32_t)(enough < groups ? enough : groups);
    s.workers[kOfGroups] = s.most[kOfGroups] > 0 ? s.workgroups : 0;
    s.workers[kOfWaves] = s.workgroups * kWaves;
    int64_t at = up(sizeof(Totals));
    for (int k = 0; k < 2; ++k) { s.at_list[k] = at; at = up(at + s.most[k] * (int64_t)sizeof(Work)); }
    s.at_cuts = at;
    at = up(at + (s.workers[0] + s.workers[1]) * (int64_t)sizeof(Cut));
    // partial results: two places for each worker (what its stretch begins inside of, what it ends inside of)
    s.at_ml = at;
    at = up(at + (s.workers[0] * (int64_t)kTile + s.workers[1] * (int64_t)kFewQueries) * 2 * (int64_t)sizeof(float2));
    s.at_o[kOfGroups] = at;
    at = up(at + s.workers[0] * (int64_t)kTile * 2 * D * 4);
    s.at_o[kOfWaves] = at;
    s.bytes = up(at + s.workers[1] * (int64_t)kFewQueries * 2 * D * 4);
    return true;
}

size_t window_attention_workspace_bytes(int64_t rows, int64_t tokens, int64_t q_heads, int64_t heads, int64_t dim)
{
    WindowShape s;
    return window_shape(rows, tokens, q_heads, heads, dim, (int64_t)1 << 31, s) ? (size_t)s.bytes : 0;
}

// ---------------------------------------------------------------- which tokens
__host__ __device__ __forceinline__ int tiles_of(int64_t queries) { return queries <= kFewQueries ? 1 : (int)((queries + kTile - 1) / kTile); }

// The tokens of a tile's item, in steps of `apart` tokens: first those of the always visible tokens that lie before the
// window's, then the window's.
struct Band {
    int p0, p1;                                 // positions of the tile's first and last query
    int first_steps, skip;                      // step k is at token (k < first_steps ? k : k + skip) * apart
    int steps;
    __device__ __forceinline__ int at(int k, int apart) const { return (k < first_steps ? k : k + skip) * apart; }
};
// (positions, queries of a row and steps of tokens stay below 2^31)
__device__ __forceinline__ Band band_of(int R, int tile, int n, int len, int window, int sinks, int apart)
{
    const int shift = apart == kStep ? 5 : 6;
    const uint32_t queries = (uint32_t)n * (uint32_t)R;
    const uint32_t q0 = (uint32_t)tile * kTile, q1 = queries <= kFewQueries || q0 + kTile > queries ? queries : q0 + kTile;
    Band b;
    b.p0 = len - n + (int)(q0 / (uint32_t)R);
    b.p1 = len - n + (int)((q1 - 1) / (uint32_t)R);
    const int hi = b.p1 + 1;                                                   // none sees a token from here on
    if (hi <= 0) { b.first_steps = b.skip = b.steps = 0; return b; }
    const int lo = (b.p0 < 0 ? 0 : b.p0) >= window ? b.p0 - window + 1 : 0;    // none sees one before it, but the first ones
    const int lo_step = lo >> shift, kept = sinks < hi ? sinks : hi;
    const int kept_steps = (kept + apart - 1) >> shift;
    b.first_steps = kept_steps < lo_step ? kept_steps : lo_step;
    b.skip = lo_step - b.first_steps;
    b.steps = ((hi + apart - 1) >> shift) - b.skip;
    return b;
}

// ---------------------------------------------------------------- plan
// Places for tiles: a row's lie from place_of_row(row) on, as many as it can have.
__device__ __forceinline__ int64_t place_of_row(int offset, int R, int row) { return (int64_t)offset * R / kTile + row; }

// f(line, record, place) for every tile among places [begin, end); offset(row), len(row): the row's first query and tokens.
template <typename Offset, typename Len, typename F>
__device__ __forceinline__ void tiles_in(const WindowArgs& a, int R, int64_t begin, int64_t end, Offset offset, Len len_of, F f)
{
    if (begin >= end) return;
    int low = 0, high = a.rows;                                                // the last row whose places begin at or before `begin`
    while (high - low > 1) {
        const int mid = (low + high) / 2;
        if (place_of_row(offset(mid), R, mid) <= begin) low = mid;
        else high = mid;
    }
    for (int r = low; r < a.rows; ++r) {
        const int off = offset(r), n = offset(r + 1) - off;
        const int64_t k = place_of_row(off, R, r);
        if (k >= end) break;
        if (n <= 0) continue;
        const int64_t queries = (int64_t)n * R;
        const int line = queries <= kFewQueries ? kOfWaves : kOfGroups;
        const int64_t last = k + tiles_of(queries);
        const int len = len_of(r);
        for (int64_t u = k > begin ? k : begin; u < last && u < end; ++u) {
            Work w;
            w.first = 0; w.row = r; w.tile = (int)(u - k); w.offset = off; w.n = n; w.len = len;
            w.cost = kCost + band_of(R, w.tile, n, len, a.window, a.sinks, line == kOfWaves ? kStep : kBlock).steps;
            f(line, w, u);
        }
    }
}

// The sum over the lanes up to this one: rows of sixteen, then the rows before.
constexpr int kDppUp = 0x110;                   // + n: from n lanes before
template <int kCtrl, int kRows>
__device__ __forceinline__ int from_before(int x) { return dpp_i<kCtrl, kRows>(0, x); }
template <int kCtrl, int kRows>
__device__ __forceinline__ int64_t from_before(int64_t x)
{
    const uint32_t lo = (uint32_t)dpp_i<kCtrl, kRows>(0, (int)(uint32_t)x), hi = (uint32_t)dpp_i<kCtrl, kRows>(0, (int)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}
template <typename T>
__device__ __forceinline__ T sum_up_to(T x)
{
    x += from_before<kDppUp + 1, 0xF>(x);                                           // 1, 2, 4, 8 lanes before, in the row
    x += from_before<kDppUp + 2, 0xF>(x);
    x += from_before<kDppUp + 4, 0xF>(x);
    x += from_before<kDppUp + 8, 0xF>(x);
    x += from_before<kDppBcast15, 0xA>(x);                                           // the last lane of the row before, for odd rows
    return x + from_before<kDppBcast31, 0xC>(x);                                     // lane 31, for the upper half
}

// Sums over the threads before this one, and over all: steps of both lines; tiles, the waves' in the upper half.
template <int kOf>
__device__ __forceinline__ void scan(const int64_t own[3], int64_t before[3], int64_t all[3], int64_t (*lds)[3])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        before[k] = sum_up_to(own[k]);
        if (lane == 63) lds[wave][k] = before[k];
        before[k] -= own[k];
        all[k] = 0;
    }
    __syncthreads();
    for (int i = 0; i < kOf; ++i)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            if (i < wave) before[k] += lds[i][k];
            all[k] += lds[i][k];
        }
}

// The plan of a large batch, a launch of one workgroup.
constexpr int kPlanWaves = 16, kPlanLanes = 64 * kPlanWaves, kPlanRows = 8192;

__global__ __launch_bounds__(kPlanLanes)
void window_plan_kernel(WindowArgs a, WindowShape s, int heads, int page_size, char* ws)
{
    __shared__ int offsets_lds[kPlanRows + 1];
    __shared__ int64_t sums[kPlanWaves][3];
    const bool in_lds = a.rows <= kPlanRows;
    if (in_lds) {
        for (int i = threadIdx.x; i <= a.rows; i += kPlanLanes) offsets_lds[i] = clamp_len(a.offsets[i], a.tokens);
        __syncthreads();
    }
    auto offset = [&](int r) { return in_lds ? offsets_lds[r] : clamp_len(a.offsets[r], a.tokens); };
    const int64_t visible = table_tokens(a.row_width, page_size);
    auto len = [&](int r) { return clamp_len(a.row_lens[r], visible); };
    const int64_t places = (int64_t)a.tokens * s.R / kTile + a.rows;
    const int64_t share = (places + kPlanLanes - 1) / kPlanLanes;
    const int64_t begin = threadIdx.x * share, end = begin + share < places ? begin + share : places;
    int64_t own[3] = {0, 0, 0}, before[3], all[3];
    tiles_in(a, s.R, begin, end, offset, len, [&](int line, const Work& w, int64_t) {
        own[0] += line == 0 ? (int64_t)w.cost * heads : 0;
        own[1] += line == 1 ? (int64_t)w.cost * heads : 0;
        own[2] += line == 1 ? 1ll << 32 : 1;
    });
    scan<kPlanWaves>(own, before, all, sums);
    int64_t index[2] = {before[2] & 0xFFFFFFFF, before[2] >> 32};
    tiles_in(a, s.R, begin, end, offset, len, [&](int line, Work w, int64_t) {
        w.first = line == 0 ? before[0] : before[1];
        const int64_t i = line == 0 ? index[0]++ : index[1]++;
        if (line == 0) before[0] += (int64_t)w.cost * heads;
        else before[1] += (int64_t)w.cost * heads;
        if (i < s.most[line]) reinterpret_cast<Work*>(ws + s.at_list[line])[i] = w;
    });
    if (threadIdx.x == 0) {
        Totals t;
        // (offsets that fall, against the contract, could give more tiles than there is room for: nothing is done then)
        const bool fits = (all[2] & 0xFFFFFFFF) <= s.most[0] && (all[2] >> 32) <= s.most[1];
        t.steps[0] = fits ? all[0] : 0;
        t.steps[1] = fits ? all[1] : 0;
        t.count[0] = fits ? (int)(all[2] & 0xFFFFFFFF) : 0;
        t.count[1] = fits ? (int)(all[2] >> 32) : 0;
        *reinterpret_cast<Totals*>(ws) = t;
    }
}

// A batch of few rows, tiles and steps is planned by every workgroup of the attend launch for itself, in LDS and 32 bits: a launch less.
// (Mixed 35.5 us, with a launch for the plan 42.0; 512 rows 303.2, 309.0.)  The list has an entry for every place; one without
// a tile of a line has the beginning of the line's next one.
constexpr int kOwnPlaces = 640;                 // what fits beside the keys of two workgroups
constexpr int kOwnSteps = 1 << 20;              // of all; what may have more takes long enough for another launch not to count
constexpr int kOwnCost = 1 << 16;               // of an item
struct OwnPlan {
    int offsets[kOwnPlaces + 1], lens[kOwnPlaces];
    int first[2][kOwnPlaces];
    uint32_t row_tile[kOwnPlaces];
    uint16_t cost[kOwnPlaces];
    int sums[kWaves][2];
};
__device__ __forceinline__ Totals plan_own(const WindowArgs& a, const WindowShape& s, int heads, int page_size, OwnPlan& p)
{
    constexpr int kThreads = 64 * kWaves;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t visible = table_tokens(a.row_width, page_size);
    for (int i = threadIdx.x; i <= a.rows; i += kThreads) {
        p.offsets[i] = clamp_len(a.offsets[i], a.tokens);
        if (i < a.rows) p.lens[i] = clamp_len(a.row_lens[i], visible);
    }
    __syncthreads();
    const int places = (int)((int64_t)a.tokens * s.R / kTile) + a.rows;        // at most kOwnPlaces
    const int share = (places + kThreads - 1) / kThreads;
    const int begin = (int)threadIdx.x * share, end = begin + share < places ? begin + share : places;
    for (int u = begin; u < end; ++u) { p.first[0][u] = 0; p.first[1][u] = 0; }
    tiles_in(a, s.R, begin, end, [&](int r) { return p.offsets[r]; }, [&](int r) { return p.lens[r]; }, [&](int line, const Work& w, int64_t u) {
        p.first[line][u] = w.cost * heads;
        p.first[1 - line][u] = 0;
        p.row_tile[u] = (uint32_t)w.row << 16 | (uint32_t)w.tile;
        p.cost[u] = (uint16_t)w.cost;
    });
    int own[2] = {0, 0}, before[2];
    for (int u = begin; u < end; ++u) { own[0] += p.first[0][u]; own[1] += p.first[1][u]; }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        before[k] = sum_up_to(own[k]);
        if (lane == 63) p.sums[wave][k] = before[k];
        before[k] -= own[k];
    }
    __syncthreads();
    Totals t{{0, 0}, {places, places}};
#pragma unroll
    for (int i = 0; i < kWaves; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (i < wave) before[k] += p.sums[i][k];
            t.steps[k] += p.sums[i][k];
        }
    for (int u = begin; u < end; ++u)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int cost = p.first[k][u];
            p.first[k][u] = before[k];
            before[k] += cost;
        }
    __syncthreads();
    return t;
}

// A line's records, in the workspace or in LDS; next(i, step): the record behind record i, which begins at that step.
struct InWorkspace {
    using Step = int64_t;
    const Work* list;
    int count;
    __device__ __forceinline__ int64_t first(int i) const { return list[i].first; }
    __device__ __forceinline__ Work get(int i) const { return list[i < count ? i : count - 1]; }
    __device__ __forceinline__ int next(int i, Step) const { return i + 1; }
};
template <typename List> __device__ __forceinline__ int find_work(const List& list, int count, typename List::Step step);
template <int kLine>
struct InLds {
    using Step = int32_t;
    const OwnPlan& p;
    int count;
    __device__ __forceinline__ Step first(int i) const { return p.first[kLine][i]; }
    __device__ __forceinline__ Work get(int i) const
    {
        Work w;
        w.first = p.first[kLine][i];
        const uint32_t x = p.row_tile[i];
        w.row = uniform((int)(x >> 16)); w.tile = uniform((int)(x & 0xFFFFu));
        w.offset = uniform(p.offsets[w.row]); w.n = uniform(p.offsets[w.row + 1]) - w.offset; w.len = uniform(p.lens[w.row]);
        w.cost = p.cost[i];
        return w;
    }
    __device__ __forceinline__ int next(int, Step step) const { return find_work(*this, count, step); }
};

// How workgroups and steps are divided.
struct Division {
    int64_t steps[2];
    int groups;                                 // workgroups of the line of workgroups
    int parts[2];                               // stretches
};
// The stretches of a line: the first `longer` of them have each + 1 steps, the others `each`.
template <typename Step>
struct Stretches {
    Step each;
    int longer;
    __device__ __forceinline__ Stretches(Step steps, int parts)
    {
        each = sizeof(Step) == 4 ? (Step)((uint32_t)steps / (uint32_t)parts) : (Step)divide(steps, parts);
        longer = (int)(steps - each * parts);
    }
    __device__ __forceinline__ Step begin(int w) const { return w * each + (w < longer ? w : longer); }
    __device__ __forceinline__ int of(Step step) const
    {
        const Step first = longer * (each + 1), x = step < first ? step : step - first, by = step < first ? each + 1 : each;
        return (step < first ? 0 : longer) + (sizeof(Step) == 4 ? (int)((uint32_t)x / (uint32_t)by) : (int)divide(x, by));
    }
};
__device__ __forceinline__ Division divide_work(const Totals& t, int workgroups)
{
    Division d;
    d.steps[0] = uniform(t.steps[0]);
    d.steps[1] = uniform(t.steps[1]);
    const float of_groups = (float)d.steps[0] * kBlockCost, of_waves = (float)d.steps[1] * (1.0f / kWaves);
    int share = (int)(of_groups / (of_groups + of_waves) * (float)workgroups + 0.5f);
    if (d.steps[1] > 0 && share > workgroups - 1) share = workgroups - 1;
    if (d.steps[0] > 0 && share < 1) share = 1;
    d.groups = d.steps[0] == 0 ? 0 : uniform(share);
    const int64_t most[2] = {d.groups, (int64_t)(workgroups - d.groups) * kWaves};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        // a stretch has one step at least, two, four (one row 10.7 us; four: 12.8)
        const int shift = d.steps[k] < 512 ? 0 : d.steps[k] < 1024 ? 1 : 2;
        const int64_t enough = (d.steps[k] + (1 << shift) - 1) >> shift;
        d.parts[k] = (int)(enough < most[k] ? enough : most[k]);
    }
    return d;
}

// The last record that begins at or before a step: every lane looks at a 64th of what is left.
template <typename List>
__device__ __forceinline__ int find_work(const List& list, int count, typename List::Step step)
{
    const int lane = threadIdx.x & 63;
    int first = 0, left = count;
    while (left > 1) {
        const int apart = (left + 63) / 64, at = lane * apart;
        const int n = (int)__popcll(__ballot(at < left && list.first(first + (at < left ? at : 0)) <= step));
        const int k = n > 0 ? n - 1 : 0;
        first += k * apart;
        left = left - k * apart < apart ? left - k * apart : apart;
    }
    return uniform(first);
}
__device__ __forceinline__ Work uniform(const Work& w)
{
    return Work{uniform(w.first), uniform(w.row), uniform(w.tile), uniform(w.offset), uniform(w.n), uniform(w.len), uniform(w.cost)};
}

// ---------------------------------------------------------------- attend
struct Piece1 {                                 // of an item: real steps [from, to)
    int head, from, to;
    bool whole;
};
// A query of a tile: where it lies and what it sees.
struct Query {
    int token, head;                            // of q and out
    int lo, hi;                                 // tokens lo .. hi - 1, and the first ones
    bool is;
};
// (a row's queries of a key head stay below 2^31: divided in 32 bits, a 64-bit division takes a hundred instructions more)
__device__ __forceinline__ Query query_of(const WindowArgs& a, int R, const Work& w, int head, uint32_t index)
{
    Query q;
    q.is = index < (uint32_t)w.n * (uint32_t)R;
    const int t = q.is ? (int)(index / (uint32_t)R) : 0, h = q.is ? (int)(index - (uint32_t)t * (uint32_t)R) : 0;
    const int p = w.len - w.n + t;
    q.token = w.offset + t;
    q.head = head * R + h;
    q.hi = p < 0 ? 0 : p + 1;
    q.lo = p >= a.window ? p - a.window + 1 : 0;
    return q;
}
__device__ __forceinline__ int64_t page_row(const CacheView& c, int head, int page, int at)
{
    const uint32_t p = (uint32_t)page < (uint64_t)c.num_pages ? (uint32_t)page : 0u;
    return (int64_t)((((uint64_t)p * (uint32_t)c.heads + (uint32_t)head) << c.page_shift) + (uint32_t)(at & (c.page_size - 1)));
}
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const bf16x2 p = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, p);
}

// A wave's item: kTiles columns of 16 queries.  One query's scores lie in one lane column (see prefix attention's step).
template <int D, bool kFp8, int kTiles>
struct Few {
    using Data = StepData<D, kFp8>;
    static constexpr int kBlocks = D / 16, kSteps = D / 32;
    bf16x8 q[kTiles][kSteps];
    f32x4 o[kTiles][kBlocks];
    float m[kTiles], l[kTiles];
    int lo[kTiles], hi[kTiles];

    __device__ __forceinline__ void run(const CacheView& c, const WindowArgs& a, int R, const Work& w, const Piece1& piece, float2* ml_out, float* o_out)
    {
        const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
        const Band band = band_of(R, w.tile, w.n, w.len, a.window, a.sinks, kStep);
        const int sure_hi = band.p0 + 1;                                       // every query sees the tokens below it
        const int sure_lo = band.p1 >= a.window ? band.p1 - a.window + 1 : 0;  // and from here on
        const int32_t* pages = a.row_pages + (int64_t)w.row * a.row_width;
        auto page_at = [&](int k) { return k < piece.to ? pages[band.at(k, kStep) >> c.page_shift] : -1; };
        Data d;
        int page = page_at(piece.from), page_next = page_at(piece.from + 1);
        {
            const int64_t row = page_row(c, piece.head, page, band.at(piece.from, kStep));
            d.load_keys(c, row, lane);
            d.load_values(c, row, lane);
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const Query x = query_of(a, R, w, piece.head, t * 16 + col);
            const uint16_t* qp = a.q + x.token * a.q_token_stride + x.head * a.q_head_stride;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                u32x4 v = *reinterpret_cast<const u32x4*>(qp + Data::key_column(s, g));
                if (!x.is) v = u32x4{0, 0, 0, 0};
                q[t][s] = __builtin_bit_cast(bf16x8, v);
            }
            lo[t] = x.lo; hi[t] = x.hi;
            m[t] = kNoScore; l[t] = 0.0f;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) o[t][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const float scale = a.scale * kLog2eF;
        for (int k = piece.from; k < piece.to; ++k) {
            const int at = band.at(k, kStep);
            const int page_after = page_at(k + 2);
            const int64_t next = page_row(c, piece.head, page_next, k + 1 < piece.to ? band.at(k + 1, kStep) : 0);   // behind the last: read for nothing
            const bool there = (uint32_t)page < (uint64_t)c.num_pages;
            const bool edge = !there || at + kStep > sure_hi || (at < sure_lo && at + kStep > a.sinks);   // uniform: not all see all
            float x[kTiles][8];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                f32x4 s[2] = {f32x4{0.0f, 0.0f, 0.0f, 0.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
#pragma unroll
                    for (int u = 0; u < 2; ++u) s[u] = mfma(d.key(u, i), q[t][i], s[u]);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[t][j] = s[j >> 2][j & 3] * (kFp8 ? scale * d.k_factor(j) : scale);
            }
            d.load_keys(c, next, lane);
            auto sees = [&](int t, int j) {
                const int token = at + 8 * g + j;
                return there && token < hi[t] && (token >= lo[t] || token < a.sinks);
            };
            if (edge) {
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[t][j] = sees(t, j) ? x[t][j] : -INFINITY;
            }
            bf16x8 p[kTiles], rest[kTiles], last[kTiles];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                float top = fmax3(fmax3(x[t][0], x[t][1], x[t][2]), fmax3(x[t][3], x[t][4], x[t][5]), fmaxf(x[t][6], x[t][7]));
                if (__any(top > m[t] + kSlack)) {
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    const float to = fmaxf(m[t], top);
                    const float f = __builtin_amdgcn_exp2f(m[t] - to);
                    m[t] = to;
                    l[t] *= f;
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b) o[t][b] *= f;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float e = __builtin_amdgcn_exp2f(x[t][j] - m[t]);
                    l[t] += e;
                    float v = kFp8 ? e * d.v_factor(j) : e;
                    if (kFp8 && edge) v = sees(t, j) ? v : 0.0f;               // a hidden token's scale may be anything
                    p[t][j] = (__bf16)v;
                    const float left = v - (float)p[t][j];
                    rest[t][j] = (__bf16)left;
                    last[t][j] = (__bf16)(left - (float)rest[t][j]);
                }
            }
            // Tokens that not all queries see: a weight of zero keeps them out, unless the value is no finite number.  Such values
            // leave the product, and one more counts those that a query sees.
            if (__builtin_expect(edge && __any(d.unbounded()), 0)) {
#pragma unroll
                for (int i = 0; i < Data::kVLoads; ++i) {
                    u32x4 ones;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t bad = Data::unbounded_in(d.v[i][j]);
                        ones[j] = bad & (kFp8 ? 0x38383838u : 0x3F803F80u);
                        d.v[i][j] &= ~bad;
                    }
#pragma unroll
                    for (int u = 0; u < kBlocks / Data::kVLoads; ++u) {
                        const int b = i * (kBlocks / Data::kVLoads) + u;
                        const bf16x8 one = kFp8 ? (u ? widen(ones.z, ones.w) : widen(ones.x, ones.y)) : __builtin_bit_cast(bf16x8, ones);
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) {
                            bf16x8 seen;
#pragma unroll
                            for (int j = 0; j < 8; ++j) seen[j] = (__bf16)(sees(t, j) ? 1.0f : 0.0f);
                            const f32x4 count = mfma(one, seen, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
                            for (int n = 0; n < 4; ++n) o[t][b][n] = count[n] > 0.0f ? __builtin_nanf("") : o[t][b][n];
                        }
                    }
                }
            }
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                const bf16x8 value = d.value(b);
#pragma unroll
                for (int t = 0; t < kTiles; ++t) o[t][b] = mfma(value, last[t], mfma(value, rest[t], mfma(value, p[t], o[t][b])));
            }
            d.load_values(c, next, lane);
            page = page_next;
            page_next = page_after;
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            l[t] += __shfl_xor(l[t], 16);
            l[t] += __shfl_xor(l[t], 32);
            const Query x = query_of(a, R, w, piece.head, t * 16 + col);
            if (!x.is) continue;
            if (!piece.whole) {
                if (g == 0) ml_out[t * 16 + col] = float2{m[t], l[t]};
                float* to = o_out + (int64_t)(t * 16 + col) * D;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) to[Data::column(b, 4 * g + i)] = o[t][b][i];
                continue;
            }
            const bool none = l[t] == 0.0f && m[t] == kNoScore;
            const float inv = none ? 0.0f : 1.0f / l[t];
            const int64_t where = (int64_t)x.token * a.q_heads + x.head;
            uint16_t* to = a.out + where * D;
            if (kFp8) {                                                        // blocks b and b + 1 hold columns in turn
#pragma unroll
                for (int b = 0; b < kBlocks; b += 2) {
                    u32x4 v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = pack2(o[t][b][i] * inv, o[t][b + 1][i] * inv);
                    *reinterpret_cast<u32x4*>(to + Data::column(b, 4 * g)) = v;
                }
            } else {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
                    *reinterpret_cast<u32x2*>(to + Data::column(b, 4 * g)) =
                        u32x2{pack2(o[t][b][0] * inv, o[t][b][1] * inv), pack2(o[t][b][2] * inv, o[t][b][3] * inv)};
            }
            if (a.lse && g == 0) a.lse[where] = none ? -INFINITY : (m[t] + __builtin_amdgcn_logf(l[t])) * (float)kLn2;
        }
    }
};

// A workgroup's item: a wave takes 32 queries, on the columns of 32 x 32 products.  S^T = K Q^T leaves 16 scores of one query in a lane,
// and since a sum over tokens may be taken in any order, row 8 a + 4 h + b of a score tile is given token 16 (a >> 1) + 8 h + 4 (a & 1) + b:
// a lane's scores are then tokens 8 h .. 8 h + 7 of either half, what it has to hold of P^T as operand of O^T = V^T P^T.
// In LDS, twice: keys as rows of 16-byte pieces whose places are turned by the token, so that the lanes of a wave, which read one
// piece of 32 rows, meet all banks; values as the cache has them, eight tokens of a column together.  A 16-bit cache goes there
// from memory without registers in between, while the block before is worked on; codes pass through registers, widened to bf16
// (once for the four waves; the powers of two are applied in fp32 to scores and weights).
template <int D, bool kFp8>
struct Many {
    static constexpr int kPieces = D / 8;                                      // 16-byte pieces of a row in bf16
    static constexpr int kKeys = kBlock * D * 2, kValues = kBlock * D * 2;
    static constexpr int kImage = kKeys + kValues;                             // two of them, within the 64 KB that a load into LDS reaches,
    static constexpr int kFactors = 2 * kBlock * 4, kExtra = kFactors + 16;    // then twice factors and four flags
    static constexpr int kLds = 2 * (kImage + kExtra);
    static_assert(kLds % 16 == 0, "what lies behind it is aligned");
    static constexpr int kElem = kFp8 ? 1 : 2;
    static constexpr int kRow = D * kElem / 16;                                // pieces of a row in the cache
    static constexpr int kLoads = kBlock * kRow / 256;                         // of 16 bytes, a thread's, of K and of V
    static constexpr int kCols = D / 32, kDeep = D / 16;

    u32x4 k[kFp8 ? kLoads : 1], v[kFp8 ? kLoads : 1];
    uint32_t factor;

    static __device__ __forceinline__ int turned(int token, int piece)
    {
        return piece ^ (kPieces == 16 ? token & 15 : (token >> 1) & 7);
    }
    // 16 bytes a lane from memory, `offset` behind `from`, into LDS, lane after lane from `to` on (from and to the same in all of them).
    // A load into LDS needs a wait state behind a write of m0, or it may go by the place of the load before; nothing adds it to assembly.
    // (m0 is named as lost so that no value of the compiler's own is kept in it; the warning is that it does not save it.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    static __device__ __forceinline__ void to_lds(const char* from, uint32_t offset, uint32_t to)
    {
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(offset), "s"(from), "s"(to) : "memory", "m0");
    }
#pragma clang diagnostic pop
    static __device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
    // Writes to LDS are there for all waves.  Loads from memory stay on their way.
    static __device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

    // Where the next block lies: its two halves' rows (the same for all lanes; what a lane takes of them is the same in every block) and the
    // image that it goes to.
    const char* keys_at[2];
    const char* values_at[2];
    uint32_t image_at;
    uint32_t of_key, of_value;                                                 // the lane's part
    __device__ __forceinline__ void begin()
    {
        // (the tokens of a thread's loads differ by a multiple of 16, which does not turn its piece)
        const int x = kFp8 && kLoads == 1 ? threadIdx.x & 127 : threadIdx.x, token = x / kRow, piece = x % kRow;
        of_key = token * D * kElem + (kFp8 ? piece : turned(token, piece)) * 16;
        of_value = x * 16;
    }
    __device__ __forceinline__ void aim(const CacheView& c, int head, const int page[2], int at)
    {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int64_t row = page_row(c, head, uniform(page[half]), at + 32 * half);        // scalar arithmetic; the same in both tensors
            keys_at[half] = static_cast<const char*>(c.k) + row * (D * kElem);
            values_at[half] = static_cast<const char*>(c.v) + row * (D * kElem);
            if (kFp8) {
                const int token = threadIdx.x & 63;
                if (half == 0) scales_row = row + (token & 31);
                else scales_row = token < 32 ? scales_row : row + (token & 31);
            }
        }
    }
    int64_t scales_row;                                                        // the row whose scale byte the thread takes
    // The next block's load i of kAll: codes into registers, 16-bit elements into LDS.
    static constexpr int kAll = 2 * kLoads + (kFp8 ? 1 : 0);
    __device__ __forceinline__ void load(const CacheView& c, int i)
    {
        if (i == 2 * kLoads) {
            factor = threadIdx.x < 64 ? c.k_scale[scales_row] : c.v_scale[scales_row];
            return;
        }
        const bool key = i < kLoads;
        const int n = key ? i : i - kLoads;
        const uint32_t of = key ? of_key : of_value;
        const int wave = uniform((int)threadIdx.x >> 6);
        if (kFp8 && kLoads == 1) {                                             // two waves a half
            const char* at = key ? (wave >= 2 ? keys_at[1] : keys_at[0]) : (wave >= 2 ? values_at[1] : values_at[0]);
            (key ? k : v)[0] = *reinterpret_cast<const u32x4*>(at + of);
            return;
        }
        constexpr int kOfHalf = kLoads / 2 > 0 ? kLoads / 2 : 1, kTokens = 256 / kRow;         // loads of a half, and the tokens of one
        const char* at = (key ? keys_at : values_at)[n / kOfHalf] + n % kOfHalf * (kTokens * D * kElem);
        if (kFp8) (key ? k : v)[n] = *reinterpret_cast<const u32x4*>(at + of);
        else to_lds(at, of, image_at + (key ? 0 : kKeys) + (n * 256 + wave * 64) * 16);
    }
    static __device__ __forceinline__ u32x4 wide(uint32_t lo, uint32_t hi) { return __builtin_bit_cast(u32x4, widen(lo, hi)); }
    static __device__ __forceinline__ uint32_t clean(u32x4& w)
    {
        uint32_t bad = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t b = StepData<D, kFp8>::unbounded_in(w[j]);
            w[j] &= ~b;
            bad |= b;
        }
        return bad;
    }
    // ... and what was fetched is in LDS as far as this wave goes.  `check`: values may be hidden from some queries; those that are no finite numbers
    // become zeros, and flags tell of them.
    __device__ __forceinline__ void put(char* image, char* extra, float scale, bool check)
    {
        u32x4* keys = reinterpret_cast<u32x4*>(image);
        u32x4* values = reinterpret_cast<u32x4*>(image + kKeys);
        uint32_t bad = 0;
        if (kFp8) {
            if (check) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) bad |= clean(v[i]);
            }
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int x = i * 256 + (int)threadIdx.x, token = x / kRow, piece = x % kRow;
                keys[token * kPieces + turned(token, 2 * piece)] = wide(k[i].x, k[i].y);
                keys[token * kPieces + turned(token, 2 * piece + 1)] = wide(k[i].z, k[i].w);
                values[2 * x] = wide(v[i].x, v[i].y);
                values[2 * x + 1] = wide(v[i].z, v[i].w);
            }
            float* factors = reinterpret_cast<float*>(extra);
            if (threadIdx.x < 128) {
                // (a hidden token's byte may be anything, 255 would be infinite: a weight of zero times it must be zero)
                const float f = __uint_as_float((factor < 254 ? factor : 254) << 23);
                factors[threadIdx.x] = threadIdx.x < 64 ? f * scale : f;
            }
        } else {
            landed();
            if (check) {
#pragma unroll 1
                for (int i = 0; i < kLoads; ++i) {                             // what the thread itself has fetched
                    u32x4 w = values[i * 256 + threadIdx.x];
                    const uint32_t b = clean(w);
                    if (b != 0) values[i * 256 + threadIdx.x] = w;
                    bad |= b;
                }
            }
        }
        const bool any = __any(bad != 0);
        if ((threadIdx.x & 63) == 0) reinterpret_cast<int*>(extra + kFactors)[threadIdx.x >> 6] = any;
    }

    static __device__ __forceinline__ f32x16 product(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x16 zero()
    {
        f32x16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.0f;
        return z;
    }

    static __device__ __forceinline__ uint64_t below(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }

    // What the workgroup has ahead of it: pages of the next two blocks and the image that the next one is in; `ready`: it is on its way.
    int page[2], after[2];
    int image_of;
    bool ready;
    // The first block of an item that follows: `is` where there is one.
    struct Next {
        Work w;
        int head;
        bool is;
    };
    static __device__ __forceinline__ int page_of(const CacheView& c, const WindowArgs& a, const Work& w, const Band& band, int s, int steps, int half)
    {
        // a half that none of the tile's queries sees may lie behind the table
        const int at = s < steps ? band.at(s, kBlock) + 32 * half : 0x7FFFFFFF;
        return at <= band.p1 ? a.row_pages[(int64_t)w.row * a.row_width + (at >> c.page_shift)] : -1;
    }

    __device__ __forceinline__ void run(const CacheView& c, const WindowArgs& a, int R, const Work& w, const Piece1& piece, const Next& next, char* lds,
                                        float2* ml_out, float* o_out)
    {
        const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), col = lane & 31, h = lane >> 5;
        const Band band = band_of(R, w.tile, w.n, w.len, a.window, a.sinks, kBlock);
        // the wave's queries
        const uint32_t first = (uint32_t)w.tile * kTile + (uint32_t)wave * 32, queries = (uint32_t)w.n * (uint32_t)R;
        const bool busy = first < queries;
        const uint32_t end = first + 32 < queries ? first + 32 : queries;
        const int p0 = w.len - w.n + (int)(first / (uint32_t)R), p1 = w.len - w.n + (int)((end - 1) / (uint32_t)R);
        const int wave_hi = p1 + 1, wave_lo = p0 >= a.window ? p0 - a.window + 1 : 0;          // what any of them sees
        const int sure_hi = p0 + 1, sure_lo = p1 >= a.window ? p1 - a.window + 1 : 0;          // what all of them see
        const int tile_sure_hi = band.p0 + 1, tile_sure_lo = band.p1 >= a.window ? band.p1 - a.window + 1 : 0;
        const Query x = query_of(a, R, w, piece.head, first + col);
        const uint32_t lds_at = (uint32_t)(uintptr_t)reinterpret_cast<__attribute__((address_space(3))) char*>(reinterpret_cast<uintptr_t>(lds));

        bf16x8 q[kDeep];
        {
            const uint16_t* qp = a.q + x.token * a.q_token_stride + x.head * a.q_head_stride;
#pragma unroll
            for (int s = 0; s < kDeep; ++s) {
                u32x4 u = *reinterpret_cast<const u32x4*>(qp + 16 * s + 8 * h);
                if (!x.is) u = u32x4{0, 0, 0, 0};
                q[s] = __builtin_bit_cast(bf16x8, u);
            }
        }
        // the next item's first pages are asked for now, its first block in this item's last step
        int next_page[2] = {-1, -1}, next_after[2] = {-1, -1}, next_at = 0;
        if (next.is) {
            const Band next_band = band_of(R, next.w.tile, next.w.n, next.w.len, a.window, a.sinks, kBlock);
            next_at = next_band.at(0, kBlock);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                next_page[half] = page_of(c, a, next.w, next_band, 0, next_band.steps, half);
                next_after[half] = page_of(c, a, next.w, next_band, 1, next_band.steps, half);
            }
        }
        if (!ready && piece.from < piece.to) {
            meet();                                                            // the last item's blocks are done with
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                page[half] = page_of(c, a, w, band, piece.from, piece.to, half);
                after[half] = page_of(c, a, w, band, piece.from + 1, piece.to, half);
            }
            image_of = 0;
            aim(c, piece.head, page, band.at(piece.from, kBlock));
            image_at = lds_at;
#pragma unroll
            for (int i = 0; i < kAll; ++i) load(c, i);
        }
        float m = kNoScore, l = 0.0f;
        f32x16 o[kCols];
#pragma unroll
        for (int b = 0; b < kCols; ++b) o[b] = zero();
        const float scale = a.scale * kLog2eF;
        // row of the score tile -> token; where its piece h lies (piece 2 i + h: that place with the bits of 2 i turned)
        const int token_of_row = 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
        const uint32_t key_row = token_of_row * (D * 2), key_piece = turned(token_of_row, h) * 16;

        for (int s = piece.from; s < piece.to; ++s) {
            char* image = lds + image_of * kImage;
            char* extra = lds + 2 * kImage + image_of * kExtra;
            image_of ^= 1;
            const int at = band.at(s, kBlock);
            const int now[2] = {uniform(page[0]), uniform(page[1])};
            const bool there[2] = {(uint32_t)now[0] < (uint64_t)c.num_pages, (uint32_t)now[1] < (uint64_t)c.num_pages};
            const bool whole = there[0] && there[1];
            const bool check = !(whole && at + kBlock <= tile_sure_hi && (at >= tile_sure_lo || at + kBlock <= a.sinks));
            put(image, extra, scale, check);
            // The next block: this item's, or the next one's first.  (Behind the last of all the same block comes once more, for nothing:
            // the loads lie between products, without branches.)
            const bool last = s + 1 == piece.to;
            ready = !last || next.is;
            if (!last) {
                page[0] = after[0]; page[1] = after[1];
                after[0] = page_of(c, a, w, band, s + 2, piece.to, 0);
                after[1] = page_of(c, a, w, band, s + 2, piece.to, 1);
            } else if (next.is) {
                page[0] = next_page[0]; page[1] = next_page[1];
                after[0] = next_after[0]; after[1] = next_after[1];
            }
            if (ready) aim(c, last ? next.head : piece.head, page, last ? next_at : band.at(s + 1, kBlock));
            image_at = lds_at + image_of * kImage;
            meet();                                                            // all waves' parts are there, and the other image is done with
            // Of two workgroups on a compute unit the older one's waves go first and it would end earlier, the other then being alone:
            // they take turns (prompts 465 us, without 473).
            if (((s >> 2) ^ (int)(blockIdx.x / (gridDim.x / kPerUnit))) & 1) __builtin_amdgcn_s_setprio(1);
            else __builtin_amdgcn_s_setprio(0);
            const bool edge = !(whole && at + kBlock <= sure_hi && (at >= sure_lo || at + kBlock <= a.sinks));
            const u32x4* values = reinterpret_cast<const u32x4*>(image + kKeys) + h * D + col;
            const float* factors = reinterpret_cast<const float*>(extra);
            // Pieces of the keys are asked for six products ahead (left to itself the compiler asks for each right before its product
            // and waits; three ahead measured the same), the next block's loads, which take the memory units 500 cycles a workgroup, one every other
            // product.
            static_assert(kAll <= kDeep, "a load every other product");
            f32x16 t[2] = {zero(), zero()};
            {
                constexpr int kAhead = 6;
                bf16x8 piece_of[kAhead];
                auto ask = [&](int j) {
                    piece_of[j % kAhead] = *reinterpret_cast<const bf16x8*>(image + key_row + (key_piece ^ (j / 2 * 32)) + j % 2 * (32 * D * 2));
                };
#pragma unroll
                for (int j = 0; j < kAhead; ++j) ask(j);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 2 * kDeep; ++j) {
                    t[j % 2] = product(piece_of[j % kAhead], q[j / 2], t[j % 2]);
                    if (j + kAhead < 2 * kDeep) ask(j + kAhead);
                    if (j % 2 == 1 && j / 2 < kAll) load(c, j / 2);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (!busy || at >= wave_hi || (at + kBlock <= wave_lo && at >= a.sinks)) continue;         // (the loads above are every wave's)
            if (kFp8) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) t[b][i] *= factors[32 * b + 16 * (i >> 3) + 8 * h + (i & 7)];
            }
            if (edge) {
                // A bit for every token from the lane's first one on; token 32 b + 16 (i >> 3) + (i & 7) is the lane's number i of half b.
                const int base = at + 8 * h, kept = a.sinks < x.hi ? a.sinks : x.hi;
                const uint64_t seen = (below(x.hi - base) & ~below(x.lo - base)) | below(kept - base);
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint32_t bits = there[b] ? (uint32_t)(seen >> (32 * b)) : 0u;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t all = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 16 * (i >> 3) + (i & 7), 1);
                        t[b][i] = __uint_as_float((__float_as_uint(t[b][i]) & all) | (0xFF800000u & ~all));
                    }
                }
            }
            float tops[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                tops[k] = t[k >> 1][8 * (k & 1)];
#pragma unroll
                for (int i = 1; i < 8; ++i) tops[k] = fmaxf(tops[k], t[k >> 1][8 * (k & 1) + i]);
            }
            float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
            if (!kFp8) top *= scale;                                           // the scale enters the exponent below
            if (__any(top > m + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 32));
                const float to = fmaxf(m, top);
                const float f = __builtin_amdgcn_exp2f(m - to);
                m = to;
                l *= f;
#pragma unroll
                for (int b = 0; b < kCols; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[b][i] *= f;
            }
            // Weights of 16 tokens as two bf16 numbers each, two weights at a time: the next tokens' between the products of these.
            float sum[2] = {0.0f, 0.0f};
            u32x4 p[2], rest[2];
            auto weigh = [&](int n, int j) {
                float u[2];
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const float y = t[n >> 1][8 * (n & 1) + 2 * j + g];
                    const float e = __builtin_amdgcn_exp2f(kFp8 ? y - m : fmaf(y, scale, -m));
                    t[n >> 1][8 * (n & 1) + 2 * j + g] = e;
                    u[g] = kFp8 ? e * factors[kBlock + 16 * n + 8 * h + 2 * j + g] : e;
                }
                uint32_t w2 = pack2(u[0], u[1]);
                asm("" : "+v"(w2));                                            // (or each half would be rounded once more on its own)
                p[n & 1][j] = w2;
                rest[n & 1][j] = pack2(u[0] - __uint_as_float(w2 << 16), u[1] - __uint_as_float(w2 & 0xFFFF0000u));
            };
            bf16x8 value[2][kCols];
            auto ask = [&](int n, int d) { value[n & 1][d] = __builtin_bit_cast(bf16x8, values[2 * n * D + 32 * d]); };
#pragma unroll
            for (int d = 0; d < kCols; ++d) ask(0, d);
#pragma unroll
            for (int j = 0; j < 4; ++j) weigh(0, j);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const bf16x8 pb = __builtin_bit_cast(bf16x8, p[n & 1]), rb = __builtin_bit_cast(bf16x8, rest[n & 1]);
#pragma unroll
                for (int d = 0; d < 2 * kCols; ++d) {                          // first all columns with p, then with the rest
                    o[d % kCols] = product(value[n & 1][d % kCols], d < kCols ? pb : rb, o[d % kCols]);
                    if (n < 3) {
                        if (d < kCols) ask(n + 1, d);
                        if (d % (kCols / 2) == kCols / 2 - 1) weigh(n + 1, d / (kCols / 2));
                    } else {                                                   // the weights' sum between the last products
                        constexpr int kAdds = 32 / (2 * kCols);
#pragma unroll
                        for (int j = d * kAdds; j < (d + 1) * kAdds; ++j) sum[j & 1] += t[j >> 4][j & 15];
                        asm volatile("" : "+v"(sum[0]), "+v"(sum[1]));         // (or they all come behind)
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            l += sum[0] + sum[1];
            const int* flags = reinterpret_cast<const int*>(extra + kFactors);
            if (__builtin_expect(check && (flags[0] | flags[1] | flags[2] | flags[3]) != 0, 0)) {
                // Values that are no finite numbers, hidden from some queries (zeros in LDS): one more product, with what the cache
                // holds, counts those that a query sees.
#pragma unroll 1
                for (int n = 0; n < 4; ++n) {
                    const bool is = n < 2 ? there[0] : there[1];
                    const int64_t row = page_row(c, piece.head, n < 2 ? now[0] : now[1], at + 16 * n + 8 * h);
                    bf16x8 seen;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int token = at + 16 * n + 8 * h + j;
                        seen[j] = (__bf16)(is && token < x.hi && (token >= x.lo || token < a.sinks) ? 1.0f : 0.0f);
                    }
                    const char* from = static_cast<const char*>(c.v) + row * (D * kElem) + col * (8 * kElem);
#pragma unroll
                    for (int d = 0; d < kCols; ++d) {
                        bf16x8 ones;
                        if (kFp8) {
                            const u32x2 v = *reinterpret_cast<const u32x2*>(from + d * 256);
                            ones = widen(StepData<D, true>::unbounded_in(v.x) & 0x38383838u, StepData<D, true>::unbounded_in(v.y) & 0x38383838u);
                        } else {
                            u32x4 v = *reinterpret_cast<const u32x4*>(from + d * 512);
#pragma unroll
                            for (int j = 0; j < 4; ++j) v[j] = StepData<D, false>::unbounded_in(v[j]) & 0x3F803F80u;
                            ones = __builtin_bit_cast(bf16x8, v);
                        }
                        const f32x16 count = product(ones, seen, zero());
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[d][i] = count[i] > 0.0f ? __builtin_nanf("") : o[d][i];
                    }
                }
            }
        }
        if (!busy) return;
        l += __shfl_xor(l, 32);
        if (!x.is) return;
        const bool none = l == 0.0f && m == kNoScore;
        if (!piece.whole) {
            const int place = wave * 32 + col;
            if (h == 0) ml_out[place] = float2{m, l};
            float* to = o_out + (int64_t)place * D + 4 * h;
#pragma unroll
            for (int b = 0; b < kCols; ++b)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<f32x4*>(to + 32 * b + 2 * i) = f32x4{o[b][i], o[b][i + 1], o[b][i + 2], o[b][i + 3]};
            return;
        }
        const float inv = none ? 0.0f : 1.0f / l;
        const int64_t where = (int64_t)x.token * a.q_heads + x.head;
        uint16_t* to = a.out + where * D + 4 * h;
#pragma unroll
        for (int b = 0; b < kCols; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<u32x2*>(to + 32 * b + 2 * i) = u32x2{pack2(o[b][i] * inv, o[b][i + 1] * inv), pack2(o[b][i + 2] * inv, o[b][i + 3] * inv)};
        if (a.lse && h == 0) a.lse[where] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * (float)kLn2;
    }
};

// The stretch of worker `part`: f(record, piece, which of the worker's two places, record and head of what lies behind the piece in the stretch,
// whether that is an item's first steps).
template <int kLine, typename List, typename F>
__device__ __forceinline__ void along(const List& list, const Division& d, int heads, int part, Cut* cut, F f)
{
    using Step = typename List::Step;
    const bool writes = (threadIdx.x & (kLine == kOfGroups ? 255 : 63)) == 0;
    Cut found{-1, 0, 0, 0, 0, 0, 0, 0};
    if (part >= d.parts[kLine]) {
        if (writes) *cut = found;
        return;
    }
    const Stretches<Step> stretches((Step)d.steps[kLine], d.parts[kLine]);
    Step at = stretches.begin(part);
    const Step end = stretches.begin(part + 1), begin = at;
    int i = find_work(list, list.count, at);
    Work w = uniform(list.get(i));
    while (at < end) {
        const Step offset = at - (Step)w.first;
        const int head = sizeof(Step) == 4 ? (int)((uint32_t)offset / (uint32_t)w.cost) : (int)divide(offset, w.cost);
        const int from = (int)(offset - (Step)head * w.cost);
        const int n = end - at < w.cost - from ? (int)(end - at) : w.cost - from;
        Piece1 piece;
        piece.head = head;
        piece.from = from > kCost ? from - kCost : 0;
        piece.to = from + n - kCost;
        piece.whole = w.cost == kCost ? from == 0 : from <= kCost && from + n == w.cost;
        if (piece.to < 0) piece.to = 0;
        if (at == begin && from > kCost) {
            // the item began before: was its first step the worker's before?
            const Step item = at - from;
            if (stretches.begin(part - 1) <= item + kCost) found = Cut{w.row, w.tile, w.offset, w.n, w.len, head, stretches.of(item + w.cost - 1), 0};
        }
        // what follows: the same tile's next head, or the next tile
        const bool done = head + 1 == heads && from + n == w.cost;
        Work after = w;
        if (done && at + n < end) {
            i = list.next(i, at + n);
            after = uniform(list.get(i));
        }
        const bool more = at + n < end && from + n == w.cost && after.cost > kCost && end - (at + n) > kCost;
        if (piece.to > piece.from || (w.cost == kCost && piece.whole)) f(w, piece, from <= kCost ? 1 : 0, after, done ? 0 : head + 1, more);
        at += n;
        if (done) w = after;
    }
    if (writes) *cut = found;
}

template <int D, bool kFp8, bool kOwn>
__global__ __launch_bounds__(64 * kWaves, kPerUnit)
void window_kernel(CacheView c, WindowArgs a, WindowShape s, char* ws)
{
    // (one array: the blocks are within the 64 KB that a load into LDS reaches)
    __shared__ __align__(16) char lds[Many<D, kFp8>::kLds + (kOwn ? sizeof(OwnPlan) : 0)];
    OwnPlan& own = *reinterpret_cast<OwnPlan*>(lds + Many<D, kFp8>::kLds);
    Totals totals;
    if constexpr (kOwn) totals = plan_own(a, s, c.heads, c.page_size, own);
    else totals = *reinterpret_cast<const Totals*>(ws);
    const int workgroups = (int)gridDim.x;
    const Division d = divide_work(totals, workgroups);
    auto list = [&](auto line) {
        if constexpr (kOwn) return InLds<decltype(line)::value>{own, uniform(totals.count[0])};
        else return InWorkspace{reinterpret_cast<const Work*>(ws + s.at_list[decltype(line)::value]), uniform(totals.count[decltype(line)::value])};
    };
    Cut* cuts = reinterpret_cast<Cut*>(ws + s.at_cuts);
    Cut* wave_cuts = cuts + s.workers[kOfGroups];
    float2* ml = reinterpret_cast<float2*>(ws + s.at_ml);
    // Workgroups of one die (dealt in turn to eight) lie next to each other on the line: they read the same keys.
    const int block = (workgroups & 7) == 0 ? (int)(blockIdx.x & 7) * (workgroups >> 3) + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
    const int wave = uniform((int)threadIdx.x >> 6);
    const Cut none{-1, 0, 0, 0, 0, 0, 0, 0};
    if (block < d.groups) {
        // (the join looks at every worker's cut: waves of these workgroups are no workers of the other line)
        if ((threadIdx.x & 63) == 0) wave_cuts[(workgroups - d.groups) * kWaves + block * kWaves + wave] = none;
        float* o = reinterpret_cast<float*>(ws + s.at_o[kOfGroups]);
        Many<D, kFp8> x;
        x.begin();
        x.ready = false;
        along<kOfGroups>(list(std::integral_constant<int, kOfGroups>{}), d, c.heads, block, cuts + block,
                         [&](const Work& w, const Piece1& piece, int which, const Work& after, int head, bool more) {
                             const int64_t place = (2 * block + which) * (int64_t)kTile;
                             x.run(c, a, s.R, w, piece, {after, head, more}, lds, ml + place, o + place * D);
                         });
        Many<D, kFp8>::landed();
        return;
    }
    if (s.workers[kOfGroups] > 0 && threadIdx.x == 0) cuts[block] = none;
    // a workgroup's waves lie far apart on their line: few stretches are spread over all workgroups
    const int part = wave * (workgroups - d.groups) + block - d.groups;
    float* o = reinterpret_cast<float*>(ws + s.at_o[kOfWaves]);
    along<kOfWaves>(list(std::integral_constant<int, kOfWaves>{}), d, c.heads, part, wave_cuts + part,
                    [&](const Work& w, const Piece1& piece, int which, const Work&, int, bool) {
                        const int64_t place = (2 * part + which) * (int64_t)kFewQueries;
                        float2* ml_out = ml + 2 * (int64_t)s.workers[0] * kTile + place;
                        if (w.n * s.R <= 16) {
                            Few<D, kFp8, 1> x;
                            x.run(c, a, s.R, w, piece, ml_out, o + place * D);
                        } else {
                            Few<D, kFp8, 2> x;
                            x.run(c, a, s.R, w, piece, ml_out, o + place * D);
                        }
                    });
}

// ---------------------------------------------------------------- join
// A workgroup per worker whose stretch begins inside an item (the first such one of the item) and a few of its queries; D / 4 lanes a query,
// fewer queries than lots of lanes have their parts spread over several.
template <int D>
__global__ __launch_bounds__(256, 8)
void window_join_kernel(WindowArgs a, WindowShape s, int group_shift, int wave_shift, const char* ws)
{
    constexpr int kLanes4 = D / 4, kSubs = 256 / kLanes4;
    __shared__ float lds[kSubs][2 + D];
    const int of_groups = s.workers[kOfGroups] << group_shift;
    const bool groups = (int)blockIdx.x < of_groups;
    const int shift = groups ? group_shift : wave_shift;                       // of the number of slices
    const int block = groups ? (int)blockIdx.x : (int)blockIdx.x - of_groups;
    const int part = block >> shift, slice = block & ((1 << shift) - 1);
    const Cut cut = reinterpret_cast<const Cut*>(ws + s.at_cuts)[(groups ? 0 : s.workers[kOfGroups]) + part];
    if (cut.row < 0) return;
    const Work w{0, cut.row, cut.tile, cut.offset, cut.n, cut.len, 0};
    const int places = groups ? kTile : kFewQueries, each = places >> shift;
    const int64_t base = groups ? (int64_t)w.tile * kTile : 0, queries = (int64_t)w.n * s.R - base;
    const int first = slice * each, end = queries < first + each ? (int)queries : first + each;
    if (first >= end) return;
    const float2* ml = reinterpret_cast<const float2*>(ws + s.at_ml) + (groups ? 0 : 2 * (int64_t)s.workers[kOfGroups] * kTile);
    const float* o = reinterpret_cast<const float*>(ws + s.at_o[groups ? kOfGroups : kOfWaves]);
    const int sub = threadIdx.x / kLanes4, col = (threadIdx.x % kLanes4) * 4;
    const int parts = cut.last - part + 2;
    const int wide = end - first < kSubs ? end - first : kSubs;                                // uniform
    const int spread_shift = 31 - __builtin_clz(kSubs) - (wide > 1 ? 32 - __builtin_clz(wide - 1) : 0), spread = 1 << spread_shift;
    for (int q0 = first; q0 < end; q0 += wide) {
        const int query = q0 + (sub >> spread_shift);
        const bool is = (sub >> spread_shift) < wide && query < end;
        float m = kNoScore, l = 0.0f;
        f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
        if (is) {
            for (int i = (sub & (spread - 1)); i < parts; i += 4 * spread) {
                float2 pw[4];
                f32x4 po[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int j = i + k * spread < parts ? i + k * spread : i;
                    // the first part lies at the end of the worker's before
                    const int64_t at = (j == 0 ? 2 * (int64_t)(part - 1) + 1 : 2 * (int64_t)(part + j - 1)) * places + query;
                    pw[k] = ml[at];
                    po[k] = *reinterpret_cast<const f32x4*>(o + at * D + col);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i + k * spread < parts) {
                        const float to = fmaxf(m, pw[k].x);
                        const float f = __builtin_amdgcn_exp2f(m - to), g = __builtin_amdgcn_exp2f(pw[k].x - to);
                        m = to;
                        l = l * f + pw[k].y * g;
                        x = x * f + po[k] * g;
                    }
            }
        }
        if (spread > 1) {
            __syncthreads();
            if (col == 0) { lds[sub][0] = m; lds[sub][1] = l; }
#pragma unroll
            for (int j = 0; j < 4; ++j) lds[sub][2 + col + j] = x[j];
            __syncthreads();
            if (is && (sub & (spread - 1)) == 0) {
                for (int k = sub + 1; k < sub + spread; ++k) {
                    const float to = fmaxf(m, lds[k][0]);
                    const float f = __builtin_amdgcn_exp2f(m - to), g = __builtin_amdgcn_exp2f(lds[k][0] - to);
                    m = to;
                    l = l * f + lds[k][1] * g;
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = x[j] * f + lds[k][2 + col + j] * g;
                }
            }
        }
        if (is && (sub & (spread - 1)) == 0) {
            const Query t = query_of(a, s.R, w, cut.head, base + query);
            const int64_t where = (int64_t)t.token * a.q_heads + t.head;
            const bool none = l == 0.0f && m == kNoScore;
            const float inv = none ? 0.0f : 1.0f / l;
            *reinterpret_cast<u32x2*>(a.out + where * D + col) = u32x2{pack2(x[0] * inv, x[1] * inv), pack2(x[2] * inv, x[3] * inv)};
            if (a.lse && col == 0) a.lse[where] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * (float)kLn2;
        }
    }
}

template <int D, bool kFp8>
static hipError_t launch_window(const CacheView& c, const WindowArgs& a, const WindowShape& s, char* ws, hipStream_t stream)
{
    if ((int64_t)a.tokens * s.R / kTile + a.rows <= kOwnPlaces && s.steps < kOwnSteps && s.most_cost < kOwnCost) {
        window_kernel<D, kFp8, true><<<s.workgroups, 64 * kWaves, 0, stream>>>(c, a, s, ws);
    } else {
        window_plan_kernel<<<1, kPlanLanes, 0, stream>>>(a, s, c.heads, c.page_size, ws);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
        window_kernel<D, kFp8, false><<<s.workgroups, 64 * kWaves, 0, stream>>>(c, a, s, ws);
    }
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    // Queries of one workgroup of the join: 16 of a tile's; of a wave's item all, fewer where there are few workers, whose items have
    // many parts (one row 10.7 us with 8, 11.3 with 4, 11.1 with 1; 512 rows, 512 workgroups, 311 with 4, 303 with 1).
    const int group_shift = 3, wave_shift = s.workgroups * kPerUnit < compute_units() ? 3 : s.workgroups < compute_units() * kPerUnit ? 2 : 0;
    const int blocks = (s.workers[kOfGroups] << group_shift) + (s.workers[kOfWaves] << wave_shift);
    window_join_kernel<D><<<blocks, 256, 0, stream>>>(a, s, group_shift, wave_shift, ws);
    return hipGetLastError();
}

hipError_t launch_window_attention(const CacheView& c, const WindowArgs& a, void* workspace, hipStream_t stream)
{
    WindowShape s;
    const int64_t table = (int64_t)a.row_width * c.page_size, band = (int64_t)a.window + a.sinks + a.tokens;
    if (!window_shape(a.rows, a.tokens, a.q_heads, c.heads, c.dim, table < band ? table : band, s)) return hipErrorInvalidValue;
    char* ws = static_cast<char*>(workspace);
    if (c.dim == 128) return c.fp8 ? launch_window<128, true>(c, a, s, ws, stream) : launch_window<128, false>(c, a, s, ws, stream);
    return c.fp8 ? launch_window<64, true>(c, a, s, ws, stream) : launch_window<64, false>(c, a, s, ws, stream);
}

}  // namespace e3
