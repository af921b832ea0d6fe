// Verification of drafted tokens against the target's probabilities (speculative sampling), with the log-probabilities
// and entropies that a rollout needs of the tokens it keeps.
//
//   p_t = softmax(z_t / tau),  q_t = softmax(d_t / tau_d)  (or the point mass on the drafted token x_t)
//   draft t is accepted while u_t q_t(x_t) < p_t(x_t);  n = number accepted;
//   the next token is drawn from (p_n - q_n)+ / sum (p_n - q_n)+ after a rejection, from p_n after the last draft.
// Accepting with probability min(1, p/q) and drawing the rest from (p - q)+ gives a token distributed as p, whatever q is.
// The draw is the library's two-level race (e3_sample_entropy), with r_i = (p_i - q_i)+ in the place of exp(a_i): a tile's
// mass over its exponential variate, then a column's; Philox streams 5 (u_t, index t), 6 (tiles), 7 (columns).
//
// A position's logits ("line") have to be read once for their sums and, where the draw falls to it, once more: r_i needs
// both normalisers.  Two ways through:
//   pairs    enough positions to fill the card: a workgroup per (row, position) takes the sums of both lines, decides
//            its own draft and, when that is rejected (or the position is the one behind the last draft), races at once,
//            while the lines are still in the caches.  A position behind a known rejection is not read: rejections are
//            published per row, positions of all rows are started in order.  What is skipped never matters to
//            the result, so the result does not depend on timing.
//   slices   few positions: every line is cut into runs of columns, each summed by a workgroup of its own; a second
//            launch merges, decides and races over slices of the one position that draws.
// Either way a last launch, a workgroup per row, draws within the winning tile and writes the outputs.  (Done by the workgroup of
// a row that ends last instead, which takes a fence over the card's caches in every workgroup, 512 x 4 drafts took 558
// us where they take 237.)
//
// What bounds it: what passes between the caches and memory for many positions (512 rows x 4 drafts of 151,936 bf16 columns 237 us; the
// positions behind a rejection left out, 0.95 GB of 1.4, and the drawn lines read once more), chains of dependent loads for few: three launches of
// 6.6, 5.8 and 3.7 us for 4 rows x 3 drafts.
#include "verify.h"
#include "vocab_common.h"
#include "vocab_pass.h"

namespace e3 {

constexpr int kVerifyWaves = 4;
constexpr int kVerifyThreads = 64 * kVerifyWaves;
constexpr int kBlockSweeps = 4;                                   // sweeps of 512 columns that a wave has in flight
constexpr int kMaxSlices = 64;

struct alignas(16) LineSum {                                      // of a run of columns
    double S, W;                                                  // sum 2^t, sum t 2^t without the excluded maximum, t = z c - rc
    float rc, top;
    float pad[2];
};
struct alignas(16) Line {                                         // of a whole line
    double l1p;                                                   // ln sum exp(a_i - a_peak)
    float peak, entropy;
};

struct VerifyShape {
    int lines;                                                    // per row: drafts + 1 targets, then the drafts' own
    int slices;                                                   // 0: pairs
    int slice_cols;                                               // columns of a slice of sums (a multiple of 2048)
    int race_slices;                                              // slices of super-tiles
    int64_t at_lines, at_sums, at_cands, at_flags, bytes;        // at_flags: first rejected draft of each row
};

static int64_t up256(int64_t x) { return (x + 255) & ~(int64_t)255; }

static VerifyShape verify_shape(int64_t rows, int32_t drafts, int64_t V, bool drafter)
{
    VerifyShape s;
    const int64_t units = rows * (drafts + 1);
    s.lines = drafts + 1 + (drafter ? drafts : 0);
    const int cus = compute_units();
    const int64_t want = (int64_t)cus * 5;                        // workgroups that are resident together
    s.slices = 0;
    s.slice_cols = 0;
    s.race_slices = drafts + 1;
    // Slices below two positions per compute unit (64 x 7 of 32,000 columns take the same time either way, 128 x 4 of 151,936 110 us
    // as pairs and 122 as slices, 4 x 3 do not fill the card as pairs), and below twelve where lines are short, whose pairs are
    // mostly waiting (300 x 3 of 10,000: 38.0 as pairs, 32.9 as slices; 1000 x 1 of 1000: 40.1 and 28.7; but 512 x 1 of 32,000
    // 47.8 and 53.3).
    if (units < (int64_t)cus * (V <= 16384 ? 12 : 2)) {
        // a block of four sweeps for each wave at least
        const int64_t blocks = (V + 2047) / 2048;
        int64_t per = (blocks * rows * s.lines + want - 1) / want;
        per = (per + kVerifyWaves - 1) / kVerifyWaves * kVerifyWaves;
        if (per * kMaxSlices < blocks) per = (blocks + kMaxSlices - 1) / kMaxSlices;
        s.slice_cols = (int)(per * 2048);
        s.slices = (int)((blocks + per - 1) / per);
        const int64_t tiles = (V + kSuperCols - 1) / kSuperCols;
        int64_t race = (want + rows - 1) / rows;
        race = race < 1 ? 1 : race > kMaxSlices ? kMaxSlices : race;
        const int64_t each = (tiles + race - 1) / race;
        s.race_slices = (int)((tiles + each - 1) / each);
    }
    s.at_lines = 0;
    s.at_sums = up256(rows * s.lines * (int64_t)sizeof(Line));
    s.at_cands = up256(s.at_sums + rows * s.lines * s.slices * (int64_t)sizeof(LineSum));
    s.at_flags = up256(s.at_cands + rows * s.race_slices * (int64_t)sizeof(Cand));
    s.bytes = up256(s.at_flags + rows * 4);
    return s;
}

size_t verify_workspace_bytes(int64_t rows, int32_t drafts, int64_t V)
{
    const int64_t with = verify_shape(rows, drafts, V, true).bytes, without = verify_shape(rows, drafts, V, false).bytes;
    return (size_t)(with > without ? with : without);
}

// ---------------------------------------------------------------- sums of a line
// Columns of -inf are columns without weight: moved to the filler that drops out of every sum (NaN stays).
__device__ __forceinline__ void bounded(float z[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = __builtin_elementwise_maximum(z[j], kAbsent);
}

__device__ __forceinline__ LaneState empty_state()
{
    LaneState s;
    s.rc = s.top = s.thr = -INFINITY;
    s.dom_lane = 0;
    s.dom_open = false;
    s.S = s.W = s.sT0 = s.sT1 = s.wT0 = s.wT1 = 0.0f;
    s.best = Cand{-1.0f, 0};
    return s;
}

// Columns [from, to) of a line, dealt to `waves` waves in blocks of four sweeps.  `from` is a multiple of 512.
template <typename Chunk>
__device__ __forceinline__ void stream_sums(LaneState& s, const char* line, int64_t from, int64_t to, float c, int lane, int wave, int waves)
{
    const int sweeps = (int)((to - from) / kSweepCols);
    const int blocks = sweeps / kBlockSweeps;
    const int64_t at0 = from + Chunk::sweep_col(lane);
    auto add = [&](const Chunk& ch) {
        float z[8];
        ch.unpack(z);                                             // which lane holds which columns does not matter here
        bounded(z);
        accumulate_chunk(s, z, c, lane);
    };
    Chunk buf[kBlockSweeps];
    int b = wave;
    if (b < blocks) {
#pragma unroll
        for (int i = 0; i < kBlockSweeps; ++i) buf[i].load_sweep(line, at0 + ((int64_t)b * kBlockSweeps + i) * kSweepCols);
    }
    for (; b < blocks; b += waves) {
        const int next = b + waves < blocks ? b + waves : b;           // the last one again: no branch
#pragma unroll
        for (int i = 0; i < kBlockSweeps; ++i) {
            const Chunk cur = buf[i];
            buf[i].load_sweep(line, at0 + ((int64_t)next * kBlockSweeps + i) * kSweepCols);
            add(cur);
        }
        close_tile<false>(s, 0, 0.0f, true, c, lane);
    }
    // sweeps behind the last block, one wave each; then the columns behind the last sweep
    const int left = sweeps - blocks * kBlockSweeps;
    for (int i = 0; i < left; ++i) {
        if ((blocks + i) % waves != wave) continue;        // uniform
        Chunk ch;
        ch.load_sweep(line, at0 + ((int64_t)blocks * kBlockSweeps + i) * kSweepCols);
        add(ch);
        close_tile<false>(s, 0, 0.0f, true, c, lane);
    }
    if (from + (int64_t)sweeps * kSweepCols < to && (blocks + left) % waves == wave) {
        const int64_t col = from + (int64_t)sweeps * kSweepCols + lane * kChunk;
        float z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = kAbsent;
        if (col + kChunk <= to) {
            Chunk ch;
            ch.load(line, col);
            ch.unpack(z);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < to) z[j] = Chunk::load_one(line, col + j);
        }
        bounded(z);
        accumulate_chunk(s, z, c, lane);
        close_tile<false>(s, 0, 0.0f, true, c, lane);
    }
}

__device__ __forceinline__ LineSum wave_sums(const LaneState& s)
{
    double S = (double)s.S, W = (double)s.W;
    wave_sum2(S, W);
    // Nothing but the filler: its product with c is rounded by so much that the sums are no numbers or infinite.
    // They stand for nothing, unless a column was NaN.
    if (!(s.top > -INFINITY)) {
        S = nothing_left(S);
        return LineSum{S, S, -INFINITY, -INFINITY, {0.0f, 0.0f}};
    }
    return LineSum{S, W, s.rc, s.top, {0.0f, 0.0f}};
}

// Merge sums of disjoint columns, one per lane (n <= 64); uniform result.
__device__ __forceinline__ LineSum merge_sums(const LineSum* parts, int n, float c, int lane)
{
    LineSum p{0.0, 0.0, -INFINITY, -INFINITY, {0.0f, 0.0f}};
    if (lane < n) p = parts[lane];
    float R = p.rc, peak = p.top;
    wave_max2(R, peak);
    const unsigned long long holders = __ballot(p.top == peak);
    const int keep = (int)__builtin_ctzll(holders | (1ull << 63));
    const double cd = (double)c;
    double S = p.S, W = p.W;                                      // 0, or NaN, where there was nothing
    if (p.rc > -INFINITY) {
        const double d = (double)p.rc - (double)R;                // <= 0, an integer
        const double f = d > -1000.0 ? (double)__builtin_amdgcn_ldexp(1.0, (int)d) : 0.0;
        S = f > 0.0 ? p.S * f : nothing_left(p.S);
        W = f > 0.0 ? fma(d, p.S, p.W) * f : nothing_left(p.W);
        if (lane != keep && p.top > -INFINITY) {                  // an excluded maximum that is not the line's
            const double t = (double)p.top * cd - (double)R;
            const double e = t > -1000.0 ? exp2(t) : 0.0;
            S += e;
            W = fma(t > -1000.0 ? t : 0.0, e, W);
        }
    }
    wave_sum2(S, W);
    return LineSum{S, W, R, peak, {0.0f, 0.0f}};
}

// With e_p = 2^{t_p} the peak's term, x = S / e_p and y = W / e_p:
//   ln sum = t_p ln2 + log1p(x),   H = log1p(x) + ln2 (t_p x - y) / (1 + x).
__device__ __forceinline__ Line line_of(const LineSum& m, float c)
{
    const double t_p = (double)m.top * (double)c - (double)m.rc;
    const double inv = exp2(-t_p);
    const double x = m.S * inv, y = m.W * inv;
    Line r;
    r.l1p = log1p_of(x);
    r.peak = m.top;
    r.entropy = (float)fma(kLn2 * (t_p * x - y), reciprocal(1.0 + x), r.l1p);
    if (!(m.top > -INFINITY)) {                                   // nothing above the filler: no distribution
        r.l1p = __builtin_nan("");
        r.entropy = __builtin_nanf("");
    }
    return r;
}

template <typename Chunk>
__device__ __forceinline__ const char* target_line(const VerifyArgs& a, int64_t row, int t)
{
    return static_cast<const char*>(a.logits) + (row * a.row_stride + t * a.position_stride) * Chunk::kElemBytes;
}
template <typename Chunk>
__device__ __forceinline__ const char* draft_line(const VerifyArgs& a, int64_t row, int t)
{
    return static_cast<const char*>(a.draft_logits) + (row * a.draft_row_stride + t * a.draft_position_stride) * Chunk::kElemBytes;
}
// log2(e) / tau; no number for a temperature that is none
__device__ __forceinline__ float factor_of(float tau) { return tau > 0.0f ? kLog2eF / tau : __builtin_nanf(""); }
__device__ __forceinline__ float target_factor(const VerifyArgs& a, int64_t row)
{
    return factor_of(a.tau_rows ? a.tau_rows[row] : a.tau_scalar);
}
__device__ __forceinline__ float draft_factor(const VerifyArgs& a, int64_t row)
{
    return a.draft_tau_rows ? factor_of(a.draft_tau_rows[row]) : target_factor(a, row);
}
__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int64_t row)
{
    if (a.draft_lens == nullptr) return a.drafts;
    const int n = a.draft_lens[row];
    return n < 0 ? 0 : n > a.drafts ? a.drafts : n;
}
__device__ __forceinline__ int64_t draft_token(const VerifyArgs& a, int64_t row, int t)
{
    return t < a.drafts ? (int64_t)a.draft_tokens[row * a.drafts + t] : -1;
}
__device__ __forceinline__ double log_p(float z, const Line& line, float c)
{
    return ((double)z - (double)line.peak) * (double)c * kLn2 - line.l1p;
}

// What a draft's decision needs besides its lines; asked for before the lines are summed.
struct Drafted {
    int64_t x;
    float zp, zq;
    double u;
};
template <typename Chunk>
__device__ __forceinline__ Drafted drafted_at(const VerifyArgs& a, int64_t row, int t)
{
    Drafted d;
    d.x = draft_token(a, row, t);
    const int64_t safe = d.x < 0 ? 0 : d.x >= a.V ? a.V - 1 : d.x;
    d.zp = Chunk::load_one(target_line<Chunk>(a, row, t), safe);
    d.zq = a.draft_logits ? Chunk::load_one(draft_line<Chunk>(a, row, t), safe) : 0.0f;
    const uint64_t grow = a.row_base + (uint64_t)row;
    uint32_t w[4];
    philox4x32_10((uint32_t)t >> 2, (uint32_t)grow, (uint32_t)(grow >> 32), 5u, (uint32_t)a.seed, (uint32_t)(a.seed >> 32), w);
    const uint32_t word = (t & 3) == 0 ? w[0] : (t & 3) == 1 ? w[1] : (t & 3) == 2 ? w[2] : w[3];
    d.u = ((double)(word >> 9) + 0.5) * 0x1p-23;
    return d;
}
// u_t q_t(x_t) < p_t(x_t).  An id outside the vocabulary, or lines that are no distribution: rejected.
__device__ __forceinline__ bool accepts(const VerifyArgs& a, int64_t row, const Drafted& d, const Line& p, const Line& q)
{
    if (d.x < 0 || d.x >= a.V) return false;
    const double px = exp(log_p(d.zp, p, target_factor(a, row)));
    const double qx = a.draft_logits ? exp(log_p(d.zq, q, draft_factor(a, row))) : 1.0;
    return d.u * qx < px;
}

// ---------------------------------------------------------------- race
// What a draw is made from: r_i = (p_i - q_i)+, p_i = wp 2^{(z_i - zp) cp}; q_i alike, or none; or none but at one column.
struct Residual {
    const char *p, *q;                // q: nullptr without a draft distribution
    float cp, cq, zp, zq, wp, wq;
    int32_t barred;                   // a column that cannot be drawn, -1: none
};

__device__ __forceinline__ float weight_of(const Residual& r, float zp, float zq, bool with_q)
{
    const float p = __builtin_amdgcn_exp2f((zp - r.zp) * r.cp) * r.wp;
    if (!with_q) return p;
    // both products rounded: fused with the difference, one of them would leave its rounding behind where p = q
    const float q = __builtin_amdgcn_exp2f((zq - r.zq) * r.cq) * r.wq;
    return fmaxf(p - q, 0.0f);
}

// The lane's share of a tile's mass: sweeps first, first + 1, ... of super-tile st, `sweeps` (one or four) of them, all requested before
// the first is used.  Complete super-tiles are read in whole sweeps, which leave tile lane `slot` with the lane.
template <typename Chunk, bool kQ, int kSweeps>
__device__ __forceinline__ float tile_mass(const VerifyArgs& a, const Residual& r, int st, int sweep, int lane)
{
    const int64_t V = a.V;
    const bool whole = (int64_t)(st + 1) * kSuperCols <= V;       // uniform
    const int64_t first = (int64_t)st * kSuperCols + (int64_t)sweep * kSweepCols;
    const int slot = whole ? Chunk::tile_lane(lane) : lane;
    float mass = 0.0f;
    auto add = [&](const float* zp, const float* zq, int64_t col) {
        // (after the exchange of a complete sweep of fp32 an odd lane holds the upper four of its columns first)
        const int at = (int)(r.barred - col) ^ (whole && Chunk::kHalves == 2 && (lane & 1) ? 4 : 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float w = weight_of(r, zp[j], kQ ? zq[j] : 0.0f, kQ);
            mass += (!kQ && j == at) ? 0.0f : w;
        }
    };
    if (whole) {
        Chunk bp[kSweeps], bq[kSweeps];
#pragma unroll
        for (int i = 0; i < kSweeps; ++i) {
            bp[i].load_sweep(r.p, first + i * kSweepCols + Chunk::sweep_col(lane));
            if (kQ) bq[i].load_sweep(r.q, first + i * kSweepCols + Chunk::sweep_col(lane));
        }
#pragma unroll
        for (int i = 0; i < kSweeps; ++i) {
            float zp[8], zq[8];
            bp[i].unpack_sweep(zp, lane);
            if (kQ) bq[i].unpack_sweep(zq, lane);
            add(zp, zq, first + i * kSweepCols + slot * kChunk);
        }
    } else {
#pragma unroll 1
        for (int i = 0; i < kSweeps; ++i) {
            const int64_t col = first + i * kSweepCols + lane * kChunk;
            float zp[8], zq[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) { zp[j] = -INFINITY; zq[j] = -INFINITY; }
            if (col + kChunk <= V) {
                Chunk ch;
                ch.load(r.p, col);
                ch.unpack(zp);
                if (kQ) { ch.load(r.q, col); ch.unpack(zq); }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (col + j < V) { zp[j] = Chunk::load_one(r.p, col + j); if (kQ) zq[j] = Chunk::load_one(r.q, col + j); }
            }
            add(zp, zq, col);
        }
    }
    return mass;
}

// The lane's tile of super-tile st in the race of level 1.
template <typename Chunk>
__device__ __forceinline__ Cand tile_entry(const VerifyArgs& a, int64_t row, int st, float mass, int lane)
{
    const bool whole = (int64_t)(st + 1) * kSuperCols <= a.V;
    const int tile = st * kLanes + (whole ? Chunk::tile_lane(lane) : lane);
    const uint64_t grow = a.row_base + (uint64_t)row;
    uint32_t w[4];
    philox4x32_10((uint32_t)tile >> 2, (uint32_t)grow, (uint32_t)(grow >> 32), 6u, (uint32_t)a.seed, (uint32_t)(a.seed >> 32), w);
    const uint32_t word = (tile & 3) == 0 ? w[0] : (tile & 3) == 1 ? w[1] : (tile & 3) == 2 ? w[2] : w[3];
    return Cand{mass > 0.0f ? mass * inv_exp_variate(word) : -1.0f, tile};
}

// Level 1 over super-tiles [from, to), dealt to the waves: the wave's best tile.  kQ: with a draft distribution.
template <typename Chunk, bool kQ>
__device__ __forceinline__ Cand stream_race(const VerifyArgs& a, const Residual& r, int64_t row, int from, int to, int lane, int wave, int waves)
{
    Cand best{-1.0f, 0};
    for (int st = from + wave; st < to; st += waves) {
        float mass = 0.0f;
#pragma unroll 1
        for (int half = 0; half < kDepth; half += kBlockSweeps) mass += tile_mass<Chunk, kQ, kBlockSweeps>(a, r, st, half, lane);
        best = better(best, tile_entry<Chunk>(a, row, st, mass, lane));
    }
    return wave_best(best);
}

// The same with each of eight waves taking one sweep of every super-tile, where there are fewer super-tiles than waves.
template <typename Chunk, bool kQ>
__device__ __forceinline__ Cand share_race(const VerifyArgs& a, const Residual& r, int64_t row, int from, int to, float (*masses)[kLanes],
                                           int lane, int wave)
{
    static_assert(kDepth == 8, "one sweep for each of eight waves");
    Cand best{-1.0f, 0};
    for (int st = from; st < to; ++st) {
        __syncthreads();                                          // the last super-tile's are read
        masses[wave][lane] = tile_mass<Chunk, kQ, 1>(a, r, st, wave, lane);
        __syncthreads();
        if (wave != (st & 7)) continue;
        float mass = 0.0f;
#pragma unroll
        for (int i = 0; i < kDepth; ++i) mass += masses[i][lane];
        best = better(best, tile_entry<Chunk>(a, row, st, mass, lane));
    }
    return wave_best(best);
}

// Level 2: the column of tile `tile` (sixteen lanes x four columns); uniform.  -1: no column has weight.
template <typename Chunk>
__device__ __forceinline__ int32_t race_in_tile(const VerifyArgs& a, const Residual& r, int64_t row, int tile, int lane)
{
    const int64_t V = a.V;
    const int st = tile / kLanes, slot = tile % kLanes;
    const int64_t col = (int64_t)st * kSuperCols + (int64_t)(lane >> 1) * kSweepCols + slot * kChunk + (lane & 1) * 4;
    const bool in = lane < 2 * kDepth && col < V;
    float zp[4], zq[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    Chunk::unpack_four(Chunk::load_four(r.p, in ? col : 0), zp);
    if (r.q) Chunk::unpack_four(Chunk::load_four(r.q, in ? col : 0), zq);
    const uint64_t grow = a.row_base + (uint64_t)row;
    uint32_t w[4];
    philox4x32_10((uint32_t)(col >> 2), (uint32_t)grow, (uint32_t)(grow >> 32), 7u, (uint32_t)a.seed, (uint32_t)(a.seed >> 32), w);
    Cand best{-1.0f, 0x7FFFFFFF};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (!in || col + j >= V || col + j == r.barred) continue;
        const float weight = weight_of(r, zp[j], zq[j], r.q != nullptr);
        const Cand mine{weight > 0.0f ? weight * inv_exp_variate(w[j]) : -1.0f, (int)col + j};
        if (mine.q > best.q) best = mine;
    }
    const Cand win = row16_best(best);
    return win.q > 0.0f ? win.idx : -1;
}

template <typename Chunk>
__device__ __forceinline__ Residual residual_of(const VerifyArgs& a, int64_t row, int t, bool cut, const Line& p, const Line& q)
{
    Residual r;
    r.p = target_line<Chunk>(a, row, t);
    r.cp = target_factor(a, row);
    r.zp = p.peak;
    r.wp = (float)exp(-p.l1p);
    const bool with = cut && a.draft_logits != nullptr;
    r.q = with ? draft_line<Chunk>(a, row, t) : nullptr;
    r.cq = with ? draft_factor(a, row) : 0.0f;
    r.zq = with ? q.peak : 0.0f;
    r.wq = with ? (float)exp(-q.l1p) : 0.0f;
    const int64_t x = cut && !with ? draft_token(a, row, t) : -1;
    r.barred = x >= 0 && x < a.V ? (int32_t)x : -1;
    return r;
}

template <typename Chunk>
__device__ __forceinline__ Cand race(const VerifyArgs& a, const Residual& r, int64_t row, int from, int to, int lane, int wave, int waves)
{
    return r.q ? stream_race<Chunk, true>(a, r, row, from, to, lane, wave, waves)
               : stream_race<Chunk, false>(a, r, row, from, to, lane, wave, waves);
}

// the workgroup's best of the waves' candidates, in every thread
__device__ __forceinline__ Cand workgroup_best(Cand c, Cand* lds, int lane, int wave, int waves)
{
    __syncthreads();
    if (lane == 0) lds[wave] = c;
    __syncthreads();
    Cand best = lds[0];
    for (int i = 1; i < waves; ++i) best = better(best, lds[i]);
    return best;
}

// ---------------------------------------------------------------- kernels
__global__ __launch_bounds__(256)
void verify_clear_kernel(int32_t* flags, int64_t rows)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < rows) flags[i] = 0x7FFFFFFF;
}

// A workgroup per (position, row), positions rising.  Four of its eight waves take the sums of the target's line, four the
// draft's; all of them the one line where there is no other.  (One line after the other by four waves
// before: 512 x 4 drafts of 151,936 columns 301 us, now 240; 64 x 7 of 32,000 38, now 34.)
constexpr int kPairWaves = 8;
// LDS that is asked for and not used: two workgroups per compute unit, not three.  Their loads fill the memory's bandwidth as
// well, and a third would start positions sooner whose row turns out to be rejected before them (512 x 4 drafts: 264 us with three).
constexpr int kPairLds = 56 * 1024;

template <typename Chunk>
__global__ __launch_bounds__(64 * kPairWaves, 4)
void verify_pair_kernel(VerifyArgs a, VerifyShape s, char* ws)
{
    __shared__ LineSum sums[kPairWaves];
    __shared__ Line found[2];
    __shared__ Cand cands[kPairWaves];
    __shared__ int known;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = (int)(blockIdx.x / a.rows);
    const int64_t row = blockIdx.x % a.rows;
    int32_t* flags = reinterpret_cast<int32_t*>(ws + s.at_flags);
    const int len = drafts_of(a, row);
    if (t > len) return;
    Line* lines = reinterpret_cast<Line*>(ws + s.at_lines) + row * s.lines;
    if (threadIdx.x == 0) known = t > 0 ? __hip_atomic_load(&flags[row], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0x7FFFFFFF;
    const bool last = t == len, two = !last && a.draft_logits != nullptr;
    Drafted d{};
    if (!last) d = drafted_at<Chunk>(a, row, t);
    __syncthreads();
    if (known < t) return;                                        // an earlier draft was rejected
    const int half = two ? kPairWaves / 2 : kPairWaves;           // waves of a line
    const int which = wave >= half ? 1 : 0;
    const char* line = which ? draft_line<Chunk>(a, row, t) : target_line<Chunk>(a, row, t);
    const float c = which ? draft_factor(a, row) : target_factor(a, row);
    LaneState state = empty_state();
    stream_sums<Chunk>(state, line, 0, a.V, c, lane, wave - which * half, half);
    const LineSum mine = wave_sums(state);
    if (lane == 0) sums[wave] = mine;
    __syncthreads();
    if (wave == which * half) {
        const Line l = line_of(merge_sums(sums + which * half, half, c, lane), c);
        if (lane == 0) {
            found[which] = l;
            lines[(which ? a.drafts + 1 : 0) + t] = l;
        }
    }
    __syncthreads();
    const Line p = found[0], q = found[two ? 1 : 0];
    if (!last) {
        if (accepts(a, row, d, p, q)) return;                     // the same in every thread
        if (threadIdx.x == 0) atomicMin(&flags[row], t);
    }
    const Residual r = residual_of<Chunk>(a, row, t, !last, p, q);
    const int tiles = (int)((a.V + kSuperCols - 1) / kSuperCols);
    const Cand best = workgroup_best(race<Chunk>(a, r, row, 0, tiles, lane, wave, kPairWaves), cands, lane, wave, kPairWaves);
    if (threadIdx.x == 0) reinterpret_cast<Cand*>(ws + s.at_cands)[row * s.race_slices + t] = best;
}

// A workgroup per (row, line, slice).
template <typename Chunk>
__global__ __launch_bounds__(kVerifyThreads)
void verify_sums_kernel(VerifyArgs a, VerifyShape s, char* ws)
{
    __shared__ LineSum sums[kVerifyWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int slice = blockIdx.x % s.slices, line = blockIdx.x / s.slices % s.lines;
    const int64_t row = blockIdx.x / s.slices / s.lines;
    const bool target = line <= a.drafts;
    const int t = target ? line : line - a.drafts - 1, len = drafts_of(a, row);
    if (target ? t > len : t >= len) return;
    const char* at = target ? target_line<Chunk>(a, row, t) : draft_line<Chunk>(a, row, t);
    const float c = target ? target_factor(a, row) : draft_factor(a, row);
    const int64_t from = (int64_t)slice * s.slice_cols;
    const int64_t to = from + s.slice_cols < a.V ? from + s.slice_cols : a.V;
    LaneState state = empty_state();
    stream_sums<Chunk>(state, at, from, to, c, lane, wave, kVerifyWaves);
    const LineSum mine = wave_sums(state);
    if (lane == 0) sums[wave] = mine;
    __syncthreads();
    if (wave == 0) {
        const LineSum m = merge_sums(sums, kVerifyWaves, c, lane);
        if (lane == 0) reinterpret_cast<LineSum*>(ws + s.at_sums)[(row * s.lines + line) * s.slices + slice] = m;
    }
}

// A workgroup per (row, slice of super-tiles): merges the row's lines, decides, races over its slice of the position that
// draws.  The first one of a row leaves the lines and the decision for the last launch.
constexpr int kRaceWaves = 8;

template <typename Chunk>
__global__ __launch_bounds__(64 * kRaceWaves)
void verify_race_kernel(VerifyArgs a, VerifyShape s, char* ws)
{
    __shared__ Line lines[2 * kMaxDrafts + 1];
    __shared__ Cand cands[kRaceWaves];
    __shared__ float masses[kRaceWaves][kLanes];
    __shared__ int rejected;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int slice = blockIdx.x % s.race_slices;
    const int64_t row = blockIdx.x / s.race_slices;
    const int len = drafts_of(a, row);
    const LineSum* sums = reinterpret_cast<const LineSum*>(ws + s.at_sums) + row * s.lines * s.slices;
    if (threadIdx.x == 0) rejected = len;
    Drafted d{};
    if (wave == 0 && lane < len) d = drafted_at<Chunk>(a, row, lane);
    for (int i = wave; i < s.lines; i += kRaceWaves) {
        const bool target = i <= a.drafts;
        if (target ? i > len : i - a.drafts - 1 >= len) continue;
        const float c = target ? target_factor(a, row) : draft_factor(a, row);
        const Line l = line_of(merge_sums(sums + i * s.slices, s.slices, c, lane), c);
        if (lane == 0) {
            lines[i] = l;
            if (slice == 0) (reinterpret_cast<Line*>(ws + s.at_lines) + row * s.lines)[i] = l;
        }
    }
    __syncthreads();
    if (wave == 0) {
        const bool no = lane < len && !accepts(a, row, d, lines[lane], lines[a.draft_logits ? a.drafts + 1 + lane : lane]);
        const unsigned long long m = __ballot(no);
        if (lane == 0 && m != 0ull) rejected = (int)__builtin_ctzll(m);
    }
    __syncthreads();
    const int n = rejected;
    const bool cut = n < len;
    if (slice == 0 && threadIdx.x == 0) reinterpret_cast<int32_t*>(ws + s.at_flags)[row] = n;
    const Residual r = residual_of<Chunk>(a, row, n, cut, lines[n], lines[cut && a.draft_logits ? a.drafts + 1 + n : n]);
    const int tiles = (int)((a.V + kSuperCols - 1) / kSuperCols);
    const int each = (tiles + s.race_slices - 1) / s.race_slices;
    const int from = slice * each, to = from + each < tiles ? from + each : tiles;
    Cand best = each >= kRaceWaves ? race<Chunk>(a, r, row, from, to, lane, wave, kRaceWaves)
              : r.q ? share_race<Chunk, true>(a, r, row, from, to, masses, lane, wave) : share_race<Chunk, false>(a, r, row, from, to, masses, lane, wave);
    best = workgroup_best(best, cands, lane, wave, kRaceWaves);
    if (threadIdx.x == 0) reinterpret_cast<Cand*>(ws + s.at_cands)[row * s.race_slices + slice] = best;
}

// A workgroup per row: the draw's second level, ids, log-probs and entropies.
template <typename Chunk>
__global__ __launch_bounds__(kVerifyThreads)
void verify_finish_kernel(VerifyArgs a, VerifyShape s, const char* ws)
{
    __shared__ Cand cands[kVerifyWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x;
    const int len = drafts_of(a, row);
    const Line* lines = reinterpret_cast<const Line*>(ws + s.at_lines) + row * s.lines;
    const int first = reinterpret_cast<const int32_t*>(ws + s.at_flags)[row];          // rejected draft
    const int n = first < len ? first : len;
    const bool cut = n < len;
    const Line p = lines[n];
    Residual r = residual_of<Chunk>(a, row, n, cut, p, lines[cut && a.draft_logits ? a.drafts + 1 + n : n]);
    const Cand* found = reinterpret_cast<const Cand*>(ws + s.at_cands) + row * s.race_slices;
    Cand best{-1.0f, 0};
    if (s.slices == 0) {
        best = found[n];
    } else {
        if (lane < s.race_slices) best = found[lane];             // at most 64
        best = wave_best(best);
    }
    int32_t token = best.q > 0.0f ? race_in_tile<Chunk>(a, r, row, best.idx, lane) : -1;
    if (token < 0 && cut) {
        // nothing is left where p > q (the two agree up to rounding, or q is no distribution): the draw is from p
        r.q = nullptr;
        r.barred = -1;
        const int tiles = (int)((a.V + kSuperCols - 1) / kSuperCols);
        best = workgroup_best(race<Chunk>(a, r, row, 0, tiles, lane, wave, kVerifyWaves), cands, lane, wave, kVerifyWaves);
        token = best.q > 0.0f ? race_in_tile<Chunk>(a, r, row, best.idx, lane) : -1;
    }
    if (token < 0) token = 0;                                     // p is no distribution
    if (wave != 0) return;
    if (lane == 0) a.accepted_out[row] = n;
    if (lane <= a.drafts) {
        const int64_t at = row * (a.drafts + 1) + lane;
        const int64_t x = lane < n ? draft_token(a, row, lane) : token;
        a.token_out[at] = lane <= n ? (int32_t)x : -1;
        float lp = 0.0f, h = 0.0f;
        if (lane <= n) {
            const Line l = lines[lane];
            lp = (float)log_p(Chunk::load_one(target_line<Chunk>(a, row, lane), x), l, target_factor(a, row));
            h = l.entropy;
        }
        if (a.logp_out) a.logp_out[at] = lp;
        if (a.entropy_out) a.entropy_out[at] = h;
    }
}

template <typename Chunk>
static hipError_t launch(const VerifyArgs& a, char* ws, hipStream_t stream)
{
    const VerifyShape s = verify_shape(a.rows, a.drafts, a.V, a.draft_logits != nullptr);
    if (s.slices == 0) {
        verify_clear_kernel<<<(uint32_t)((a.rows + 255) / 256), 256, 0, stream>>>(reinterpret_cast<int32_t*>(ws + s.at_flags), a.rows);
        if (const hipError_t err = hipGetLastError(); err != hipSuccess) return err;
        verify_pair_kernel<Chunk><<<(uint32_t)(a.rows * (a.drafts + 1)), 64 * kPairWaves, kPairLds, stream>>>(a, s, ws);
    } else {
        verify_sums_kernel<Chunk><<<(uint32_t)(a.rows * s.lines * s.slices), kVerifyThreads, 0, stream>>>(a, s, ws);
        if (const hipError_t err = hipGetLastError(); err != hipSuccess) return err;
        verify_race_kernel<Chunk><<<(uint32_t)(a.rows * s.race_slices), 64 * kRaceWaves, 0, stream>>>(a, s, ws);
    }
    if (const hipError_t err = hipGetLastError(); err != hipSuccess) return err;
    verify_finish_kernel<Chunk><<<(uint32_t)a.rows, kVerifyThreads, 0, stream>>>(a, s, ws);
    return hipGetLastError();
}

hipError_t launch_verify(const VerifyArgs& a, bool is_bf16, void* workspace, hipStream_t stream)
{
    char* ws = static_cast<char*>(workspace);
    return is_bf16 ? launch<ChunkBf16>(a, ws, stream) : launch<ChunkF32>(a, ws, stream);
}

}  // namespace e3
