// C ABI of the decode step: argument checks on the host, then kernel launches.
#include <hip/hip_runtime.h>
#include <cmath>
#include <cstdint>

#include "../../include/e3.h"
#include "beam.h"
#include "kv_cache.h"
#include "rotary.h"
#include "verify.h"
#include "vocab_pass.h"
#include "window_attention.h"

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_cache(const e3_cache* c, e3::CacheView* view)
{
    if (c == nullptr) return E3_ERR_NULL;
    if (c->dtype != E3_BF16 && c->dtype != E3_E4M3) return E3_ERR_DTYPE;
    if (c->num_pages < 1 || c->num_pages > 0x7FFFFFFF || c->kv_heads < 1 || c->kv_heads > 65536) return E3_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128) return E3_ERR_SHAPE;
    if (c->page_size < 32 || c->page_size > (1 << 20) || (c->page_size & (c->page_size - 1)) != 0) return E3_ERR_SHAPE;
    const bool fp8 = c->dtype == E3_E4M3;
    if (c->k == nullptr || c->v == nullptr || (fp8 && (c->k_scale == nullptr || c->v_scale == nullptr))) return E3_ERR_NULL;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || (fp8 && (!aligned(c->k_scale, 8) || !aligned(c->v_scale, 8)))) return E3_ERR_ALIGN;
    view->k = c->k; view->v = c->v; view->k_scale = c->k_scale; view->v_scale = c->v_scale;
    view->num_pages = c->num_pages; view->page_size = c->page_size; view->page_shift = __builtin_ctz((unsigned)c->page_size);
    view->heads = c->kv_heads; view->dim = c->head_dim; view->fp8 = fp8;
    return E3_OK;
}

constexpr int64_t kMostTokens = (int64_t)1 << 28;   // tokens x heads of one call: eight a wave, its threads below 2^32

}  // namespace

extern "C" int e3_cache_append(const e3_cache* cache, const void* k, const void* v, int dtype, int64_t tokens,
                               int64_t k_token_stride, int64_t k_head_stride,
                               int64_t v_token_stride, int64_t v_head_stride,
                               const int64_t* slots, void* hip_stream)
{
    e3::CacheView view;
    const int rc = check_cache(cache, &view);
    if (rc != E3_OK) return rc;
    if (dtype != E3_F32 && dtype != E3_BF16) return E3_ERR_DTYPE;
    if (tokens < 0 || tokens > kMostTokens || tokens * view.heads > kMostTokens) return E3_ERR_SHAPE;
    if (tokens == 0) return E3_OK;
    if (k == nullptr || v == nullptr || slots == nullptr) return E3_ERR_NULL;
    const int64_t per = dtype == E3_F32 ? 4 : 8;                    // elements in 16 bytes
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8) || k_token_stride % per || k_head_stride % per ||
        v_token_stride % per || v_head_stride % per)
        return E3_ERR_ALIGN;
    const hipError_t err = e3::launch_cache_append(view, {k, k_token_stride, k_head_stride}, {v, v_token_stride, v_head_stride},
                                                   dtype == E3_BF16, slots, tokens, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? E3_OK : E3_ERR_LAUNCH;
}

extern "C" int e3_cache_read(const e3_cache* cache, const int64_t* slots, int64_t tokens,
                             void* k_out, void* v_out, int dtype, void* hip_stream)
{
    e3::CacheView view;
    const int rc = check_cache(cache, &view);
    if (rc != E3_OK) return rc;
    if (dtype != E3_F32 && dtype != E3_BF16) return E3_ERR_DTYPE;
    if (tokens < 0 || tokens > kMostTokens || tokens * view.heads > kMostTokens) return E3_ERR_SHAPE;
    if (tokens == 0) return E3_OK;
    if (k_out == nullptr || v_out == nullptr || slots == nullptr) return E3_ERR_NULL;
    if (!aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(slots, 8)) return E3_ERR_ALIGN;
    const hipError_t err = e3::launch_cache_read(view, slots, tokens, k_out, v_out, dtype == E3_BF16,
                                                 static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? E3_OK : E3_ERR_LAUNCH;
}

static int check_rotary(const e3_rotary* r, const int64_t* positions, int64_t position_stride, int64_t head_dim, e3::Rotary* view)
{
    if (r == nullptr) return E3_ERR_NULL;
    if (r->rot_dim < 16 || r->rot_dim % 16 || r->rot_dim > head_dim || r->axes < 1 || r->axes > E3_MAX_AXES) return E3_ERR_SHAPE;
    if (r->neighbours != 0 && r->neighbours != 1) return E3_ERR_VALUE;
    if (r->freqs == nullptr || (r->axis == nullptr && r->axes > 1)) return E3_ERR_NULL;
    if (!aligned(r->freqs, 8) || !aligned(positions, 8)) return E3_ERR_ALIGN;
    view->freqs = r->freqs; view->axis = r->axis; view->positions = positions; view->stride = position_stride;
    view->rot = r->rot_dim; view->axes = r->axes; view->neighbours = r->neighbours != 0; view->sign = 1.0f;
    return E3_OK;
}

constexpr int64_t kMostTurned = (int64_t)1 << 25;   // tokens of one call that turns: its threads stay below 2^32

extern "C" int e3_rotate(const e3_rotary* rotary, const int64_t* positions, int64_t position_stride, const void* x, int dtype,
                         int64_t tokens, int64_t heads, int64_t head_dim, int64_t x_token_stride, int64_t x_head_stride,
                         void* out, int64_t out_token_stride, int64_t out_head_stride, int inverse, void* hip_stream)
{
    e3::Rotary r;
    if (dtype != E3_F32 && dtype != E3_BF16) return E3_ERR_DTYPE;
    if (tokens < 0 || tokens > kMostTurned || heads < 0 || heads > 65536 || head_dim < 16 || head_dim > 1024 || head_dim % 8) return E3_ERR_SHAPE;
    const int rc = check_rotary(rotary, positions, position_stride, head_dim, &r);
    if (rc != E3_OK) return rc;
    if (inverse != 0 && inverse != 1) return E3_ERR_VALUE;
    if (tokens == 0 || heads == 0) return E3_OK;
    if (x == nullptr || out == nullptr || positions == nullptr) return E3_ERR_NULL;
    const int64_t per = dtype == E3_F32 ? 4 : 8;                    // elements in 16 bytes
    if (!aligned(x, 16) || !aligned(out, 16) || x_token_stride % per || x_head_stride % per || out_token_stride % per || out_head_stride % per)
        return E3_ERR_ALIGN;
    // in place: element for element, or a row would be read after another one's result is there
    if (x == out && ((tokens > 1 && x_token_stride != out_token_stride) || (heads > 1 && x_head_stride != out_head_stride))) return E3_ERR_VALUE;
    r.sign = inverse ? -1.0f : 1.0f;
    const e3::TurnArgs a{{x, x_token_stride, x_head_stride}, out, out_token_stride, out_head_stride, tokens, (int32_t)heads, (int32_t)head_dim};
    const hipError_t err = e3::launch_rotate(a, r, dtype == E3_BF16, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? E3_OK : E3_ERR_LAUNCH;
}

extern "C" int e3_cache_append_rotated(const e3_cache* cache, const e3_rotary* rotary, const int64_t* positions, int64_t position_stride,
                                       const void* q, const void* k, const void* v, int dtype, int64_t tokens, int64_t q_heads,
                                       int64_t q_token_stride, int64_t q_head_stride, int64_t k_token_stride, int64_t k_head_stride,
                                       int64_t v_token_stride, int64_t v_head_stride, const int64_t* slots,
                                       void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, void* hip_stream)
{
    e3::CacheView view;
    int rc = check_cache(cache, &view);
    if (rc != E3_OK) return rc;
    if (dtype != E3_F32 && dtype != E3_BF16) return E3_ERR_DTYPE;
    if (tokens < 0 || tokens > kMostTurned || tokens * view.heads > kMostTokens || q_heads < 0 || q_heads > 65536) return E3_ERR_SHAPE;
    e3::Rotary r;
    rc = check_rotary(rotary, positions, position_stride, view.dim, &r);
    if (rc != E3_OK) return rc;
    if (tokens == 0) return E3_OK;
    if (k == nullptr || v == nullptr || slots == nullptr || positions == nullptr || (q_heads > 0 && (q == nullptr || q_out == nullptr))) return E3_ERR_NULL;
    const int64_t per = dtype == E3_F32 ? 4 : 8;                    // elements in 16 bytes
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8) || k_token_stride % per || k_head_stride % per || v_token_stride % per ||
        v_head_stride % per)
        return E3_ERR_ALIGN;
    e3::TurnArgs a{};
    if (q_heads > 0) {
        if (!aligned(q, 16) || !aligned(q_out, 16) || q_token_stride % per || q_head_stride % per || q_out_token_stride % per || q_out_head_stride % per)
            return E3_ERR_ALIGN;
        if (q == q_out && ((tokens > 1 && q_token_stride != q_out_token_stride) || (q_heads > 1 && q_head_stride != q_out_head_stride)))
            return E3_ERR_VALUE;
        a = e3::TurnArgs{{q, q_token_stride, q_head_stride}, q_out, q_out_token_stride, q_out_head_stride, tokens, (int32_t)q_heads, view.dim};
    }
    const hipError_t err = e3::launch_cache_append_rotated(view, {k, k_token_stride, k_head_stride}, {v, v_token_stride, v_head_stride}, a, r,
                                                           dtype == E3_BF16, slots, tokens, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? E3_OK : E3_ERR_LAUNCH;
}

static bool attention_shape(int64_t rows, int64_t queries, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t num_groups)
{
    return rows >= 0 && rows <= (1 << 24) && queries >= 1 && queries <= (1 << 16) && kv_heads >= 1 && kv_heads <= 65536 && q_heads >= kv_heads &&
           q_heads <= (1 << 20) && q_heads % kv_heads == 0 && (head_dim == 64 || head_dim == 128) && num_groups >= 0 &&
           num_groups <= (1 << 24) && rows * queries * q_heads <= 0x7FFFFFFF;
}

extern "C" size_t e3_prefix_attention_workspace_bytes(int64_t rows, int64_t queries, int64_t q_heads, int64_t kv_heads,
                                                      int64_t head_dim, int64_t num_groups)
{
    if (rows == 0 || !attention_shape(rows, queries, q_heads, kv_heads, head_dim, num_groups)) return 0;
    return e3::prefix_attention_workspace_bytes(rows, queries, q_heads, kv_heads, head_dim, num_groups);
}

extern "C" int e3_prefix_attention(const e3_cache* cache, const void* q, int64_t rows, int64_t queries, int64_t q_heads,
                                   int64_t q_row_stride, int64_t q_token_stride, int64_t q_head_stride,
                                   const int32_t* group_offsets, int64_t num_groups,
                                   const int32_t* prefix_pages, int64_t prefix_width, const int32_t* prefix_lens,
                                   const int32_t* row_pages, int64_t row_width, const int32_t* row_lens,
                                   float scale, void* out, float* lse_out,
                                   void* workspace, size_t workspace_bytes, void* hip_stream)
{
    e3::CacheView view;
    const int rc = check_cache(cache, &view);
    if (rc != E3_OK) return rc;
    if (!attention_shape(rows, queries, q_heads, view.heads, view.dim, num_groups) || prefix_width < 0 || row_width < 0 ||
        prefix_width > 0x7FFFFFFF || row_width > 0x7FFFFFFF)
        return E3_ERR_SHAPE;
    if (!std::isfinite(scale) || !(scale > 0.0f)) return E3_ERR_VALUE;
    if (rows == 0) return E3_OK;
    const size_t need = e3::prefix_attention_workspace_bytes(rows, queries, q_heads, view.heads, view.dim, num_groups);
    if (need == 0) return E3_ERR_SHAPE;
    if (q == nullptr || out == nullptr || row_lens == nullptr || (row_pages == nullptr && row_width > 0)) return E3_ERR_NULL;
    if (num_groups > 0 && (group_offsets == nullptr || prefix_lens == nullptr || (prefix_pages == nullptr && prefix_width > 0)))
        return E3_ERR_NULL;
    if (workspace == nullptr || workspace_bytes < need) return E3_ERR_WORKSPACE;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256) || q_row_stride % 8 || q_token_stride % 8 || q_head_stride % 8)
        return E3_ERR_ALIGN;
    e3::AttentionArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.q_row_stride = q_row_stride; a.q_token_stride = q_token_stride; a.q_head_stride = q_head_stride;
    a.rows = (int32_t)rows; a.T = (int32_t)queries; a.q_heads = (int32_t)q_heads; a.groups = (int32_t)num_groups;
    a.group_offsets = group_offsets; a.prefix_pages = prefix_pages; a.prefix_lens = prefix_lens;
    a.row_pages = row_pages; a.row_lens = row_lens;
    a.prefix_width = (int32_t)prefix_width; a.row_width = (int32_t)row_width;
    a.scale = scale; a.out = static_cast<uint16_t*>(out); a.lse = lse_out;
    const hipError_t err = e3::launch_prefix_attention(view, a, workspace, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? E3_OK : E3_ERR_LAUNCH;
}

static bool window_dims(int64_t rows, int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t head_dim)
{
    return rows >= 0 && rows <= (1 << 24) && tokens >= 0 && tokens <= 0x7FFFFFFF && kv_heads >= 1 && kv_heads <= 65536 && q_heads >= kv_heads &&
           q_heads <= (1 << 20) && q_heads % kv_heads == 0 && (head_dim == 64 || head_dim == 128);
}

extern "C" size_t e3_window_attention_workspace_bytes(int64_t rows, int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t head_dim)
{
    if (rows == 0 || tokens == 0 || !window_dims(rows, tokens, q_heads, kv_heads, head_dim)) return 0;
    return e3::window_attention_workspace_bytes(rows, tokens, q_heads, kv_heads, head_dim);
}

extern "C" int e3_window_attention(const e3_cache* cache, const void* q, int64_t tokens, int64_t q_heads, int64_t q_token_stride,
                                   int64_t q_head_stride, const int32_t* query_offsets, int64_t rows,
                                   const int32_t* row_pages, int64_t row_width, const int32_t* row_lens,
                                   int64_t window, int64_t sinks, float scale, void* out, float* lse_out,
                                   void* workspace, size_t workspace_bytes, void* hip_stream)
{
    e3::CacheView view;
    const int rc = check_cache(cache, &view);
    if (rc != E3_OK) return rc;
    if (!window_dims(rows, tokens, q_heads, view.heads, view.dim) || row_width < 0 || row_width > 0x7FFFFFFF) return E3_ERR_SHAPE;
    if (!std::isfinite(scale) || !(scale > 0.0f) || window < 1 || sinks < 0) return E3_ERR_VALUE;
    if (rows == 0 || tokens == 0) return E3_OK;
    const size_t need = e3::window_attention_workspace_bytes(rows, tokens, q_heads, view.heads, view.dim);
    if (need == 0) return E3_ERR_SHAPE;
    if (q == nullptr || out == nullptr || query_offsets == nullptr || row_lens == nullptr || (row_pages == nullptr && row_width > 0)) return E3_ERR_NULL;
    if (workspace == nullptr || workspace_bytes < need) return E3_ERR_WORKSPACE;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256) || q_token_stride % 8 || q_head_stride % 8) return E3_ERR_ALIGN;
    constexpr int64_t kMost = 0x7F000000;                           // no sequence is longer
    e3::WindowArgs a{};
    a.q = static_cast<const uint16_t*>(q);
    a.q_token_stride = q_token_stride; a.q_head_stride = q_head_stride;
    a.tokens = (int32_t)tokens; a.rows = (int32_t)rows; a.q_heads = (int32_t)q_heads;
    a.offsets = query_offsets; a.row_pages = row_pages; a.row_lens = row_lens; a.row_width = (int32_t)row_width;
    a.window = (int32_t)(window < kMost ? window : kMost); a.sinks = (int32_t)(sinks < kMost ? sinks : kMost);
    a.scale = scale; a.out = static_cast<uint16_t*>(out); a.lse = lse_out;
    const hipError_t err = e3::launch_window_attention(view, a, workspace, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? E3_OK : E3_ERR_LAUNCH;
}

static bool verify_dims(int64_t rows, int32_t drafts, int64_t V)
{
    return rows >= 0 && drafts >= 0 && drafts <= E3_MAX_DRAFTS && V >= 1 && V <= 0x7FFFFFFF - 8192 && e3::vocab_pass_fits(V) &&
           rows * (drafts + 1) < 1 << 23;                            // workgroups of 512: threads below 2^32
}

extern "C" size_t e3_verify_workspace_bytes(int64_t rows, int32_t drafts, int64_t V)
{
    return rows > 0 && rows < 1 << 23 && verify_dims(rows, drafts, V) ? e3::verify_workspace_bytes(rows, drafts, V) : 0;
}

extern "C" int e3_verify_drafts(const void* logits, int dtype, int64_t rows, int32_t drafts, int64_t V,
                                int64_t row_stride, int64_t position_stride,
                                const int32_t* draft_tokens, const int32_t* draft_lens,
                                const void* draft_logits, int64_t draft_row_stride, int64_t draft_position_stride,
                                const float* tau_rows, float tau_scalar, const float* draft_tau_rows,
                                uint64_t seed, uint64_t row_base,
                                int32_t* accepted_out, int32_t* token_out, float* logp_out, float* entropy_out,
                                void* workspace, size_t workspace_bytes, void* hip_stream)
{
    static_assert(E3_MAX_DRAFTS == e3::kMaxDrafts, "one lane per position");
    if (dtype != E3_F32 && dtype != E3_BF16) return E3_ERR_DTYPE;
    if (rows >= 1 << 23 || !verify_dims(rows, drafts, V) || position_stride < V) return E3_ERR_SHAPE;
    if (draft_logits != nullptr && drafts > 0 && draft_position_stride < V) return E3_ERR_SHAPE;
    if (tau_rows == nullptr && !(std::isfinite(tau_scalar) && tau_scalar > 0.0f)) return E3_ERR_VALUE;
    if (rows == 0) return E3_OK;
    if (logits == nullptr || accepted_out == nullptr || token_out == nullptr || (draft_tokens == nullptr && drafts > 0)) return E3_ERR_NULL;
    const size_t need = e3::verify_workspace_bytes(rows, drafts, V);
    if (workspace == nullptr || workspace_bytes < need) return E3_ERR_WORKSPACE;
    const int64_t per = dtype == E3_F32 ? 4 : 8;                    // elements in 16 bytes
    if (!aligned(logits, 16) || !aligned(draft_logits, 16) || !aligned(workspace, 256) || row_stride % per || position_stride % per ||
        draft_row_stride % per || draft_position_stride % per)
        return E3_ERR_ALIGN;
    e3::VerifyArgs a{};
    a.logits = logits; a.draft_logits = drafts > 0 ? draft_logits : nullptr;
    a.rows = rows; a.V = V; a.row_stride = row_stride; a.position_stride = position_stride;
    a.draft_row_stride = draft_row_stride; a.draft_position_stride = draft_position_stride;
    a.drafts = drafts; a.draft_tokens = draft_tokens; a.draft_lens = draft_lens;
    a.tau_rows = tau_rows; a.tau_scalar = tau_scalar; a.draft_tau_rows = draft_tau_rows;
    a.seed = seed; a.row_base = row_base;
    a.accepted_out = accepted_out; a.token_out = token_out; a.logp_out = logp_out; a.entropy_out = entropy_out;
    const hipError_t err = e3::launch_verify(a, dtype == E3_BF16, workspace, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? E3_OK : E3_ERR_LAUNCH;
}

static bool beam_dims(int64_t seqs, int32_t beams, int64_t V)
{
    return seqs >= 0 && seqs < 1 << 24 && beams >= 1 && beams <= E3_MAX_BEAMS && V >= 1 && V <= 1040384;
}

extern "C" size_t e3_beam_workspace_bytes(int64_t seqs, int32_t beams, int64_t V)
{
    return seqs > 0 && beam_dims(seqs, beams, V) ? e3::beam_workspace_bytes(seqs, beams, V) : 0;
}

extern "C" int e3_beam_select(const void* logits, int dtype, int64_t seqs, int32_t beams, int64_t V, int64_t seq_stride, int64_t beam_stride,
                              const float* scores, int32_t keep, float tau, const uint8_t* finished, int32_t eos_token,
                              int32_t* parent_out, int32_t* token_out, float* score_out,
                              void* workspace, size_t workspace_bytes, void* hip_stream)
{
    static_assert(E3_MAX_BEAMS == e3::kMaxBeams && E3_MAX_KEEP == e3::kMaxKeep, "one lane per kept candidate");
    if (dtype != E3_F32 && dtype != E3_BF16) return E3_ERR_DTYPE;
    if (!beam_dims(seqs, beams, V) || keep < 1 || keep > E3_MAX_KEEP || beam_stride < V) return E3_ERR_SHAPE;
    if (!(std::isfinite(tau) && tau > 0.0f) || (finished != nullptr && (eos_token < 0 || eos_token >= V))) return E3_ERR_VALUE;
    if (seqs == 0) return E3_OK;
    const size_t need = e3::beam_workspace_bytes(seqs, beams, V);
    if (need == 0) return E3_ERR_SHAPE;
    if (logits == nullptr || scores == nullptr || parent_out == nullptr || token_out == nullptr || score_out == nullptr) return E3_ERR_NULL;
    if (workspace == nullptr || workspace_bytes < need) return E3_ERR_WORKSPACE;
    const int64_t per = dtype == E3_F32 ? 4 : 8;                    // elements in 16 bytes
    if (!aligned(logits, 16) || !aligned(workspace, 256) || seq_stride % per || beam_stride % per) return E3_ERR_ALIGN;
    const e3::BeamArgs a{logits, seqs, V, seq_stride, beam_stride, beams, keep, scores, finished, eos_token, tau, parent_out, token_out, score_out};
    const hipError_t err = e3::launch_beam_select(a, dtype == E3_BF16, workspace, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? E3_OK : E3_ERR_LAUNCH;
}

extern "C" int e3_beam_reorder(const int32_t* parent, int64_t seqs, int32_t beams, const int32_t* row_pages, int64_t row_width,
                               const int32_t* row_lens, int32_t page_size, int32_t* pages_out, int32_t* lens_out,
                               int32_t* src_out, int32_t* dst_out, int32_t* counts_out, void* hip_stream)
{
    if (seqs < 0 || seqs >= 1 << 24 || beams < 1 || beams > E3_MAX_BEAMS || row_width < 0 || row_width > 0x7FFFFFFF || page_size < 32 ||
        page_size > (1 << 20) || (page_size & (page_size - 1)) != 0)
        return E3_ERR_SHAPE;
    if (seqs == 0) return E3_OK;
    if (parent == nullptr || row_lens == nullptr || lens_out == nullptr || src_out == nullptr || dst_out == nullptr || counts_out == nullptr ||
        (row_width > 0 && (row_pages == nullptr || pages_out == nullptr)))
        return E3_ERR_NULL;
    // rows are read after others were written
    if ((row_width > 0 && row_pages == pages_out) || row_lens == lens_out) return E3_ERR_VALUE;
    const e3::ReorderArgs a{parent, seqs, beams, (int32_t)row_width, page_size, row_pages, row_lens, pages_out, lens_out, src_out, dst_out, counts_out};
    const hipError_t err = e3::launch_beam_reorder(a, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? E3_OK : E3_ERR_LAUNCH;
}

extern "C" int e3_cache_copy(const e3_cache* cache, const int32_t* src_pages, const int32_t* dst_pages, const int32_t* counts, int64_t n,
                             void* hip_stream)
{
    e3::CacheView view;
    const int rc = check_cache(cache, &view);
    if (rc != E3_OK) return rc;
    if (n < 0 || n >= 1 << 24 || n * view.heads >= 1 << 24) return E3_ERR_SHAPE;   // a workgroup of 256 threads each: below 2^32
    if (n == 0) return E3_OK;
    if (src_pages == nullptr || dst_pages == nullptr || counts == nullptr) return E3_ERR_NULL;
    const hipError_t err = e3::launch_cache_copy(view, src_pages, dst_pages, counts, n, static_cast<hipStream_t>(hip_stream));
    return err == hipSuccess ? E3_OK : E3_ERR_LAUNCH;
}
