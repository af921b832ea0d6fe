// C ABI of the decode step: argument checks on the host, then kernel launches.
#include <hip/hip_runtime.h>
#include <cmath>
#include <cstdint>

#include "../../include/e3.h"
#include "kv_cache.h"
#include "verify.h"
#include "vocab_pass.h"

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
