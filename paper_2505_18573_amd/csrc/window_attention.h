// Launch interface of the attention with a sliding window (window_attention.hip).
#pragma once
#include "kv_cache.h"

namespace e3 {

struct WindowArgs {
    const uint16_t* q;                // bf16 [tokens][q_heads][D]
    int64_t q_token_stride, q_head_stride;
    int32_t tokens, rows, q_heads;
    const int32_t* offsets;           // [rows + 1]: each row's queries
    const int32_t* row_pages;         // [rows][row_width]
    const int32_t* row_lens;          // [rows]
    int32_t row_width;                // pages
    int32_t window, sinks;            // at most 0x7F000000
    float scale;
    uint16_t* out;                    // bf16 [tokens][q_heads][D]
    float* lse;                       // [tokens][q_heads] or nullptr
};

// 0: the shape does not fit (see e3_window_attention)
size_t window_attention_workspace_bytes(int64_t rows, int64_t tokens, int64_t q_heads, int64_t heads, int64_t dim);
hipError_t launch_window_attention(const CacheView& c, const WindowArgs& a, void* workspace, hipStream_t stream);

}  // namespace e3
