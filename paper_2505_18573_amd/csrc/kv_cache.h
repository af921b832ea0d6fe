// The paged cache of keys and values as the kernels see it, and the launches that work on it.
//
// keys    [pages][heads][page][D]            values  [pages][heads][page / 8][D][8]
// With 8-bit elements (e4m3) an element is code * 2^e, e one exponent per token and head and per tensor, stored as
// the byte e + 127 in k_scale / v_scale [pages][heads][page].  A block of eight tokens of the values is stored column
// by column: what a lane of a matrix instruction needs for P.V (eight tokens of one column) is then eight
// neighbouring elements, so the attention reads both tensors straight into its operand registers, without a pass
// through LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace e3 {

struct CacheView {
    void* k;
    void* v;
    uint8_t* k_scale;                 // nullptr: 16-bit cache (bf16)
    uint8_t* v_scale;
    int64_t num_pages;
    int32_t page_size;                // a power of two, at least 32
    int32_t page_shift;
    int32_t heads;
    int32_t dim;                      // 64 or 128
    bool fp8;
};

struct TokenRows {                    // [tokens][heads][dim], strides in elements, columns next to each other
    const void* base;
    int64_t token_stride, head_stride;
};

hipError_t launch_cache_append(const CacheView& c, const TokenRows& k, const TokenRows& v, bool in_bf16,
                               const int64_t* slots, int64_t tokens, hipStream_t stream);
hipError_t launch_cache_read(const CacheView& c, const int64_t* slots, int64_t tokens, void* k_out, void* v_out,
                             bool out_bf16, hipStream_t stream);

struct AttentionArgs {
    const uint16_t* q;                // bf16 [rows][T][q_heads][D]
    int64_t q_row_stride, q_token_stride, q_head_stride;
    int32_t rows, T, q_heads, groups;
    const int32_t* group_offsets;     // [groups + 1]
    const int32_t* prefix_pages;      // [groups][prefix_width]
    const int32_t* prefix_lens;       // [groups]
    const int32_t* row_pages;         // [rows][row_width]
    const int32_t* row_lens;          // [rows]
    int32_t prefix_width, row_width;  // pages
    float scale;
    uint16_t* out;                    // bf16 [rows][T][q_heads][D]
    float* lse;                       // [rows][T][q_heads] or nullptr
};

// 0: the shape does not fit (see e3_prefix_attention)
size_t prefix_attention_workspace_bytes(int64_t rows, int64_t T, int64_t q_heads, int64_t heads, int64_t dim, int64_t groups);
hipError_t launch_prefix_attention(const CacheView& c, const AttentionArgs& a, void* workspace, hipStream_t stream);

}  // namespace e3
