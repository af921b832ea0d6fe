// Verification of drafted tokens: launch interface between the C ABI and the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace e3 {

struct VerifyArgs {
    const void* logits;               // [rows][drafts + 1][V]
    const void* draft_logits;         // [rows][drafts][V] or nullptr: drafts without a distribution
    int64_t rows, V;
    int64_t row_stride, position_stride, draft_row_stride, draft_position_stride;     // elements
    int32_t drafts;
    const int32_t* draft_tokens;      // [rows][drafts]
    const int32_t* draft_lens;        // [rows] or nullptr: all of them
    const float* tau_rows;            // [rows] or nullptr: tau_scalar
    float tau_scalar;
    const float* draft_tau_rows;      // [rows] or nullptr: the same as the target's
    uint64_t seed, row_base;
    int32_t* accepted_out;            // [rows]
    int32_t* token_out;               // [rows][drafts + 1]
    float* logp_out;                  // [rows][drafts + 1], nullable
    float* entropy_out;               // [rows][drafts + 1], nullable
};

constexpr int kMaxDrafts = 63;        // one lane per position

size_t verify_workspace_bytes(int64_t rows, int32_t drafts, int64_t V);
hipError_t launch_verify(const VerifyArgs& a, bool is_bf16, void* workspace, hipStream_t stream);

}  // namespace e3
