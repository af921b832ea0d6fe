// Launch interface of beam search: selection over beams and vocabulary, reordering of the beams' pages (beam.hip).
#pragma once
#include "kv_cache.h"

namespace e3 {

constexpr int kMaxBeams = 32, kMaxKeep = 64;

struct BeamArgs {
    const void* logits;               // [seqs][beams][V]
    int64_t seqs, V, seq_stride, beam_stride;     // strides in elements
    int32_t beams, keep;
    const float* scores;              // [seqs][beams]
    const uint8_t* finished;          // [seqs][beams] or nullptr
    int32_t eos;
    float tau;
    int32_t* parent_out;              // [seqs][keep]
    int32_t* token_out;
    float* score_out;
};

// 0: the shape does not fit (see e3_beam_select)
size_t beam_workspace_bytes(int64_t seqs, int32_t beams, int64_t V);
hipError_t launch_beam_select(const BeamArgs& a, bool bf16, void* workspace, hipStream_t stream);

struct ReorderArgs {
    const int32_t* parent;            // [seqs][beams]
    int64_t seqs;
    int32_t beams, width, page_size;
    const int32_t* row_pages;         // [seqs * beams][width]
    const int32_t* row_lens;
    int32_t* pages_out;
    int32_t* lens_out;
    int32_t* src_out;                 // [seqs * beams] each
    int32_t* dst_out;
    int32_t* counts_out;
};
hipError_t launch_beam_reorder(const ReorderArgs& a, hipStream_t stream);

// the first counts[i] tokens (up to the next multiple of eight) of page src[i] to page dst[i]
hipError_t launch_cache_copy(const CacheView& c, const int32_t* src, const int32_t* dst, const int32_t* counts, int64_t n, hipStream_t stream);

}  // namespace e3
