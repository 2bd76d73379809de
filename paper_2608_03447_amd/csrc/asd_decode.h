// Arguments and launches of the decoding operators (asd_rope_append,
// asd_block_attention, asd_sample), shared by their host code and kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/asd.h"

namespace asd {

// From asd_api.cpp: the workspace of (current device, stream), grown to at
// least `bytes`; the compute units of the current device; and the address of its
// error word.
asd_status decode_workspace(hipStream_t stream, size_t bytes, void** out);
asd_status decode_compute_units(int* out);
asd_status decode_error_word(uint32_t** out);

// Bits of the error word that these operators set (the values of ASD_DEVERR_*).
constexpr uint32_t kDecodeErrNegativeK = ASD_DEVERR_NEGATIVE_K, kDecodeErrRows = ASD_DEVERR_ROWS,
                   kDecodeErrCache = ASD_DEVERR_CACHE, kDecodeErrSample = ASD_DEVERR_SAMPLE;

// The requests of a batch and the cache they fill and read.
struct Blocks {
    asd_paged_cache cache;
    int32_t num_requests;
    int64_t total_rows;
    const int32_t* block_lens;
    const int64_t* row_offsets;      // or nullptr: packed
    const int64_t* cache_lens;
    uint32_t* error_word;
};

#ifdef __HIPCC__
// Rows of a block of K drafts (a K beyond any batch stays one that does not fit).
__device__ __forceinline__ int32_t rows_of_block(int32_t k) { return min(max(k, 0), 0x7ffffffe) + 1; }

// LDS written by one lane of a wavefront is read by another after this.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
#endif

struct RopeAppendArgs {
    Blocks b;
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    int32_t num_q_heads;
    const void *q_norm, *k_norm;
    float eps;
    const float* inv_freq;
    int32_t rot_dim;
    bool interleaved;
    const int64_t* positions;
    void* out_q;
    int64_t out_q_stride;
};
hipError_t launch_rope_append(const RopeAppendArgs& a, bool bf16, hipStream_t stream);

struct AttentionArgs {
    Blocks b;
    const void* q;
    int64_t q_stride;
    int32_t num_q_heads;
    float scale;
    const uint64_t* mask;
    int32_t mask_words;
    void* out;
    uint32_t page_magic;   // of Tokens
    int32_t page_shift;
    int32_t team;          // workgroups that share a stretch
};
size_t attention_workspace_bytes(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                 int32_t num_requests, int64_t total_rows, int cus);
hipError_t launch_block_attention(const AttentionArgs& a, bool bf16, void* workspace, int cus,
                                  hipStream_t stream);

struct SampleArgs {
    const void* logits;
    int64_t vocab, rows, row_stride;
    const float* temperature;
    const int32_t* top_k;
    const float *top_p, *min_p, *uniform;
    int32_t* out_token;
    float* out_prob;
    uint32_t* error_word;
};
size_t sample_workspace_bytes(int64_t vocab, int64_t rows, int cus);
hipError_t launch_sample(const SampleArgs& a, asd_dtype dtype, void* workspace, int cus,
                         hipStream_t stream);

}  // namespace asd
