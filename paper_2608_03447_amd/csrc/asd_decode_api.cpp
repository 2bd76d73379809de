// C ABI of the decoding operators: host-side argument checks and workspaces.
// Their kernels are in asd_cache.hip (append), asd_attend.hip (attention) and
// asd_sample.hip.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/asd.h"
#include "asd_decode.h"

namespace {

using namespace asd;

constexpr int64_t k2G = (int64_t)1 << 31;

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// A stride in elements of rows of `least` dense elements.
bool bad_stride(int64_t stride, int64_t least, int64_t rows) {
    return stride % 8 != 0 || stride < 0 || (rows > 1 && stride < least) ||
           (stride > 0 && rows > INT64_MAX / 2 / stride);
}

// The cache's sizes and strides; its pointers only where a request is there.
bool bad_cache(const asd_paged_cache& c, int32_t num_requests) {
    if (c.num_pages < 1 || c.num_pages >= k2G || c.max_pages < 1 || c.page_size < 1 ||
        (int64_t)c.max_pages * c.page_size >= k2G || c.num_heads < 1 || c.num_heads > 4096)
        return true;
    const int64_t strides[3] = {c.page_stride, c.token_stride, c.head_stride};
    const int64_t counts[3] = {c.num_pages, c.page_size, c.num_heads};
    for (int i = 0; i < 3; ++i)
        if (strides[i] < 0 || strides[i] % 8 != 0 ||
            (strides[i] > 0 && counts[i] > INT64_MAX / 8 / strides[i]))
            return true;
    if (num_requests == 0) return false;
    return !c.keys || !c.values || !c.page_table || misaligned(c.keys) || misaligned(c.values);
}

bool bad_batch(int32_t num_requests, int64_t total_rows) {
    return num_requests < 0 || total_rows < (int64_t)num_requests || total_rows >= k2G;
}

asd_status dtype_16(asd_dtype dtype) {
    return dtype == ASD_BF16 || dtype == ASD_F16 ? ASD_OK : ASD_EDTYPE;
}

// The caller's workspace when given, else the library's.
asd_status workspace_of(hipStream_t s, size_t need, void* given, size_t given_bytes, void** out) {
    *out = nullptr;
    if (given) {
        if (given_bytes < need) return ASD_ENOMEM;
        *out = given;
        return ASD_OK;
    }
    return need == 0 ? ASD_OK : decode_workspace(s, need, out);
}

}  // namespace

extern "C" {

asd_status asd_rope_append(const void* q, const void* k, const void* v, asd_dtype dtype,
                           int64_t q_stride, int64_t k_stride, int64_t v_stride,
                           int32_t num_q_heads, const void* q_norm, const void* k_norm, float eps,
                           const float* inv_freq, int32_t rot_dim, uint32_t flags,
                           const int64_t* positions, const asd_paged_cache* cache,
                           int32_t num_requests, int64_t total_rows, const int32_t* block_lens,
                           const int64_t* row_offsets, const int64_t* cache_lens, void* out_q,
                           int64_t out_q_stride, void* stream) {
    asd_status st = dtype_16(dtype);
    if (st != ASD_OK) return st;
    if (!cache || bad_batch(num_requests, total_rows) || bad_cache(*cache, num_requests))
        return ASD_EINVAL;
    const int32_t d = cache->head_dim;
    if (d < 8 || d > 256 || d % 8 != 0 || num_q_heads < 0 || num_q_heads > 4096) return ASD_EINVAL;
    if (rot_dim < 0 || rot_dim > d || rot_dim % 2 != 0 || (flags & ~(uint32_t)ASD_ROPE_INTERLEAVED))
        return ASD_EINVAL;
    if (!(eps >= 0.0f) || std::isinf(eps)) return ASD_EINVAL;
    if (num_requests == 0) return ASD_OK;
    if (!k || !v || !block_lens || !cache_lens || (rot_dim > 0 && !inv_freq)) return ASD_EINVAL;
    if ((num_q_heads > 0) != (q != nullptr) || (q != nullptr) != (out_q != nullptr))
        return ASD_EINVAL;
    if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out_q) ||
        misaligned(q_norm) || misaligned(k_norm))
        return ASD_EINVAL;
    const int64_t kv_row = (int64_t)cache->num_heads * d, q_row = (int64_t)num_q_heads * d;
    if (bad_stride(k_stride, kv_row, total_rows) || bad_stride(v_stride, kv_row, total_rows))
        return ASD_EINVAL;
    if (q && (bad_stride(q_stride, q_row, total_rows) || bad_stride(out_q_stride, q_row, total_rows)))
        return ASD_EINVAL;

    RopeAppendArgs a{};
    a.b = {*cache, num_requests, total_rows, block_lens, row_offsets, cache_lens, nullptr};
    if ((st = decode_error_word(&a.b.error_word)) != ASD_OK) return st;
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.num_q_heads = num_q_heads;
    a.q_norm = q_norm;
    a.k_norm = k_norm;
    a.eps = eps;
    a.inv_freq = inv_freq;
    a.rot_dim = rot_dim;
    a.interleaved = (flags & ASD_ROPE_INTERLEAVED) != 0;
    a.positions = positions;
    a.out_q = out_q;
    a.out_q_stride = out_q_stride;
    return launch_rope_append(a, dtype == ASD_BF16, (hipStream_t)stream) == hipSuccess ? ASD_OK
                                                                                       : ASD_EHIP;
}

static bool bad_heads(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim) {
    return (head_dim != 64 && head_dim != 128 && head_dim != 256) || num_kv_heads < 1 ||
           num_kv_heads > 4096 || num_q_heads < 1 || num_q_heads > 65536 ||
           num_q_heads % num_kv_heads != 0;
}

size_t asd_block_attention_workspace_bytes(int32_t num_q_heads, int32_t num_kv_heads,
                                           int32_t head_dim, int32_t num_requests,
                                           int64_t total_rows) {
    int cus = 0;
    if (bad_heads(num_q_heads, num_kv_heads, head_dim) || bad_batch(num_requests, total_rows) ||
        decode_compute_units(&cus) != ASD_OK)
        return 0;
    return attention_workspace_bytes(num_q_heads, num_kv_heads, head_dim, num_requests, total_rows,
                                     cus);
}

asd_status asd_block_attention(const void* q, asd_dtype dtype, int64_t q_stride,
                               int32_t num_q_heads, float scale, const asd_paged_cache* cache,
                               int32_t num_requests, int64_t total_rows,
                               const int32_t* block_lens, const int64_t* row_offsets,
                               const int64_t* cache_lens, const uint64_t* mask,
                               int32_t mask_words, void* out, void* stream, void* workspace,
                               size_t workspace_bytes) {
    asd_status st = dtype_16(dtype);
    if (st != ASD_OK) return st;
    if (!cache || bad_batch(num_requests, total_rows) || bad_cache(*cache, num_requests))
        return ASD_EINVAL;
    // (scale log2(e) has to be finite)
    if (bad_heads(num_q_heads, cache->num_heads, cache->head_dim) || !(std::fabs(scale) <= 0x1p127f))
        return ASD_EINVAL;
    if (total_rows * num_q_heads >= k2G) return ASD_EINVAL;
    if (mask_words < 0 || (mask != nullptr) != (mask_words > 0)) return ASD_EINVAL;
    if (workspace && ((uintptr_t)workspace & 255) != 0) return ASD_EINVAL;
    if (num_requests == 0) return ASD_OK;
    const int64_t row = (int64_t)num_q_heads * cache->head_dim;
    if (!q || !out || !block_lens || !cache_lens || misaligned(q) || misaligned(out) ||
        ((uintptr_t)mask & 7) != 0 || bad_stride(q_stride, row, total_rows))
        return ASD_EINVAL;

    AttentionArgs a{};
    a.b = {*cache, num_requests, total_rows, block_lens, row_offsets, cache_lens, nullptr};
    a.q = q;
    a.q_stride = q_stride;
    a.num_q_heads = num_q_heads;
    a.scale = scale;
    a.mask = mask;
    a.mask_words = mask_words;
    a.out = out;
    int cus = 0;
    void* ws = nullptr;
    hipStream_t s = (hipStream_t)stream;
    if ((st = decode_error_word(&a.b.error_word)) != ASD_OK) return st;
    if ((st = decode_compute_units(&cus)) != ASD_OK) return st;
    const size_t need = attention_workspace_bytes(num_q_heads, cache->num_heads, cache->head_dim,
                                                  num_requests, total_rows, cus);
    if ((st = workspace_of(s, need, workspace, workspace_bytes, &ws)) != ASD_OK) return st;
    return launch_block_attention(a, dtype == ASD_BF16, ws, cus, s) == hipSuccess ? ASD_OK
                                                                                  : ASD_EHIP;
}

static bool bad_logits(int64_t vocab, int64_t rows) {
    return vocab < 1 || vocab >= ((int64_t)1 << 30) || rows < 0 || rows >= k2G;
}

size_t asd_sample_workspace_bytes(asd_dtype dtype, int64_t vocab, int64_t rows) {
    int cus = 0;
    if ((dtype != ASD_F32 && dtype_16(dtype) != ASD_OK) || bad_logits(vocab, rows) ||
        decode_compute_units(&cus) != ASD_OK)
        return 0;
    return sample_workspace_bytes(vocab, rows, cus);
}

asd_status asd_sample(const void* logits, asd_dtype dtype, int64_t vocab, int64_t rows,
                      int64_t row_stride, const float* temperature, const int32_t* top_k,
                      const float* top_p, const float* min_p, const float* uniform,
                      int32_t* out_token, float* out_prob, void* stream, void* workspace,
                      size_t workspace_bytes) {
    asd_status st;
    if (dtype != ASD_F32 && (st = dtype_16(dtype)) != ASD_OK) return st;
    if (bad_logits(vocab, rows) || row_stride < vocab) return ASD_EINVAL;
    if (workspace && ((uintptr_t)workspace & 255) != 0) return ASD_EINVAL;
    if (rows == 0) return ASD_OK;
    if (!logits || !uniform || !out_token || rows > INT64_MAX / 8 / row_stride) return ASD_EINVAL;
    if (((uintptr_t)logits % (dtype == ASD_F32 ? 4 : 2)) != 0) return ASD_EINVAL;

    SampleArgs a{logits, vocab, rows, row_stride, temperature, top_k, top_p, min_p, uniform,
                 out_token, out_prob, nullptr};
    int cus = 0;
    void* ws = nullptr;
    hipStream_t s = (hipStream_t)stream;
    if ((st = decode_error_word(&a.error_word)) != ASD_OK) return st;
    if ((st = decode_compute_units(&cus)) != ASD_OK) return st;
    if ((st = workspace_of(s, sample_workspace_bytes(vocab, rows, cus), workspace, workspace_bytes,
                           &ws)) != ASD_OK)
        return st;
    return launch_sample(a, dtype, ws, cus, s) == hipSuccess ? ASD_OK : ASD_EHIP;
}

}  // extern "C"
