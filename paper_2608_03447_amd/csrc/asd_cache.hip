// gfx950 kernel of the paged cache: norms, rotation and append of a block's rows.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "asd_decode.h"

namespace asd {
namespace {

// ------------------------------------------------------------ 16-bit types

__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }
__device__ __forceinline__ float widen(_Float16 x) { return (float)x; }

// ------------------------------------------------------------ geometry

struct Request {
    int64_t row;      // o_i
    int64_t cached;   // tokens in the cache before the block
    int32_t count;    // rows: max(K_i, 0) + 1
    bool ok;          // rows inside the batch, tokens inside the page table
};

// Request i, by one wavefront with every lane active: the packed layout sums the lengths before it.
__device__ __forceinline__ Request request_of(const Blocks& b, int32_t i, int lane) {
    Request r;
    const int32_t k = b.block_lens[i];
    r.count = rows_of_block(k);
    if (b.row_offsets) {
        r.row = b.row_offsets[i];
    } else {
        long long sum = 0;
        for (int32_t j = lane; j < i; j += 64) sum += rows_of_block(b.block_lens[j]);
        for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
        r.row = sum;
    }
    r.cached = b.cache_lens[i];
    const int64_t room = (int64_t)b.cache.max_pages * b.cache.page_size;
    const bool rows_ok = r.row >= 0 && r.row <= b.total_rows - r.count;
    const bool cache_ok = r.cached >= 0 && r.cached <= room - r.count;
    r.ok = rows_ok && cache_ok;
    const uint32_t err = (k < 0 ? kDecodeErrNegativeK : 0u) | (rows_ok ? 0u : kDecodeErrRows) |
                         (cache_ok ? 0u : kDecodeErrCache);
    if (err != 0 && lane == 0) atomicOr(b.error_word, err);
    return r;
}

// Element offset of a token's head 0 in the cache, or -1 for a bad page (reported).
__device__ __forceinline__ int64_t slot_of(const Blocks& b, int32_t i, int64_t token) {
    const int32_t page = (int32_t)((uint32_t)token / (uint32_t)b.cache.page_size);
    const int32_t at = (int32_t)token - page * b.cache.page_size;
    const int32_t id = b.cache.page_table[(int64_t)i * b.cache.max_pages + page];
    if (id < 0 || id >= b.cache.num_pages) {
        atomicOr(b.error_word, kDecodeErrCache);
        return -1;
    }
    return (int64_t)id * b.cache.page_stride + (int64_t)at * b.cache.token_stride;
}

// ------------------------------------------------------------ append

constexpr int kAppendThreads = 256;

// One wavefront per head of a row: the head is staged in LDS as binary32, normed, then turned pair by pair.
template <typename T>
__global__ __launch_bounds__(kAppendThreads) void asd_rope_append_kernel(RopeAppendArgs a) {
    __shared__ float head[kAppendThreads / 64][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t i = (int32_t)blockIdx.x;
    const Request r = request_of(a.b, i, lane);
    if (!r.ok) return;
    const int d = a.b.cache.head_dim, half = a.rot_dim / 2;
    const int hq = a.num_q_heads, hkv = a.b.cache.num_heads, heads = hq + 2 * hkv;
    for (int32_t p = (int32_t)blockIdx.y; p < r.count; p += (int32_t)gridDim.y) {
        const int64_t row = r.row + p;
        const int64_t slot = slot_of(a.b, i, r.cached + p);
        const double pos = (double)(a.positions ? a.positions[row] : r.cached + p);
        for (int h = wave; h < heads; h += kAppendThreads / 64) {
            const bool is_q = h < hq, is_k = !is_q && h < hq + hkv;
            const int hk = is_q ? h : is_k ? h - hq : h - hq - hkv;
            const T* src = is_q ? (const T*)a.q + row * a.q_stride
                                : is_k ? (const T*)a.k + row * a.k_stride
                                       : (const T*)a.v + row * a.v_stride;
            src += (int64_t)hk * d;
            if (!is_q && slot < 0) continue;
            T* dst = is_q ? (T*)a.out_q + row * a.out_q_stride + (int64_t)hk * d
                          : (T*)(is_k ? a.b.cache.keys : a.b.cache.values) + slot +
                                (int64_t)hk * a.b.cache.head_stride;
            if (!is_q && !is_k) {
                for (int e = lane; e < d; e += 64) dst[e] = src[e];
                continue;
            }
            float* x = head[wave];
            const T* w = (const T*)(is_q ? a.q_norm : a.k_norm);
            float sum = 0.0f;
            for (int e = lane; e < d; e += 64) {
                x[e] = widen(src[e]);
                sum = fmaf(x[e], x[e], sum);
            }
            if (w) {
                for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
                const float scale = 1.0f / sqrtf(sum / (float)d + a.eps);
                for (int e = lane; e < d; e += 64) x[e] = x[e] * scale * widen(w[e]);
            }
            wave_sync();
            for (int j = lane; j < half; j += 64) {
                const int ea = a.interleaved ? 2 * j : j, eb = a.interleaved ? 2 * j + 1 : j + half;
                double turns = pos * (double)a.inv_freq[j] * 0.15915494309189533577;
                turns -= rint(turns);
                float s, c;
                sincospif(2.0f * (float)turns, &s, &c);
                const float xa = x[ea], xb = x[eb];
                dst[ea] = (T)(xa * c - xb * s);
                dst[eb] = (T)(xa * s + xb * c);
            }
            for (int e = a.rot_dim + lane; e < d; e += 64) dst[e] = (T)x[e];
            wave_sync();
        }
    }
}

// Workgroups per request: its share of the rows, the batch's requests of any length.
unsigned rows_share(const Blocks& b) {
    const int64_t y = (b.total_rows + b.num_requests - 1) / b.num_requests;
    return (unsigned)(y < 65535 ? y : 65535);
}

}  // namespace

hipError_t launch_rope_append(const RopeAppendArgs& a, bool bf16, hipStream_t stream) {
    const dim3 grid((unsigned)a.b.num_requests, rows_share(a.b));
    if (bf16)
        asd_rope_append_kernel<__bf16><<<grid, kAppendThreads, 0, stream>>>(a);
    else
        asd_rope_append_kernel<_Float16><<<grid, kAppendThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace asd
