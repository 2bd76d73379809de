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

constexpr int kMostDim = 256;        // of a head
constexpr int kAppendThreads = 256, kAppendWaves = kAppendThreads / 64;

// Request i, by the whole workgroup: the packed layout sums the lengths before it.
__device__ __forceinline__ Request request_of(const Blocks& b, int32_t i) {
    __shared__ long long part[kAppendWaves];
    Request r;
    const int32_t k = b.block_lens[i];
    r.count = rows_of_block(k);
    r.cached = b.cache_lens[i];
    if (b.row_offsets) {
        r.row = b.row_offsets[i];
    } else {
        long long sum = 0;
        for (int32_t j = (int32_t)threadIdx.x; j < i; j += kAppendThreads) sum += rows_of_block(b.block_lens[j]);
        for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
        __syncthreads();
        sum = 0;
        for (int w = 0; w < kAppendWaves; ++w) sum += part[w];
        r.row = sum;
    }
    const int64_t room = (int64_t)b.cache.max_pages * b.cache.page_size;
    const bool rows_ok = r.row >= 0 && r.row <= b.total_rows - r.count;
    const bool cache_ok = r.cached >= 0 && r.cached <= room - r.count;
    r.ok = rows_ok && cache_ok;
    const uint32_t err = (k < 0 ? kDecodeErrNegativeK : 0u) | (rows_ok ? 0u : kDecodeErrRows) |
                         (cache_ok ? 0u : kDecodeErrCache);
    if (err != 0 && threadIdx.x == 0) atomicOr(b.error_word, err);
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

// cos and sin of pos * f: the product is reduced to a part of a turn in binary64, so a position of 2^31
// keeps an angle that is right to 2^-22 of a turn.
__device__ __forceinline__ void turn(double pos, float f, float* c, float* s) {
    double turns = pos * (double)f * 0.15915494309189533577;
    turns -= rint(turns);
    sincospif(2.0f * (float)turns, s, c);
}

union Piece {
    uint4 raw;
    uint16_t h[8];
};

template <typename T> __device__ __forceinline__ float at(const Piece& x, int e) {
    return widen(__builtin_bit_cast(T, x.h[e]));
}
template <typename T> __device__ __forceinline__ void put(Piece& x, int e, float v) {
    x.h[e] = __builtin_bit_cast(uint16_t, (T)v);
}

// Heads whose size and rotated part are multiples of 16 elements.  The work is memory's: a row is read and
// written once, and 4,352 rows of 32 + 2 x 8 heads of 128 (107 MB) take 25.3 us, some 9,200 rows of 64 + 2 x 8
// (377 MB) 77 us, 4.2 and 4.9 TB/s, where a library copy of as many bytes takes 21.6 and 71, an elementwise kernel 20.6
// and 63.6 (a wavefront per head with 2-byte loads took 99 and 640).
//
// A lane holds two 16-byte pieces of a head, those whose elements it turns against each other, and kLanes
// lanes a head: no element changes its lane, and a head's square sum goes over kLanes lanes.  A step is
// 64 / kLanes heads of q, of k or of v, so where its rows lie is one scalar; a wavefront has the loads of
// kAhead steps on the way before it uses the first (two 1.07 times, four 1.08 times the time), finds the
// row's cosines and sines once meanwhile, a pair to a lane, and hands them round through LDS.  With 2^chunks
// wavefronts to a row each takes every 2^chunks-th step.  A unit is the rows of one workgroup, and
// neighbouring units are rows of one request: with the requests side by side in the grid instead each
// request's rows went to one of the eight dies, and 8 uneven requests took 147 us.
constexpr int kAhead = 3;
struct Step {
    int head, heads;      // its first head, and the heads from there on
    bool is_q, is_v;
};
__host__ __device__ __forceinline__ int steps_of(int heads, int lanes) {
    return (heads + 64 / lanes - 1) / (64 / lanes);
}

template <typename T, int kLanes, bool kNorm, bool kPairs>
__global__ __launch_bounds__(kAppendThreads, 4) void asd_rope_append_kernel(RopeAppendArgs a, int chunks,
                                                                            uint32_t share, uint32_t units) {
    static_assert(kMostDim == kAppendThreads, "a thread takes an element of each norm");
    __shared__ __align__(16) float cosine[kAppendWaves][kMostDim / 2], sine[kAppendWaves][kMostDim / 2];
    __shared__ __align__(16) T weight[2][kNorm ? kMostDim : 8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int d = a.b.cache.head_dim, half = a.rot_dim / 2;
    T weights[2];
    if (kNorm) {
        weights[0] = ((const T*)(a.q_norm ? a.q_norm : a.k_norm))[min((int)threadIdx.x, d - 1)];
        weights[1] = ((const T*)(a.k_norm ? a.k_norm : a.q_norm))[min((int)threadIdx.x, d - 1)];
    }
    const int hq = a.num_q_heads, hkv = a.b.cache.num_heads;
    const int part = lane % kLanes, sub = lane / kLanes;
    const bool turned = part < a.rot_dim / 16, in = part < d / 16;
    const int ea = turned && !kPairs ? part * 8 : part * 16, eb = turned && !kPairs ? ea + half : ea + 8;
    const int rows = kAppendWaves >> chunks;
    const int q_steps = steps_of(hq, kLanes), kv_steps = steps_of(hkv, kLanes), steps = q_steps + 2 * kv_steps;
    const auto step = [&](int n) -> Step {
        const bool is_q = n < q_steps, is_v = n >= q_steps + kv_steps;
        const int head = (n - (is_q ? 0 : q_steps + (is_v ? kv_steps : 0))) * (64 / kLanes);
        return {head, n >= steps ? 0 : (is_q ? hq : hkv) - head, is_q, is_v};
    };
    for (uint64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const uint32_t i = (uint32_t)unit / share, at_row = (uint32_t)unit % share;
        const Request r = request_of(a.b, (int32_t)i);
        if (kNorm && unit == blockIdx.x) {
            weight[0][threadIdx.x] = weights[0];
            weight[1][threadIdx.x] = weights[1];
            __syncthreads();
        }
        if (!r.ok) continue;
        for (int64_t p = (int64_t)at_row * rows + (wave >> chunks); p < r.count; p += (int64_t)share * rows) {
            const int64_t row = r.row + p;
            Piece x[kAhead][2];
            int first = wave & ((1 << chunks) - 1);
            const auto load = [&] {
#pragma unroll
                for (int n = 0; n < kAhead; ++n) {
                    const Step st = step(first + (n << chunks));
                    if (sub >= st.heads || !in) continue;
                    const T* const from = (const T*)(st.is_q ? a.q : st.is_v ? a.v : a.k) +
                                          row * (st.is_q ? a.q_stride : st.is_v ? a.v_stride : a.k_stride) +
                                          st.head * d;
                    x[n][0].raw = *(const uint4*)(from + (uint32_t)(sub * d + ea));
                    x[n][1].raw = *(const uint4*)(from + (uint32_t)(sub * d + eb));
                }
            };
            load();
            const int64_t slot = slot_of(a.b, (int32_t)i, r.cached + p);
            const double pos = (double)(a.positions ? a.positions[row] : r.cached + p);
            wave_sync();
            for (int j = lane; j < half; j += 64) turn(pos, a.inv_freq[j], &cosine[wave][j], &sine[wave][j]);
            wave_sync();
            while (true) {
#pragma unroll
                for (int n = 0; n < kAhead; ++n) {
                    const Step st = step(first + (n << chunks));
                    if (st.heads <= 0 || (!st.is_q && slot < 0)) continue;
                    if (!st.is_v) {
                        float y[16], scale = 1.0f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] = at<T>(x[n][e / 8], e % 8);
                        if (kNorm && (st.is_q ? a.q_norm : a.k_norm)) {
                            float sum = 0.0f;
#pragma unroll
                            for (int e = 0; e < 16; ++e) sum = fmaf(y[e], y[e], sum);
                            if (!in) sum = 0.0f;
#pragma unroll
                            for (int w = kLanes / 2; w > 0; w /= 2) sum += __shfl_xor(sum, w);
                            scale = 1.0f / sqrtf(sum / (float)d + a.eps);
                            Piece w[2];
                            w[0].raw = *(const uint4*)&weight[st.is_q ? 0 : 1][ea];
                            w[1].raw = *(const uint4*)&weight[st.is_q ? 0 : 1][eb];
#pragma unroll
                            for (int e = 0; e < 16; ++e) y[e] *= scale * at<T>(w[e / 8], e % 8);
                        }
                        if (turned) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float c = cosine[wave][part * 8 + e], s = sine[wave][part * 8 + e];
                                constexpr int kNext = kPairs ? 1 : 8;
                                const int ia = kPairs ? 2 * e : e, ib = ia + kNext;
                                const float xa = y[ia], xb = y[ib];
                                y[ia] = xa * c - xb * s;
                                y[ib] = xa * s + xb * c;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) put<T>(x[n][e / 8], e % 8, y[e]);
                    }
                    if (sub < st.heads && in) {
                        T* const to = st.is_q ? (T*)a.out_q + row * a.out_q_stride + st.head * d + sub * d
                                              : (T*)(st.is_v ? a.b.cache.values : a.b.cache.keys) + slot +
                                                    (st.head + sub) * a.b.cache.head_stride;
                        *(uint4*)(to + ea) = x[n][0].raw;
                        *(uint4*)(to + eb) = x[n][1].raw;
                    }
                    // one step's values in registers at a time: interleaved they spill
                    __builtin_amdgcn_sched_barrier(0);
                }
                first += kAhead << chunks;
                if (first >= steps) break;
                load();
            }
        }
    }
}

// Heads of any other size or rotated part.  One wavefront per head of a row: the head is staged in LDS as
// binary32, normed, then turned pair by pair.
template <typename T>
__global__ __launch_bounds__(kAppendThreads) void asd_rope_append_any_kernel(RopeAppendArgs a, uint32_t share,
                                                                             uint32_t units) {
    __shared__ float head[kAppendWaves][kMostDim];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int d = a.b.cache.head_dim, half = a.rot_dim / 2;
    const int hq = a.num_q_heads, hkv = a.b.cache.num_heads, heads = hq + 2 * hkv;
    for (uint64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const uint32_t i = (uint32_t)unit / share, at_row = (uint32_t)unit % share;
        const Request r = request_of(a.b, (int32_t)i);
        if (!r.ok) continue;
        for (int64_t p = at_row; p < r.count; p += share) {
            const int64_t row = r.row + p;
            const int64_t slot = slot_of(a.b, i, r.cached + p);
            const double pos = (double)(a.positions ? a.positions[row] : r.cached + p);
            for (int h = wave; h < heads; h += kAppendWaves) {
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
                    float s, c;
                    turn(pos, a.inv_freq[j], &c, &s);
                    const float xa = x[ea], xb = x[eb];
                    dst[ea] = (T)(xa * c - xb * s);
                    dst[eb] = (T)(xa * s + xb * c);
                }
                for (int e = a.rot_dim + lane; e < d; e += 64) dst[e] = (T)x[e];
                wave_sync();
            }
        }
    }
}

// Workgroups of a launch; each takes units kMostGroups apart.
constexpr unsigned kMostGroups = 65536;

template <typename T, int kLanes>
void append(const RopeAppendArgs& a, int chunks, uint32_t share, uint32_t units,
            hipStream_t stream) {
    const unsigned grid = units < kMostGroups ? units : kMostGroups;
    const bool norm = a.q_norm || a.k_norm;
    const auto kernel = a.interleaved ? norm ? asd_rope_append_kernel<T, kLanes, true, true>
                                             : asd_rope_append_kernel<T, kLanes, false, true>
                                      : norm ? asd_rope_append_kernel<T, kLanes, true, false>
                                             : asd_rope_append_kernel<T, kLanes, false, false>;
    kernel<<<grid, kAppendThreads, 0, stream>>>(a, chunks, share, units);
}

template <typename T> void append(const RopeAppendArgs& a, hipStream_t stream) {
    const int d = a.b.cache.head_dim;
    const bool any = d % 16 != 0 || a.rot_dim % 16 != 0;
    const int lanes = d <= 64 ? 4 : d <= 128 ? 8 : 16;
    // wavefronts to a row: as many as leave each no more than kAhead steps
    const int steps = steps_of(a.num_q_heads, lanes) + 2 * steps_of(a.b.cache.num_heads, lanes);
    const int chunks = steps <= kAhead ? 0 : steps <= 2 * kAhead ? 1 : 2;
    // units of rows: as many to a request as its share of the rows has; a longer one's take several
    const int64_t rows = any ? 1 : kAppendWaves >> chunks;
    const int64_t mean = (a.b.total_rows + a.b.num_requests - 1) / a.b.num_requests;
    const uint32_t share = (uint32_t)((mean + rows - 1) / rows);
    const uint32_t units = share * (uint32_t)a.b.num_requests;      // < 2^32: each n, rows < 2^31
    if (any)
        asd_rope_append_any_kernel<T>
            <<<units < kMostGroups ? units : kMostGroups, kAppendThreads, 0, stream>>>(a, share, units);
    else if (lanes == 4)
        append<T, 4>(a, chunks, share, units, stream);
    else if (lanes == 8)
        append<T, 8>(a, chunks, share, units, stream);
    else
        append<T, 16>(a, chunks, share, units, stream);
}

}  // namespace

hipError_t launch_rope_append(const RopeAppendArgs& a, bool bf16, hipStream_t stream) {
    if (bf16)
        append<__bf16>(a, stream);
    else
        append<_Float16>(a, stream);
    return hipGetLastError();
}

}  // namespace asd
