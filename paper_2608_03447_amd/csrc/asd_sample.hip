// gfx950 kernels that draw a token from every logit row.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "asd_decode.h"

namespace asd {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 1024, kWaves = kThreads / 64;

template <int kType> struct Element;
template <> struct Element<ASD_F32> {
    typedef float T;
};
template <> struct Element<ASD_BF16> {
    typedef __bf16 T;
};
template <> struct Element<ASD_F16> {
    typedef _Float16 T;
};

// Unsigned keys in the order of the logits, -0 as +0; a NaN has the greatest.
__device__ __forceinline__ uint32_t key_of(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
constexpr uint32_t kKeyNegInf = 0x007fffffu, kKeyNan = 0xffffffffu;

template <typename V, typename Op>
__device__ __forceinline__ V block_reduce(V v, Op op, V* box) {
    for (int s = 32; s > 0; s >>= 1) v = op(v, (V)__shfl_xor(v, s));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = v;
    __syncthreads();
    v = box[0];
    for (int w = 1; w < kWaves; ++w) v = op(v, box[w]);
    __syncthreads();
    return v;
}

// A row's weights, exp((z - max) / T) in units of 2^-bits.
struct Weights {
    double top, per;       // max z; log2(e) / T
    double unit;           // 2^bits
    float top_f;
    __device__ __forceinline__ double real(float z) const {
        if (z == top_f) return 1.0;
        if (z == -INFINITY || top_f == INFINITY) return 0.0;
        return exp2(((double)z - top) * per);
    }
    __device__ __forceinline__ u64 fixed(double w) const { return (u64)(w * unit + 0.5); }
};

// ceil(f * total) of a float 0 <= f < 1 and an integer below 2^63, exactly.
__device__ __forceinline__ u64 share_ceil(float f, u64 total) {
    if (!(f > 0.0f)) return 0;
    int e;
    const uint32_t m = (uint32_t)ldexpf(frexpf(f, &e), 24);   // f = m 2^(e - 24)
    const int shift = 24 - e;
    const unsigned __int128 x = (unsigned __int128)total * m;
    if (shift >= 120) return x != 0;
    return (u64)((x + (((unsigned __int128)1 << shift) - 1)) >> shift);
}
__device__ __forceinline__ u64 share_floor(float f, u64 total) {
    if (!(f > 0.0f)) return 0;
    int e;
    const uint32_t m = (uint32_t)ldexpf(frexpf(f, &e), 24);
    const int shift = 24 - e;
    if (shift >= 120) return 0;
    return (u64)(((unsigned __int128)total * m) >> shift);
}

// One workgroup per row, which it reads several times: the greatest logit, the
// ranking's cut by two radix selections (by count, by weight), the kept
// weights of 1,024 stretches of the row, and the stretch the draw falls in.
template <int kType>
__global__ __launch_bounds__(kThreads) void asd_sample_kernel(SampleArgs a, int bits) {
    typedef typename Element<kType>::T T;
    __shared__ u64 box[kWaves];
    __shared__ u64 weight_bin[256];
    __shared__ unsigned count_bin[256];
    __shared__ u64 part[kThreads];
    __shared__ unsigned ties[kThreads];
    __shared__ u64 pick[4];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x, vocab = a.vocab;
    const T* z = (const T*)a.logits + row * a.row_stride;

    uint32_t top = 0;
    for (int64_t v = tid; v < vocab; v += kThreads) {
        const uint32_t k = key_of((float)z[v]);
        top = k > top ? k : top;
    }
    top = (uint32_t)block_reduce<u64>(top, [](u64 x, u64 y) { return x > y ? x : y; }, box);
    if (top == kKeyNan || top == kKeyNegInf) {
        if (tid == 0) {
            a.out_token[row] = -1;
            if (a.out_prob) a.out_prob[row] = 0.0f;
            atomicOr(a.error_word, kDecodeErrSample);
        }
        return;
    }
    const float t = a.temperature ? a.temperature[row] : 1.0f;
    if (!(t > 0.0f)) {
        u64 first = ~0ull;
        for (int64_t v = tid; v < vocab; v += kThreads)
            if (key_of((float)z[v]) == top) {
                first = (u64)v;
                break;
            }
        first = block_reduce<u64>(first, [](u64 x, u64 y) { return x < y ? x : y; }, box);
        if (tid == 0) {
            a.out_token[row] = (int32_t)first;
            if (a.out_prob) a.out_prob[row] = 1.0f;
        }
        return;
    }
    Weights w;
    w.top_f = value_of(top);
    w.top = (double)w.top_f;
    w.per = 1.44269504088896340736 / (double)t;
    w.unit = (double)(1ull << bits);

    // The kept prefix: keys above `cut`, and the first `cut_ties` tokens whose key is `cut`.
    const int32_t k = a.top_k ? a.top_k[row] : 0;
    const float p = a.top_p ? a.top_p[row] : 1.0f;
    const bool by_count = k > 0 && k < vocab, by_mass = p < 1.0f;
    uint32_t cut = 0;
    u64 cut_ties = ~0ull;
    const auto add = [](u64 x, u64 y) { return x + y; };
    for (int stage = 0; stage < 2; ++stage) {
        if (!(stage == 0 ? by_count : by_mass)) continue;
        // what the keys of earlier stages leave: stage 1 counts keys above `limit` whole and
        // `limit_ties` tokens at it
        const uint32_t limit = cut;
        const u64 limit_ties = cut_ties;
        u64 want = (u64)k;
        if (stage == 1) {
            u64 sum = 0, at = 0;
            for (int64_t v = tid; v < vocab; v += kThreads) {
                const float x = (float)z[v];
                const uint32_t key = key_of(x);
                if (key > limit) sum += w.fixed(w.real(x));
                at += key == limit;
            }
            sum = block_reduce<u64>(sum, add, box);
            at = block_reduce<u64>(at, add, box);
            at = at < limit_ties ? at : limit_ties;
            sum += at * w.fixed(w.real(value_of(limit)));
            want = share_ceil(p, sum);
            if (want < 1) want = 1;
        }
        uint32_t prefix = 0;
        for (int level = 3; level >= 0; --level) {
            for (int b = tid; b < 256; b += kThreads) weight_bin[b] = count_bin[b] = 0;
            __syncthreads();
            const uint32_t above = level == 3 ? 0u : ~0u << (8 * level + 8);
            for (int64_t v = tid; v < vocab; v += kThreads) {
                const float x = (float)z[v];
                const uint32_t key = key_of(x);
                if ((key & above) != prefix || key < limit) continue;
                const int b = (key >> (8 * level)) & 255;
                if (stage == 1 && key > limit) atomicAdd(&weight_bin[b], w.fixed(w.real(x)));
                if (stage == 0 || key == limit) atomicAdd(&count_bin[b], 1u);
            }
            __syncthreads();
            if (tid == 0) {
                // the bin in which the wanted amount is reached, from the greatest key down
                u64 have = 0;
                int b = 255;
                const u64 limit_weight = stage == 1 ? w.fixed(w.real(value_of(limit))) : 0;
                for (; b > 0; --b) {
                    u64 here = count_bin[b];
                    if (stage == 1) {
                        here = here < limit_ties ? here : limit_ties;
                        here = weight_bin[b] + here * limit_weight;
                    }
                    if (have + here >= want) break;
                    have += here;
                }
                pick[0] = (u64)b;
                pick[1] = want - have;
            }
            __syncthreads();
            prefix |= (uint32_t)pick[0] << (8 * level);
            want = pick[1];
            __syncthreads();
        }
        cut = prefix;
        if (stage == 0) {
            cut_ties = want;
        } else {
            const u64 one = w.fixed(w.real(value_of(cut)));
            u64 n = one > 0 ? (want + one - 1) / one : 1;
            if (n < 1) n = 1;
            cut_ties = cut == limit && n > limit_ties ? limit_ties : n;
        }
    }
    const float m = a.min_p ? a.min_p[row] : 0.0f;
    const double least = m > 0.0f ? (m < 1.0f ? (double)m : 1.0) : 0.0;

    // The kept weight of every thread's stretch, ties at the cut in index order.
    const int64_t stretch = (vocab + kThreads - 1) / kThreads;
    const int64_t from = tid * stretch < vocab ? tid * stretch : vocab;
    const int64_t to = from + stretch < vocab ? from + stretch : vocab;
    unsigned n = 0;
    for (int64_t v = from; v < to; ++v) n += key_of((float)z[v]) == cut;
    ties[tid] = n;
    __syncthreads();
    if (tid == 0) {
        unsigned sum = 0;
        for (int j = 0; j < kThreads; ++j) {
            const unsigned c = ties[j];
            ties[j] = sum;
            sum += c;
        }
    }
    __syncthreads();
    const auto kept = [&](float x, u64& seen) -> u64 {
        const uint32_t key = key_of(x);
        if (key < cut || (key == cut && seen++ >= cut_ties)) return 0;
        const double real = w.real(x);
        return real >= least ? w.fixed(real) : 0;
    };
    u64 seen = ties[tid], sum = 0;
    for (int64_t v = from; v < to; ++v) sum += kept((float)z[v], seen);
    part[tid] = sum;
    __syncthreads();
    if (tid == 0) {
        u64 total = 0;
        for (int j = 0; j < kThreads; ++j) total += part[j];
        float u = a.uniform[row];
        u = u < 0x1.fffffep-1f ? u : u >= 1.0f ? 0x1.fffffep-1f : u;
        const u64 target = share_floor(u, total);      // the running sum has to exceed it
        u64 before = 0;
        int j = 0;
        while (before + part[j] <= target) before += part[j++];
        pick[0] = (u64)j;
        pick[1] = before;
        pick[2] = target;
        pick[3] = total;
    }
    __syncthreads();
    if ((u64)tid == pick[0]) {
        u64 run = pick[1];
        seen = ties[tid];
        for (int64_t v = from; v < to; ++v) {
            const u64 x = kept((float)z[v], seen);
            run += x;
            if (run > pick[2]) {
                a.out_token[row] = (int32_t)v;
                if (a.out_prob) a.out_prob[row] = (float)((double)x / (double)pick[3]);
                break;
            }
        }
    }
}

}  // namespace

size_t sample_workspace_bytes(int64_t, int64_t, int) { return 0; }

hipError_t launch_sample(const SampleArgs& a, asd_dtype dtype, void*, int, hipStream_t stream) {
    int bits = 62;
    while (((int64_t)1 << (62 - bits)) < a.vocab) --bits;
    if (bits > 52) bits = 52;
    const dim3 grid((unsigned)a.rows);
    if (dtype == ASD_F32)
        asd_sample_kernel<ASD_F32><<<grid, kThreads, 0, stream>>>(a, bits);
    else if (dtype == ASD_BF16)
        asd_sample_kernel<ASD_BF16><<<grid, kThreads, 0, stream>>>(a, bits);
    else
        asd_sample_kernel<ASD_F16><<<grid, kThreads, 0, stream>>>(a, bits);
    return hipGetLastError();
}

}  // namespace asd
