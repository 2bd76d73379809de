// gfx950 kernels of the attention of draft blocks and trees to the paged cache.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "asd_decode.h"

namespace asd {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// Work is shared out in units of kUnit tokens of one item: a request, one of its
// key heads and a tile of kRows = 16 kTiles of its (row, head of the group) pairs.
// The batch's units lie in one line and every workgroup takes an equal stretch of
// it, so ragged caches balance and one long sequence spreads over the chip.  An
// item that a stretch cuts leaves binary32 partials (its greatest score, sum and
// weighted values so far) that a second kernel joins; an item inside one stretch
// is finished at once.

constexpr int kAttendThreads = 256, kAttendWaves = kAttendThreads / 64;
constexpr int kStrip = 32;                          // tokens a wavefront takes at a time
constexpr int kUnit = kStrip * kAttendWaves;

// Where stretch x of the batch's `total` units begins: floor(total x / wgs).
__device__ __forceinline__ int64_t bound_of(int64_t total, int64_t wgs, int64_t x) {
    const int64_t q = total / wgs;
    return q * x + (total - q * wgs) * x / wgs;
}

struct Where {
    int64_t total;      // units of the batch
    int64_t unit;       // the unit asked for, counted within its request
    int64_t row;        // the request's first row
    int32_t request;    // -1: the unit lies behind the last one
};

__device__ __forceinline__ int64_t units_of(const Blocks& b, int32_t group, int32_t rows, int64_t row,
                                            int32_t count, int64_t cached, uint32_t& err) {
    const int64_t room = (int64_t)b.cache.max_pages * b.cache.page_size;
    const bool rows_ok = row >= 0 && row <= b.total_rows - count;
    const bool cache_ok = cached >= 0 && cached <= room - count;
    err |= (rows_ok ? 0u : kDecodeErrRows) | (cache_ok ? 0u : kDecodeErrCache);
    if (!rows_ok || !cache_ok) return 0;
    const int64_t tiles = ((int64_t)count * group + rows - 1) / rows;
    return tiles * b.cache.num_heads * ((cached + count + kUnit - 1) / kUnit);
}

// Sum of v over the threads before this one, and over all of them.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* box, int64_t* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    long long sum = v;
    for (int s = 1; s < 64; s <<= 1) {
        const long long up = __shfl_up(sum, s);
        if (lane >= s) sum += up;
    }
    __syncthreads();
    if (lane == 63) box[wave] = sum;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int w = 0; w < kAttendWaves; ++w) {
        before += w < wave ? box[w] : 0;
        all += box[w];
    }
    *total = all;
    return before + sum - v;
}

// The unit at which stretch `id` of `wgs` begins, found by the whole workgroup.
__device__ Where locate(const Blocks& b, int32_t group, int32_t rows, int64_t id, int64_t wgs,
                        bool report, int64_t* box, Where* out) {
    const int32_t n = b.num_requests, per = (n + kAttendThreads - 1) / kAttendThreads;
    const int32_t first = min(n, (int32_t)threadIdx.x * per), last = min(n, first + per);
    int64_t row = 0, unused;
    uint32_t err = 0;
    if (!b.row_offsets) {
        int64_t mine = 0;
        for (int32_t i = first; i < last; ++i) mine += max(b.block_lens[i], 0) + 1;
        row = block_scan(mine, box, &unused);
    }
    int64_t units = 0, at = row;
    for (int32_t i = first; i < last; ++i) {
        const int32_t k = b.block_lens[i], count = max(k, 0) + 1;
        err |= k < 0 ? kDecodeErrNegativeK : 0u;
        units += units_of(b, group, rows, b.row_offsets ? b.row_offsets[i] : at, count, b.cache_lens[i], err);
        at += count;
    }
    if (report && err != 0) atomicOr(b.error_word, err);
    int64_t total;
    int64_t before = block_scan(units, box, &total);
    const int64_t unit = bound_of(total, wgs, id);
    if (threadIdx.x == 0) *out = Where{total, 0, 0, -1};
    __syncthreads();
    if (unit >= before && unit < before + units) {
        for (int32_t i = first; i < last; ++i) {
            const int32_t count = max(b.block_lens[i], 0) + 1;
            const int64_t at_row = b.row_offsets ? b.row_offsets[i] : row;
            const int64_t u = units_of(b, group, rows, at_row, count, b.cache_lens[i], err);
            if (unit < before + u) {
                *out = Where{total, unit - before, at_row, i};
                break;
            }
            before += u;
            row += count;
        }
    }
    __syncthreads();
    return *out;
}

template <typename T> struct Half;
template <> struct Half<__bf16> {
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 mfma(x8 a, x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    static constexpr uint32_t kExponent = 0x7f80u;
};
template <> struct Half<_Float16> {
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 mfma(x8 a, x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    static constexpr uint32_t kExponent = 0x7c00u;
};

// The greatest / the sum over the four lanes that hold one query row (lanes l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float rows_max(float x) {
    u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float rows_sum(float x) {
    u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r.x) + __uint_as_float(r.y);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// Weights are exp2 of scores less a reference that trails the greatest one: they reach 2^kLead
// at most, and the reference is moved, and what was summed rescaled, only when one would pass that.
// Then the greatest is put at 2^kSet, which keeps weights down to 2^-30 of it normal in binary16.
constexpr float kLead = 14.0f, kSet = 6.0f;

// One workgroup per stretch.  Every wavefront walks strips of 32 tokens of its
// own: no barrier until an item's end, when the four wavefronts' sums are joined.
//
// Scores are formed transposed, S^T = K Q^T (A: 16 tokens, B: 16 query rows), so
// that a lane holds 8 tokens' scores of one query row and the weights, as they lie
// in the registers, are the B operand of O^T = V^T P^T; the order of a product's
// inner index is free, so that operand's token order (4 g + j of either 16, g =
// lane / 16) is simply the order in which V is loaded.  A lane loads D / 16
// neighbouring elements of each of its 8 tokens' values and pairs them up by
// v_perm: nothing goes through LDS but page offsets, and O^T leaves every lane
// with D / 4 neighbouring elements of its query row.
template <typename T, int D, int kTiles>
__global__ __launch_bounds__(kAttendThreads, D == 256 ? 1 : 2) void asd_attend_kernel(AttentionArgs a, float* partials) {
    constexpr int kRows = 16 * kTiles, NC = D / 16, kSteps = D / 32, kVecs = (NC + 7) / 8;
    constexpr bool kQueriesInLds = kTiles > 2;
    typedef typename Half<T>::x8 x8;
    __shared__ int64_t box[kAttendWaves];
    __shared__ Where where_box;
    __shared__ int64_t offsets[kAttendWaves][kStrip];
    __shared__ float joined[kAttendWaves][16][D + 4];
    __shared__ float tops[kAttendWaves][16], sums[kAttendWaves][16];
    __shared__ x8 queries[kQueriesInLds ? kTiles * kSteps * 64 : 1];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    const asd_paged_cache& cache = a.b.cache;
    const int32_t group = a.num_q_heads / cache.num_heads;
    // neighbouring stretches, which may share keys and values, on one XCD
    const int64_t wgs = gridDim.x, eighth = wgs / 8;
    const int64_t id = blockIdx.x < eighth * 8 ? (blockIdx.x % 8) * eighth + blockIdx.x / 8 : blockIdx.x;
    Where at = locate(a.b, group, kRows, id, wgs, blockIdx.x == 0, box, &where_box);
    int64_t left = bound_of(at.total, wgs, id + 1) - bound_of(at.total, wgs, id);
    const float per = a.scale * 1.44269504f;

    while (left > 0) {
        const int32_t count = max(a.b.block_lens[at.request], 0) + 1;
        const int64_t cached64 = a.b.cache_lens[at.request];
        const int64_t pairs = (int64_t)count * group, units = (cached64 + count + kUnit - 1) / kUnit;
        const int64_t tiles = (pairs + kRows - 1) / kRows;
        uint32_t unused = 0;
        if (units_of(a.b, group, kRows, at.row, count, cached64, unused) <= at.unit) {
            // on to the next request
            at.row = a.b.row_offsets ? a.b.row_offsets[at.request + 1] : at.row + count;
            at.request += 1;
            at.unit = 0;
            continue;
        }
        const int64_t item = at.unit / units, from = at.unit - item * units;
        const int64_t to = from + left < units ? from + left : units;
        const int32_t head = (int32_t)(item / tiles);
        const int64_t first = (item - head * tiles) * kRows;      // of the pairs
        at.unit += to - from;
        left -= to - from;

        // the tile's queries: B operands, lane n's row, 8 elements of every 32
        const auto query = [&](int tile, int step) -> x8 {
            const int64_t m = first + 16 * tile + n;
            if (m >= pairs) return x8{};
            const int64_t p = m / group;
            const int32_t x = (int32_t)(m - p * group);
            return *(const x8*)((const T*)a.q + (at.row + p) * a.q_stride +
                                ((int64_t)head * group + x) * D + 32 * step + 8 * g);
        };
        x8 q[kQueriesInLds ? 1 : kTiles][kSteps];
        if constexpr (kQueriesInLds) {
            __syncthreads();
            for (int tile = wave; tile < kTiles; tile += kAttendWaves)
                #pragma unroll
                for (int step = 0; step < kSteps; ++step)
                    queries[(tile * kSteps + step) * 64 + lane] = query(tile, step);
            __syncthreads();
        } else {
            #pragma unroll
            for (int tile = 0; tile < kTiles; ++tile)
                #pragma unroll
                for (int step = 0; step < kSteps; ++step) q[tile][step] = query(tile, step);
        }

        f32x4 o[kTiles][NC];
        float ref[kTiles], sum[kTiles];
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile) {
#pragma unroll
            for (int c = 0; c < NC; ++c) o[tile][c] = f32x4{0, 0, 0, 0};
            ref[tile] = -INFINITY;
            sum[tile] = 0.0f;
        }
        // a chain's rows see no token behind the tile's last one
        const int32_t cached = (int32_t)cached64, end_all = cached + count;
        const int32_t last_p = (int32_t)((min(first + kRows, pairs) - 1) / group);
        const int32_t end = a.mask ? end_all : cached + last_p + 1;
        const int32_t strip_end = (int32_t)min(to * kUnit, (int64_t)end);
        int32_t strip = (int32_t)(from * kUnit) + wave * kStrip;
        int64_t* const offs = offsets[wave];
        const int32_t* const table = cache.page_table + (int64_t)at.request * cache.max_pages;
        const T* const keys = (const T*)cache.keys + (int64_t)head * cache.head_stride;
        const T* const values = (const T*)cache.values + (int64_t)head * cache.head_stride;

        // A strip's page ids (lanes l and l + 32 hold token l), its tokens' offsets (negative: not
        // there), and its keys and values as operands.
        const auto page_of = [&](int32_t t0) -> int32_t {
            const int32_t t = t0 + (lane & 31);
            return t < end_all ? table[(uint32_t)t / (uint32_t)cache.page_size] : 0;
        };
        x8 k[2][kSteps];
        u32x4 v[8][kVecs];
        const auto put_offsets = [&](int32_t t0, int32_t page) -> bool {
            const int32_t t = t0 + (lane & 31);
            const bool in = t < end_all, ok = in && page >= 0 && page < cache.num_pages;
            if (in && !ok) atomicOr(a.b.error_word, kDecodeErrCache);
            const int32_t slot = (int32_t)((uint32_t)t % (uint32_t)cache.page_size);
            wave_sync();
            if (lane < 32)
                offs[lane] = ok ? (int64_t)page * cache.page_stride + (int64_t)slot * cache.token_stride : -1;
            wave_sync();
            return __all(ok);
        };
        const auto load_keys = [&]() {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const T* src = keys + max(offs[16 * h + n], (int64_t)0) + 8 * g;
#pragma unroll
                for (int step = 0; step < kSteps; ++step) k[h][step] = *(const x8*)(src + 32 * step);
            }
        };
        const auto load_values = [&]() {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const T* src = values + max(offs[(j & 3) + 4 * g + 16 * (j >> 2)], (int64_t)0) + NC * n;
                if constexpr (NC == 4) {
                    const u32x2 w = *(const u32x2*)src;
                    v[j][0].x = w.x;
                    v[j][0].y = w.y;
                } else {
#pragma unroll
                    for (int x = 0; x < kVecs; ++x) v[j][x] = *(const u32x4*)(src + 8 * x);
                }
            }
        };

        int32_t page = 0;
        bool whole = false;
        if (strip < strip_end) {
            page = page_of(strip);
            whole = put_offsets(strip, page);
            load_keys();
            load_values();
            page = page_of(strip + kUnit);
        }
        for (; strip < strip_end; strip += kUnit) {
            const bool more = strip + kUnit < strip_end;
            // Which of the lane's 8 tokens its rows see, 8 bits a tile, and which are there at all.
            const bool plain = whole && strip + kStrip <= cached;
            uint32_t seen = ~0u, there = 0xffu;
            if (!plain) {
                seen = there = 0;
#pragma unroll 1
                for (int j = 0; j < 8; ++j) {
                    const int32_t at_strip = (j & 3) + 4 * g + 16 * (j >> 2), x = strip + at_strip - cached;
                    if (offs[at_strip] < 0) continue;
                    there |= 1u << j;
#pragma unroll 1
                    for (int tile = 0; tile < kTiles; ++tile) {
                        const int64_t p = min(first + 16 * tile + n, pairs - 1) / group;
                        const bool sees = x < 0 || (!a.mask ? x <= p
                                                            : x < 64 * (int64_t)a.mask_words &&
                            ((a.mask[(at.row + p) * a.mask_words + x / 64] >> (x % 64)) & 1) != 0);
                        seen |= (uint32_t)sees << (8 * tile + j);
                    }
                }
            }

            x8 w[kTiles];
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile) {
                f32x4 s[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
                for (int step = 0; step < kSteps; ++step) {
                    x8 qq;
                    if constexpr (kQueriesInLds) qq = queries[(tile * kSteps + step) * 64 + lane];
                    else qq = q[tile][step];
#pragma unroll
                    for (int h = 0; h < 2; ++h) s[h] = Half<T>::mfma(k[h][step], qq, s[h]);
                }
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = s[j >> 2][j & 3] * per;
                if (!plain) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = (seen >> (8 * tile + j)) & 1 ? x[j] : -INFINITY;
                }
                float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                                  fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
                top = rows_max(top);
                if (__any(top > ref[tile] + kLead)) {
                    const float now = top > ref[tile] + kLead ? top - kSet : ref[tile];
                    const float keep = now == ref[tile] ? 1.0f : __builtin_amdgcn_exp2f(ref[tile] - now);
                    ref[tile] = now;
                    sum[tile] *= keep;
#pragma unroll
                    for (int c = 0; c < NC; ++c) o[tile][c] *= keep;
                }
                const float from_ref = ref[tile] == -INFINITY ? 0.0f : ref[tile];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] = __builtin_amdgcn_exp2f(x[j] - from_ref);
                    sum[tile] += x[j];
                    w[tile][j] = (T)x[j];
                }
            }
            bool next_whole = false;
            if (more) {
                next_whole = put_offsets(strip + kUnit, page);
                load_keys();
                page = page_of(strip + 2 * kUnit);
            }

            // Values that are not there are zeros.  A token that holds an infinity or a NaN
            // would reach every row through its weight 0: it leaves the product and is added by
            // hand to the rows that see it.
            uint32_t odd = 0;
            if (!plain) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    bool special = false;
#pragma unroll
                    for (int x = 0; x < kVecs; ++x)
#pragma unroll
                        for (int y = 0; y < (NC == 4 ? 2 : 4); ++y) {
                            const uint32_t word = (there >> j) & 1 ? v[j][x][y] : 0u;
                            v[j][x][y] = word;
                            constexpr uint32_t e = Half<T>::kExponent;
                            special |= (word & e) == e || (word >> 16 & e) == e;
                        }
                    const uint64_t lanes = __ballot(special);
#pragma unroll
                    for (int gg = 0; gg < 4; ++gg)
                        odd |= (uint32_t)((lanes >> (16 * gg) & 0xffff) != 0) << ((j & 3) + 4 * gg + 16 * (j >> 2));
                }
                if (odd != 0) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const bool mine = (odd >> ((j & 3) + 4 * g + 16 * (j >> 2))) & 1;
#pragma unroll
                        for (int x = 0; x < kVecs; ++x) v[j][x] = mine ? u32x4{0, 0, 0, 0} : v[j][x];
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                u32x4 f;
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    f[y] = __builtin_amdgcn_perm(v[2 * y + 1][c / 8][c / 2 % 4], v[2 * y][c / 8][c / 2 % 4],
                                                 c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int tile = 0; tile < kTiles; ++tile)
                    o[tile][c] = Half<T>::mfma(__builtin_bit_cast(x8, f), w[tile], o[tile][c]);
            }
            if (odd != 0) {
#pragma unroll
                for (int tile = 0; tile < kTiles; ++tile) {
                    wave_sync();
#pragma unroll
                    for (int j = 0; j < 8; ++j)       // -1: not seen
                        joined[wave][n][(j & 3) + 4 * g + 16 * (j >> 2)] =
                            (seen >> (8 * tile + j)) & 1 ? (float)w[tile][j] : -1.0f;
                    wave_sync();
#pragma unroll 1
                    for (uint32_t rest = odd; rest != 0; rest &= rest - 1) {
                        const int32_t at_strip = __builtin_ctz(rest), t = strip + at_strip;
                        const float weight = joined[wave][n][at_strip];
                        if (weight == -1.0f) continue;
                        const int64_t off =
                            (int64_t)table[(uint32_t)t / (uint32_t)cache.page_size] * cache.page_stride +
                            (int64_t)((uint32_t)t % (uint32_t)cache.page_size) * cache.token_stride;
                        const T* src = values + off + 4 * NC * g;
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int c = 0; c < NC; ++c)
                                o[tile][c][r] = fmaf(weight, (float)src[NC * r + c], o[tile][c][r]);
                    }
                }
            }
            if (more) load_values();
            whole = next_whole;
        }

        // the wavefronts' sums, joined tile by tile
        const bool complete = from == 0 && to == units;
        float* const slot = partials + (2 * id + (from > 0 ? 0 : 1)) * (int64_t)(kRows * (D + 2));
        #pragma unroll
        for (int tile = 0; tile < kTiles; ++tile) {
            sum[tile] = rows_sum(sum[tile]);
            if (ref[tile] == -INFINITY && sum[tile] != sum[tile]) ref[tile] = 0.0f;   // every score a NaN
            __syncthreads();
            if (g == 0) {
                tops[wave][n] = ref[tile];
                sums[wave][n] = sum[tile];
            }
            __syncthreads();
            float best = tops[0][n];
            #pragma unroll
            for (int w = 1; w < kAttendWaves; ++w) best = fmaxf(best, tops[w][n]);
            const float mine = ref[tile] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref[tile] - best);
            #pragma unroll
            for (int r = 0; r < 4; ++r)
                #pragma unroll
                for (int c = 0; c < NC; c += 4)
                    *(f32x4*)&joined[wave][n][4 * NC * g + NC * r + c] =
                        f32x4{o[tile][c][r], o[tile][c + 1][r], o[tile][c + 2][r], o[tile][c + 3][r]} * mine;
            __syncthreads();
            // 16 threads a row, each every 16th vector of 4 elements
            const int row = threadIdx.x >> 4;
            best = tops[0][row];
            #pragma unroll
            for (int w = 1; w < kAttendWaves; ++w) best = fmaxf(best, tops[w][row]);
            float total = 0.0f;
            #pragma unroll
            for (int w = 0; w < kAttendWaves; ++w)
                total += tops[w][row] == -INFINITY ? 0.0f
                                                   : sums[w][row] * __builtin_amdgcn_exp2f(tops[w][row] - best);
            const int64_t m = first + 16 * tile + row;
            if (!complete && (threadIdx.x & 15) == 0) {
                slot[kRows * D + 16 * tile + row] = best;
                slot[kRows * (D + 1) + 16 * tile + row] = total;
            }
            const int64_t p = m / group;
            const float over = best == -INFINITY ? 0.0f : 1.0f / total;
            for (int e = 4 * (threadIdx.x & 15); e < D; e += 64) {
                f32x4 x = *(const f32x4*)&joined[0][row][e];
                #pragma unroll
                for (int w = 1; w < kAttendWaves; ++w) x += *(const f32x4*)&joined[w][row][e];
                if (!complete) {
                    *(f32x4*)&slot[(16 * tile + row) * D + e] = x;
                } else if (m < pairs) {
                    T* dst = (T*)a.out + ((at.row + p) * a.num_q_heads + (int64_t)head * group +
                                          (m - p * group)) * D + e;
                    typename Half<T>::x2 y[2];
                    #pragma unroll
                    for (int z = 0; z < 4; ++z) y[z / 2][z % 2] = (T)(x[z] * over);
                    *(u32x2*)dst = u32x2{__builtin_bit_cast(uint32_t, y[0]), __builtin_bit_cast(uint32_t, y[1])};
                }
            }
        }
        __syncthreads();
    }
}

// Joins the partials of the item that the bound of two stretches, blockIdx.x and the one before, cuts; the
// first of an item's bounds does it.  A wavefront takes a row.
template <typename T, int D, int kTiles>
__global__ __launch_bounds__(kAttendThreads) void asd_attend_join_kernel(AttentionArgs a, const float* partials,
                                                                         int64_t wgs) {
    constexpr int kRows = 16 * kTiles, kPer = D / 64;
    __shared__ int64_t box[kAttendWaves];
    __shared__ Where where_box;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t group = a.num_q_heads / a.b.cache.num_heads;
    const int64_t id = blockIdx.x + 1;
    const Where at = locate(a.b, group, kRows, id, wgs, false, box, &where_box);
    if (at.request < 0) return;
    const auto bound = [&](int64_t x) { return bound_of(at.total, wgs, x); };
    const int32_t count = max(a.b.block_lens[at.request], 0) + 1;
    const int64_t pairs = (int64_t)count * group;
    const int64_t units = (a.b.cache_lens[at.request] + count + kUnit - 1) / kUnit;
    const int64_t tiles = (pairs + kRows - 1) / kRows;
    const int64_t item = at.unit / units, inside = at.unit - item * units;
    const int64_t u = bound(id), begin = u - inside, end = begin + units;
    if (inside == 0 || bound(id - 1) > begin) return;
    const int32_t head = (int32_t)(item / tiles);
    const int64_t first = (item - head * tiles) * kRows;
    int64_t last = id;                                   // the last stretch of the item
    while (bound(last + 1) < end) ++last;
    constexpr int64_t kSize = (int64_t)kRows * (D + 2);
    const int64_t parts = last - id + 2;
    const auto part = [&](int64_t j) { return partials + (2 * (id - 1 + j) + (j == 0 ? 1 : 0)) * kSize; };
    for (int row = (int)blockIdx.y * kAttendWaves + wave; row < kRows; row += kAttendWaves * (int)gridDim.y) {
        const int64_t m = first + row;
        if (m >= pairs) break;
        float best = -INFINITY;
        for (int64_t j = lane; j < parts; j += 64)
            if (bound(id - 1 + j) < bound(id + j)) best = fmaxf(best, part(j)[kRows * D + row]);
        for (int s = 32; s > 0; s >>= 1) best = fmaxf(best, __shfl_xor(best, s));
        float total = 0.0f, o[kPer];
        for (int e = 0; e < kPer; ++e) o[e] = 0.0f;
        for (int64_t j0 = 0; j0 < parts; j0 += 64) {
            float f = 0.0f;
            if (j0 + lane < parts && bound(id - 1 + j0 + lane) < bound(id + j0 + lane)) {
                const float* x = part(j0 + lane);
                const float top = x[kRows * D + row];
                f = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - best);
                total += top == -INFINITY ? 0.0f : f * x[kRows * (D + 1) + row];
            }
            const int here = (int)min((int64_t)64, parts - j0);

            for (int j = 0; j < here; ++j) {
                const float fj = __shfl(f, j);
                const float* x = part(j0 + j) + row * D;
                if (fj != 0.0f)
                    for (int e = 0; e < kPer; ++e) o[e] = fmaf(fj, x[kPer * lane + e], o[e]);
            }
        }
        for (int s = 32; s > 0; s >>= 1) total += __shfl_xor(total, s);
        const float over = best == -INFINITY ? 0.0f : 1.0f / total;
        const int64_t p = m / group;
        T* dst = (T*)a.out + ((at.row + p) * a.num_q_heads + (int64_t)head * group + (m - p * group)) * D;
        for (int e = 0; e < kPer; ++e) dst[kPer * lane + e] = (T)(o[e] * over);
    }
}

}  // namespace

namespace {

// 16-row tiles of an item: what the batch's blocks fill on average.  Wide heads take at most two.
int tiles_of(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t num_requests,
             int64_t total_rows) {
    const int64_t pairs = total_rows / num_requests * (num_q_heads / num_kv_heads);
    return pairs <= 16 ? 1 : pairs <= 32 || head_dim == 256 ? 2 : 4;
}

// Two workgroups fit on a compute unit.
int64_t stretches_of(int cus) { return 2 * (int64_t)cus; }

template <typename T, int D, int kTiles>
hipError_t attend(const AttentionArgs& a, float* partials, int64_t wgs, hipStream_t stream) {
    asd_attend_kernel<T, D, kTiles><<<(unsigned)wgs, kAttendThreads, 0, stream>>>(a, partials);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || wgs < 2) return err;
    asd_attend_join_kernel<T, D, kTiles>
        <<<dim3((unsigned)(wgs - 1), kTiles), kAttendThreads, 0, stream>>>(a, partials, wgs);
    return hipGetLastError();
}

template <typename T>
hipError_t attend_any(const AttentionArgs& a, float* partials, int64_t wgs, int tiles, hipStream_t stream) {
    switch (a.b.cache.head_dim) {
        case 64:
            return tiles == 1 ? attend<T, 64, 1>(a, partials, wgs, stream)
                   : tiles == 2 ? attend<T, 64, 2>(a, partials, wgs, stream)
                                : attend<T, 64, 4>(a, partials, wgs, stream);
        case 128:
            return tiles == 1 ? attend<T, 128, 1>(a, partials, wgs, stream)
                   : tiles == 2 ? attend<T, 128, 2>(a, partials, wgs, stream)
                                : attend<T, 128, 4>(a, partials, wgs, stream);
        default:
            return tiles == 1 ? attend<T, 256, 1>(a, partials, wgs, stream)
                              : attend<T, 256, 2>(a, partials, wgs, stream);
    }
}

}  // namespace

size_t attention_workspace_bytes(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                 int32_t num_requests, int64_t total_rows, int cus) {
    if (num_requests == 0) return 0;
    const int tiles = tiles_of(num_q_heads, num_kv_heads, head_dim, num_requests, total_rows);
    return (size_t)(2 * stretches_of(cus)) * 16 * tiles * (head_dim + 2) * sizeof(float);
}

hipError_t launch_block_attention(const AttentionArgs& a, bool bf16, void* workspace, int cus,
                                  hipStream_t stream) {
    const asd_paged_cache& c = a.b.cache;
    const int tiles = tiles_of(a.num_q_heads, c.num_heads, c.head_dim, a.b.num_requests, a.b.total_rows);
    // no more stretches than units the batch can have
    const int64_t group = a.num_q_heads / c.num_heads;
    const __int128 items = (__int128)c.num_heads * (a.b.num_requests + a.b.total_rows * group / (16 * tiles));
    const __int128 units = items * (((int64_t)c.max_pages * c.page_size + kUnit - 1) / kUnit);
    int64_t wgs = stretches_of(cus);
    if (units < wgs) wgs = (int64_t)units;
    return bf16 ? attend_any<__bf16>(a, (float*)workspace, wgs, tiles, stream)
                : attend_any<_Float16>(a, (float*)workspace, wgs, tiles, stream);
}

}  // namespace asd
