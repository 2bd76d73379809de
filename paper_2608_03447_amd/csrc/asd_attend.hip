// gfx950 kernels of the attention of draft blocks and trees to the paged cache.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "asd_decode.h"
#include "asd_tokens.h"

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
// is finished at once.  Where an item's rows need several tiles, a team of
// workgroups takes one stretch together, a tile each, so that all but one of them
// find its keys and values in the L2.
//
// Bounds and measurements (128-element heads in bfloat16, 32 query heads to 8 key heads unless said):
//  - single tokens and blocks: the cache's bytes.  64 single tokens over up to 8,192: 217 us, 5.0 TB/s where a
//    plain read reaches 6.9; some 25 us of it are the batch's sharing out, each item's first loads and the
//    join.  9 rows over 65,000: 75 us for 266 MB, of it the join 11.  One token over 700: 12.2 us, a chain of
//    dependent loads (lengths, page table, keys, values) in two launches.
//  - trees: the vector unit between the two products and the matrix cores, which wait for it.  16 trees of 64
//    over 16,000, 64 query heads to 8: 830-870 us by the box, 620-650 TFLOP/s where a large matrix product reaches
//    1,150 to 1,400.  By counters a SIMD's matrix core is busy for 29% of its cycles, its vector unit for about half.
// A kernel of a workgroup per (row, head), one token at a time, took 13,309, 56,835, 466 and 476,524 us.

constexpr int kAttendThreads = 64 * kAttendWaves;
constexpr int32_t kMostTeam = 32;

// The same value in every lane, in scalar registers.
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int32_t)x) | (uint64_t)(uint32_t)uniform((int32_t)(x >> 32)) << 32);
}

// The same value, as the compiler sees it a new one: what is computed from it is not kept in registers
// from before the point where it is taken.
__device__ __forceinline__ int32_t fresh(int32_t x) {
    asm volatile("" : "+v"(x));
    return x;
}

// floor(a / b) of uniform 0 <= a < 2^53 and b > 0: a quotient in binary64, put right by one step at most.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    int64_t q = (int64_t)((double)a * (1.0 / (double)b));
    q -= q * b > a;
    return uniform(q + ((q + 1) * b <= a));
}

// Where a workgroup's stretch begins.
struct Where {
    int64_t id;         // the stretch, -1: there is none for this workgroup
    int32_t member;     // which of the stretch's workgroups this is
    int64_t per;        // units a stretch; the last one may have fewer
    int64_t total;      // units of the batch
    int64_t unit;       // the stretch's first unit, counted within its request
    int64_t row;        // that request's first row
    int64_t cached;
    int32_t request, count;
};

template <int kRows>
__device__ __forceinline__ int64_t units_of(const Blocks& b, int32_t group, int32_t team, int64_t row, int32_t count,
                                            int64_t cached, uint32_t& err) {
    const int64_t room = (int64_t)b.cache.max_pages * b.cache.page_size;
    const bool rows_ok = row >= 0 && row <= b.total_rows - count;
    const bool cache_ok = cached >= 0 && cached <= room - count;
    err |= (rows_ok ? 0u : kDecodeErrRows) | (cache_ok ? 0u : kDecodeErrCache);
    if (!rows_ok || !cache_ok) return 0;
    const int32_t tiles = (count * group + kRows - 1) / kRows, rounds = (tiles + team - 1) / team;
    return (int64_t)rounds * b.cache.num_heads * ((cached + count + kUnit - 1) / kUnit);
}

// Sum of v over the threads before this one, and over all of them.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* box, int64_t* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    long long sum = v;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const long long up = __shfl_up(sum, s);
        if (lane >= s) sum += up;
    }
    __syncthreads();
    if (lane == 63) box[wave] = sum;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) {
        before += w < wave ? box[w] : 0;
        all += box[w];
    }
    *total = all;
    return before + sum - v;
}

// Stretches there are to a request's key head, where these are few: the join of more takes longer than they
// save (51,325 tokens of one head of 64: 33 us with 64, 34 with 128, 40 with 32, 56 with as many as the card holds).
constexpr int kMostParts = 64;

// Equal stretches, the last one short.  Workgroups go to the XCDs in turn; those of a stretch,
// which read the same keys and values, go to one of them, and so do neighbouring stretches.
struct Shares {
    int64_t per;
    int32_t worker;     // -1: this workgroup has none
    __device__ __forceinline__ Shares(int64_t total, int64_t items, int32_t team) {
        const int64_t most = min((int64_t)(gridDim.x / team), items * kMostParts);
        per = total <= most ? 1 : quotient(total + most - 1, most);
        const int32_t used = (int32_t)(per == 1 ? total : quotient(total + per - 1, per)) * team;
        const int32_t eighth = (used + 7) / 8, at = (int32_t)(blockIdx.x >> 3);
        worker = (int32_t)(blockIdx.x & 7) * eighth + at;
        if (at >= eighth || worker >= used) worker = -1;
    }
};

// The same for up to 64 requests, every wavefront for itself, a lane a request: no barrier (1.2 us of a call).
template <int kRows>
__device__ __forceinline__ Where locate_few(const Blocks& b, int32_t group, int32_t team) {
    const int32_t n = b.num_requests, lane = threadIdx.x & 63;
    const bool in = lane < n;
    const int32_t k = in ? b.block_lens[lane] : 0, count = rows_of_block(k);
    const int64_t cached = in ? b.cache_lens[lane] : 0;
    const auto scan = [&](long long x) {
        for (int s = 1; s < n; s <<= 1) {
            const long long up = __shfl_up(x, s);
            if (lane >= s) x += up;
        }
        return (int64_t)x;
    };
    int64_t row = 0;
    if (b.row_offsets)
        row = in ? b.row_offsets[lane] : 0;
    else if (n > 1)
        row = scan(in ? count : 0) - count;
    uint32_t err = k < 0 ? kDecodeErrNegativeK : 0u;
    const int64_t units = in ? units_of<kRows>(b, group, team, row, count, cached, err) : 0;
    if (blockIdx.x == 0 && threadIdx.x < 64 && err != 0) atomicOr(b.error_word, err);
    const int64_t upto = scan(units), total = uniform((int64_t)__shfl((long long)upto, n - 1));
    const Shares shares(total, (int64_t)n * b.cache.num_heads, team);
    if (shares.worker < 0) return Where{-1, 0, 0, 0, 0, 0, 0, 0, 0};
    const int32_t id = shares.worker / team;
    const int64_t unit = id * shares.per;
    const int at = __builtin_ctzll(__ballot(in && unit < upto));
    const auto of = [&](int64_t x) { return uniform((int64_t)__shfl((long long)x, at)); };
    return Where{id,          shares.worker - id * team, shares.per, total, unit - of(upto - units), of(row),
                 of(cached), at,                        uniform(__shfl(count, at))};
}

// The workgroup's stretch: every thread sums its share of the requests (one, up to 256 requests),
// and the one whose share holds the stretch's first unit says where it is.
template <int kRows>
__device__ __forceinline__ Where locate(const Blocks& b, int32_t group, int32_t team, int64_t* box, Where* out) {
    const int32_t n = b.num_requests, per_thread = (n + kAttendThreads - 1) / kAttendThreads;
    const int32_t first = min(n, (int32_t)threadIdx.x * per_thread), last = min(n, first + per_thread);
    int64_t row = 0, unused, mine = 0;
    uint32_t err = 0;
    const int32_t k0 = first < last ? b.block_lens[first] : 0;
    const int64_t c0 = first < last ? b.cache_lens[first] : 0;
    if (!b.row_offsets) {
        for (int32_t i = first; i < last; ++i) mine += rows_of_block(i == first ? k0 : b.block_lens[i]);
        row = block_scan(mine, box, &unused);
    }
    int64_t units = 0, at = row;
    for (int32_t i = first; i < last; ++i) {
        const int32_t k = i == first ? k0 : b.block_lens[i], count = rows_of_block(k);
        err |= k < 0 ? kDecodeErrNegativeK : 0u;
        units += units_of<kRows>(b, group, team, b.row_offsets ? b.row_offsets[i] : at, count,
                                 i == first ? c0 : b.cache_lens[i], err);
        at += count;
    }
    if (blockIdx.x == 0 && err != 0) atomicOr(b.error_word, err);
    int64_t total;
    int64_t before = block_scan(units, box, &total);
    const Shares shares(total, (int64_t)n * b.cache.num_heads, team);
    if (shares.worker < 0) return Where{-1, 0, 0, 0, 0, 0, 0, 0, 0};
    const int32_t worker = shares.worker, id = worker / team;
    const int64_t per = shares.per, unit = id * per;
    if (unit >= before && unit < before + units) {
        for (int32_t i = first; i < last; ++i) {
            const int32_t count = rows_of_block(i == first ? k0 : b.block_lens[i]);
            const int64_t cached = i == first ? c0 : b.cache_lens[i];
            const int64_t at_row = b.row_offsets ? b.row_offsets[i] : row;
            const int64_t u = units_of<kRows>(b, group, team, at_row, count, cached, err);
            if (unit < before + u) {
                *out = Where{id, worker - id * team, per, total, unit - before, at_row, cached, i, count};
                break;
            }
            before += u;
            row += count;
        }
    }
    __syncthreads();
    return Where{uniform(out->id),   uniform(out->member), uniform(out->per),    uniform(out->total),  uniform(out->unit),
                 uniform(out->row), uniform(out->cached), uniform(out->request), uniform(out->count)};
}

// The item that the end of a workgroup's stretch cuts, if that stretch is its first: every
// workgroup writes one, those without a stretch too, since nothing else clears them.
struct alignas(32) Cut {
    int64_t row;        // the request's first row
    int32_t worker;     // stretch and workgroup of it, counted through
    int32_t head, first, pairs;
    int32_t parts;      // stretches that hold a part of the item, 0: it is not cut here
};

template <typename T> struct Half;
template <> struct Half<__bf16> {
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 mfma(x8 a, x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ float add(x2 a, float c) {
        return __builtin_amdgcn_fdot2_f32_bf16(a, x2{(__bf16)1.0f, (__bf16)1.0f}, c, false);
    }
    static constexpr uint32_t kExponent = 0x7f80u;
};
template <> struct Half<_Float16> {
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 mfma(x8 a, x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ float add(x2 a, float c) {
        return __builtin_amdgcn_fdot2(a, x2{(_Float16)1.0f, (_Float16)1.0f}, c, false);
    }
    static constexpr uint32_t kExponent = 0x7c00u;
};

// Workgroups that fit on a compute unit, by their registers and LDS.
constexpr int resident(int head_dim, int tiles) { return head_dim == 256 ? 1 : head_dim == 64 && tiles == 1 ? 3 : 2; }

// 64 lanes' 16 bytes each to LDS, from `lds` on; counted by vmcnt and waited for by the caller.
// (In asm since the compiler takes the builtin to write one lane's bytes alone and moves reads of
// the others' past it.  The s_nop: it does not see the address or m0 as just written.)
__device__ __forceinline__ void copy_to_lds(const char* src, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds), "v"(src) : "memory");
}

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
// Then the greatest is put at 2^kSet, which keeps weights down to 2^-20 of it normal in binary16 and those down to
// 2^-30 subnormal, rounded by 2^-31 of it at most.
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
// v_perm, so values never go through LDS, and O^T leaves every lane with D / 4
// neighbouring elements of its query row.  Keys do, copied there a strip ahead
// without passing through registers: a lane's part of a token is 16 bytes in
// each of D / 32 places, which as loads of their own fetched every line several times.
template <typename T, int D, int kTiles>
__global__ __launch_bounds__(kAttendThreads, resident(D, kTiles)) void asd_attend_kernel(AttentionArgs a, float* partials,
                                                                       Cut* cuts) {
    constexpr int kRows = 16 * kTiles, NC = D / 16, kSteps = D / 32, kVecs = (NC + 7) / 8;
    constexpr bool kQueriesInLds = kTiles > 2;
    typedef typename Half<T>::x8 x8;
    __shared__ int64_t box[kAttendWaves];
    __shared__ Where where_box;
    __shared__ int64_t offsets[kAttendWaves][2][kStrip];
    // a wavefront's keys of two strips; its rows of the join at an item's end
    constexpr int kKeyBytes = kStrip * D * 2;
    __shared__ __align__(16) char region[kAttendWaves][2 * kKeyBytes];
    float(*const joined)[sizeof(region[0]) / 4] = (float(*)[sizeof(region[0]) / 4])region;
    constexpr int kPitch = D + 4;
    static_assert(16 * kPitch * 4 <= 2 * kKeyBytes, "the join's rows fit");
    __shared__ float tops[kAttendWaves][16], sums[kAttendWaves][16];
    __shared__ int32_t row_p[kRows];                  // the block's row of every row of the tile
    __shared__ x8 queries[kQueriesInLds ? kTiles * kSteps * 64 : 1];

    const asd_paged_cache& cache = a.b.cache;
    const int32_t group = a.num_q_heads / cache.num_heads;
    Where at = a.b.num_requests <= 64 ? locate_few<kRows>(a.b, group, a.team)
                                      : locate<kRows>(a.b, group, a.team, box, &where_box);
    if (at.id < 0) {
        if (threadIdx.x == 0) cuts[blockIdx.x] = Cut{0, 0, 0, 0, 0, 0};
        return;
    }
    int64_t left = min(at.per, at.total - at.id * at.per);
    const int64_t worker = at.id * a.team + at.member;
    bool cut = false;
    // Scores enter as scale > 0: a negative scale turns the queries' signs, a zero one makes them zeros.
    const float per = __uint_as_float((uint32_t)uniform((int32_t)__float_as_uint(
        a.scale == 0.0f ? 1.0f : fabsf(a.scale) * 1.44269504f)));
    const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u, keep_q = a.scale == 0.0f ? 0u : ~0u;

    while (left > 0) {
        const int32_t count = at.count;
        const int64_t cached64 = at.cached;
        uint32_t unused = 0;
        if (units_of<kRows>(a.b, group, a.team, at.row, count, cached64, unused) <= at.unit) {
            // on to the next request
            at.row = a.b.row_offsets ? uniform(a.b.row_offsets[at.request + 1]) : at.row + count;
            at.request += 1;
            at.count = uniform(rows_of_block(a.b.block_lens[at.request]));
            at.cached = uniform(a.b.cache_lens[at.request]);
            at.unit = 0;
            continue;
        }
        const int32_t pairs = count * group, tiles = (pairs + kRows - 1) / kRows;
        const int64_t units = (cached64 + count + kUnit - 1) / kUnit;
        const int64_t item = at.unit < units ? 0 : quotient(at.unit, units), from = at.unit - item * units;
        const int64_t to = from + left < units ? from + left : units;
        const int32_t rounds = (tiles + a.team - 1) / a.team, head = (int32_t)item / rounds;
        const int32_t mine = ((int32_t)item - head * rounds) * a.team + at.member, first = mine * kRows;      // of the pairs
        at.unit += to - from;
        left -= to - from;
        if (mine >= tiles) continue;
        const bool complete = from == 0 && to == units;
        if (from == 0 && !complete) {           // the stretch ends here
            cut = true;
            if (threadIdx.x == 0)
                cuts[blockIdx.x] = Cut{at.row, (int32_t)worker, head, first, pairs,
                                       1 + (int32_t)quotient(units - to + at.per - 1, at.per)};
        }

        const int tid = fresh(threadIdx.x), lane = tid & 63, wave = uniform(tid >> 6), n = lane & 15, g = lane >> 4;
        // the tile's queries: B operands, lane n's row, 8 elements of every 32
        const auto query = [&](int tile, int step) -> x8 {
            const int32_t m = first + 16 * tile + n;
            if (m >= pairs) return x8{};
            const int32_t p = m / group;
            const u32x4 x = *(const u32x4*)((const T*)a.q + (at.row + p) * a.q_stride +
                                            (head * group + m - p * group) * D + 32 * step + 8 * g);
            return __builtin_bit_cast(x8, (x ^ flip) & keep_q);
        };
        x8 q[kQueriesInLds ? 1 : kTiles][kSteps];
        __syncthreads();
        if (tid < kRows) row_p[tid] = min(first + tid, pairs - 1) / group;
        if constexpr (kQueriesInLds) {
            for (int tile = wave; tile < kTiles; tile += kAttendWaves)
                #pragma unroll
                for (int step = 0; step < kSteps; ++step)
                    queries[(tile * kSteps + step) * 64 + lane] = query(tile, step);
        } else {
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
                for (int step = 0; step < kSteps; ++step) q[tile][step] = query(tile, step);
        }
        __syncthreads();

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
        const int32_t cached = (int32_t)cached64;
        const Tokens tokens{(Token)(cached + count), (uint32_t)cache.page_size, a.page_magic, a.page_shift};
        const int32_t last_p = uniform(row_p[kRows - 1]);
        const int32_t end = a.mask ? (int32_t)tokens.end : cached + last_p + 1;
        const Token strip_end = (Token)min(to * kUnit, (int64_t)end);
        Token strip = (Token)(from * kUnit) + wave * kStrip;
        const int32_t* const table = cache.page_table + (int64_t)at.request * cache.max_pages;
        const char* const keys = (const char*)((const T*)cache.keys + (int64_t)head * cache.head_stride ); 
        const char* const values = (const char*)((const T*)cache.values + (int64_t)head * cache.head_stride + NC * n);

        // A strip's page ids (lanes l and l + 32 hold token l; tokens behind the last one take
        // its page) and, from them, its tokens' byte offsets in LDS; the mask of the tokens that
        // are there, the others' offsets being 0.
        const auto page_of = [&](Token t0) -> int32_t { return table[tokens.entry(t0 + (lane & 31))]; };
        const auto put_offsets = [&](int b, Token t0, int32_t page) -> uint32_t {
            const Token t = t0 + (lane & 31);
            const bool ok = tokens.has(t) && (uint32_t)page < (uint32_t)cache.num_pages;
            const int64_t off = ((int64_t)page * cache.page_stride + (int64_t)tokens.slot(t) * cache.token_stride) * 2;
            wave_sync();
            if (lane < 32) offsets[wave][b][lane] = ok ? off : 0;
            wave_sync();
            return (uint32_t)__ballot(ok);
        };
        u32x4 v[8][kVecs];
        // Keys go to LDS as they lie in memory, D / 8 lanes a token, so that 16 lanes read whole lines
        // (16 tokens' pieces of 16 bytes, as the operand wants them, cost the L1 64 lookups an instruction:
        // 64 single tokens over up to 8,192 took 226 us); a token's pieces of 16 bytes are
        // turned by its number, so that the operand's reads of 16 tokens meet no bank twice.
        constexpr int kLanes = D / 8, kAtOnce = 64 / kLanes, kTurn = D == 64 ? 1 : 0, kTurns = D == 64 ? 7 : 15;
        const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)region[wave];
        const auto load_keys = [&](int b) {
            const int r0 = lane / kLanes, piece = lane % kLanes;
#pragma unroll
            for (int i = 0; i < kStrip / kAtOnce; ++i) {
                const int r = kAtOnce * i + r0;
                copy_to_lds(keys + offsets[wave][b][r] + 16 * (piece ^ (r >> kTurn & kTurns)),
                            lds + b * kKeyBytes + 1024 * i);
            }
        };
        const auto key = [&](int b, int h, int step) -> x8 {
            return *(const x8*)(region[wave] + b * kKeyBytes + (16 * h + n) * (2 * D) +
                                16 * ((4 * step + g) ^ (n >> kTurn & kTurns)));
        };
        const auto load_values = [&](int b) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const char* src = values + offsets[wave][b][(j & 3) + 4 * g + 16 * (j >> 2)];
                if constexpr (NC == 4) {
                    const u32x2 w = *(const u32x2*)src;
                    v[j][0].x = w.x;
                    v[j][0].y = w.y;
                } else {
#pragma unroll
                    for (int x = 0; x < kVecs; ++x) v[j][x] = *(const u32x4*)(src + 16 * x);
                }
            }
        };
        // Scores and weights of a strip; a lane's row of tile i sees the tokens of bits 8 i.. of `seen`.
        x8 w[kTiles];
        const auto weigh = [&](int b, bool all, uint32_t seen) {
            f32x4 s[kTiles][2];
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile) s[tile][0] = s[tile][1] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int step = 0; step < kSteps; ++step) {
                const x8 k[2] = {key(b, 0, step), key(b, 1, step)};
#pragma unroll
                for (int tile = 0; tile < kTiles; ++tile) {
                    x8 qq;
                    if constexpr (kQueriesInLds) qq = queries[(tile * kSteps + step) * 64 + lane];
                    else qq = q[tile][step];
#pragma unroll
                    for (int h = 0; h < 2; ++h) s[tile][h] = Half<T>::mfma(k[h], qq, s[tile][h]);
                }
            }
            float top[kTiles];
            bool moves = false;
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile) {
                if (!all) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (!((seen >> (8 * tile + j)) & 1)) s[tile][j >> 2][j & 3] = -INFINITY;
                }
                const f32x4 x = s[tile][0], y = s[tile][1];
                top[tile] = rows_max(fmaxf(fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w)),
                                           fmaxf(fmaxf(y.x, y.y), fmaxf(y.z, y.w)))) * per;
                moves |= top[tile] > ref[tile] + kLead;
            }
            if (__any(moves)) {
#pragma unroll
                for (int tile = 0; tile < kTiles; ++tile) {
                    const float now = top[tile] > ref[tile] + kLead ? top[tile] - kSet : ref[tile];
                    const float keep = now == ref[tile] ? 1.0f : __builtin_amdgcn_exp2f(ref[tile] - now);
                    ref[tile] = now;
                    sum[tile] *= keep;
#pragma unroll
                    for (int c = 0; c < NC; ++c) o[tile][c] *= keep;
                }
            }
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile) {
                const float from_ref = ref[tile] == -INFINITY ? 0.0f : ref[tile];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    w[tile][j] = (T)__builtin_amdgcn_exp2f(fmaf(s[tile][j >> 2][j & 3], per, -from_ref));
                // The weights are rounded to T, as the matrix cores take them, and the sum is that of the rounded
                // ones: a row is then off by half a step of T times how far its values lie apart, and equal values
                // come out as they are (summed unrounded, ragged blocks in binary16 were off by 0.0017 at most, by
                // 0.0007 so).  The dot products with ones, which round down, add up a strip's eight alone; converted
                // back and added one by one the weights cost 5% of a call on trees.
                float strip_sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; j += 2)
                    strip_sum = Half<T>::add(typename Half<T>::x2{w[tile][j], w[tile][j + 1]}, strip_sum);
                sum[tile] += strip_sum;
            }
        };
        const auto add_values = [&]() {
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
        };

        // While a strip's scores are formed, its values and the next strip's keys are on the way, and
        // the page ids of the one after it.  Loads return in order and the next keys are
        // asked for before this strip's values, so that they are in once these are used, with no wait
        // of their own.  (Strips behind the last one load what offset 0 holds, for nothing.)
        uint32_t valid = 0, ahead = 0;
        int b = 0;
        if (strip < strip_end) {
            const int32_t page = page_of(strip), next = page_of(strip + kUnit);
            valid = put_offsets(0, strip, page);
            load_keys(0);
            ahead = put_offsets(1, strip + kUnit, next);
            load_keys(1);
            load_values(0);
            asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kStrip / kAtOnce + 8 * kVecs) : "memory");
        }
        // Strips that every row sees whole.
        while (strip < strip_end && valid == ~0u && strip + kStrip <= (Token)cached) {
            const int32_t after = page_of(strip + 2 * kUnit);
            weigh(b, true, 0);
            add_values();
            asm volatile("s_waitcnt vmcnt(1)" ::: "memory");       // all but `after`: waited for by its uses already
            strip += kUnit;
            valid = ahead;
            ahead = put_offsets(b, strip + kUnit, after);
            load_keys(b);
            b ^= 1;
            load_values(b);
        }
        // The others: the block's own tokens, the strip that the sequence ends in, bad pages.
#pragma unroll 1
        while (strip < strip_end) {
            if (lane < 32 && tokens.has(strip + lane) && !((valid >> lane) & 1))
                atomicOr(a.b.error_word, kDecodeErrCache);
            // the tokens that each tile's row sees, a bit each: cached ones, and the block's by the mask
            uint32_t window[kTiles];
            const int32_t past = (int32_t)strip - cached;         // the block's first token; negative: before it
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile) {
                const int32_t p = row_p[16 * tile + n];
                if (a.mask) {
                    const uint64_t* const words = a.mask + (at.row + p) * a.mask_words;
                    const int32_t x = max(past, 0), at_word = x >> 6, bit = x & 63;
                    uint64_t bits = 0;
                    if (at_word < a.mask_words) bits = words[at_word] >> bit;
                    if (bit > 32 && at_word + 1 < a.mask_words) bits |= words[at_word + 1] << (64 - bit);
                    const int32_t before = min(max(-past, 0), 32);
                    window[tile] = (uint32_t)(bits << before) | (uint32_t)((1ull << before) - 1);
                } else {
                    window[tile] = (uint32_t)((1ull << chain_sees(p, past)) - 1);
                }
            }
            // of the lane's 8 tokens: which its rows see, 8 bits a tile, and which are there at all
            const auto mine = [&](uint32_t x) { return (x >> (4 * g) & 0xf) | (x >> (16 + 4 * g) & 0xf) << 4; };
            const uint32_t there = mine(valid);
            uint32_t seen = 0;
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile) seen |= mine(window[tile] & valid) << (8 * tile);
            weigh(b, false, seen);

            // Values that are not there are zeros.  A token that holds an infinity or a NaN
            // would reach every row through its weight 0: it leaves the product and is added by
            // hand to the rows that see it.
            uint32_t odd = 0;
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
            add_values();
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (odd != 0) {
                float* const special_weights = (float*)(region[wave] + b * kKeyBytes);     // its keys are used
#pragma unroll
                for (int tile = 0; tile < kTiles; ++tile) {
                    wave_sync();
#pragma unroll
                    for (int j = 0; j < 8; ++j)       // -1: not seen
                        special_weights[n * (kStrip + 1) + (j & 3) + 4 * g + 16 * (j >> 2)] =
                            (seen >> (8 * tile + j)) & 1 ? (float)w[tile][j] : -1.0f;
                    wave_sync();
#pragma unroll 1
                    for (uint32_t rest = odd; rest != 0; rest &= rest - 1) {
                        const int32_t at_strip = __builtin_ctz(rest);
                        const float weight = special_weights[n * (kStrip + 1) + at_strip];
                        if (weight == -1.0f) continue;
                        const T* src = (const T*)(values - 2 * NC * n + offsets[wave][b][at_strip]) + 4 * NC * g;
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int c = 0; c < NC; ++c)
                                o[tile][c][r] = fmaf(weight, (float)src[NC * r + c], o[tile][c][r]);
                    }
                }
            }
            strip += kUnit;
            valid = ahead;
            if (strip < strip_end) {
                ahead = put_offsets(b, strip + kUnit, page_of(strip + kUnit));
                load_keys(b);
            }
            b ^= 1;
            if (strip < strip_end) load_values(b);
        }
        // (keys loaded ahead for nothing have to be in before their place is used again)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

        // the wavefronts' sums, joined tile by tile
        const int tid_end = fresh(tid), n_end = tid_end & 15, g_end = tid_end >> 4 & 3, row = tid_end >> 4;
        float* const slot = partials + (2 * worker + (from > 0 ? 0 : 1)) * (int64_t)(kRows * (D + 2));
        #pragma unroll
        for (int tile = 0; tile < kTiles; ++tile) {
            sum[tile] = rows_sum(sum[tile]);
            if (ref[tile] == -INFINITY && sum[tile] != sum[tile]) ref[tile] = 0.0f;   // every score a NaN
            __syncthreads();
            if (g_end == 0) {
                tops[wave][n_end] = ref[tile];
                sums[wave][n_end] = sum[tile];
            }
            __syncthreads();
            float best = tops[0][n_end];
            #pragma unroll
            for (int w = 1; w < kAttendWaves; ++w) best = fmaxf(best, tops[w][n_end]);
            const float mine = ref[tile] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref[tile] - best);
            #pragma unroll
            for (int r = 0; r < 4; ++r)
                #pragma unroll
                for (int c = 0; c < NC; c += 4)
                    *(f32x4*)&joined[wave][n_end * kPitch + 4 * NC * g_end + NC * r + c] =
                        f32x4{o[tile][c][r], o[tile][c + 1][r], o[tile][c + 2][r], o[tile][c + 3][r]} * mine;
            __syncthreads();
            // 16 threads a row, each every 16th vector of 4 elements
            best = tops[0][row];
            #pragma unroll
            for (int w = 1; w < kAttendWaves; ++w) best = fmaxf(best, tops[w][row]);
            float total = 0.0f;
            #pragma unroll
            for (int w = 0; w < kAttendWaves; ++w)
                total += tops[w][row] == -INFINITY ? 0.0f
                                                   : sums[w][row] * __builtin_amdgcn_exp2f(tops[w][row] - best);
            const int32_t m = first + 16 * tile + row;
            if (!complete && n_end == 0 && m < pairs) {
                slot[kRows * D + 16 * tile + row] = best;
                slot[kRows * (D + 1) + 16 * tile + row] = total;
            }
            const int32_t p = row_p[16 * tile + row];
            const float over = best == -INFINITY ? 0.0f : 1.0f / total;
            for (int e = 4 * n_end; e < D; e += 64) {
                f32x4 x = *(const f32x4*)&joined[0][row * kPitch + e];
                #pragma unroll
                for (int w = 1; w < kAttendWaves; ++w) x += *(const f32x4*)&joined[w][row * kPitch + e];
                if (m >= pairs) break;
                if (!complete) {
                    *(f32x4*)&slot[(16 * tile + row) * D + e] = x;
                } else {
                    T* dst = (T*)a.out + ((at.row + p) * a.num_q_heads + head * group + m - p * group) * D + e;
                    typename Half<T>::x2 y[2];
                    #pragma unroll
                    for (int z = 0; z < 4; ++z) y[z / 2][z % 2] = (T)(x[z] * over);
                    *(u32x2*)dst = u32x2{__builtin_bit_cast(uint32_t, y[0]), __builtin_bit_cast(uint32_t, y[1])};
                }
            }
        }
        __syncthreads();
    }
    if (threadIdx.x == 0 && !cut) cuts[blockIdx.x] = Cut{0, 0, 0, 0, 0, 0};
}

// Joins the partials of the item that is cut by the end of workgroup blockIdx.x's stretch, if one is; a
// workgroup takes four of its rows.  Few parts are loaded all at once by a wavefront a row; of many, kSplit
// wavefronts a row take a share each.  Four are launched where there are so few items that they have many parts
// (64 parts of 36 rows: 11 us, 17 with one); one elsewhere, where most of them would find nothing to do
// (32 blocks over short caches: 8 us, 14 with four).
constexpr int kFewParts = 8, kPartsAhead = 16, kJoinRows = 4;
template <typename T, int D, int kTiles, int kSplit>
__global__ __launch_bounds__(kJoinRows * kSplit * 64) void asd_attend_join_kernel(AttentionArgs a, const float* partials,
                                                                                 const Cut* cuts) {
    constexpr int kRows = 16 * kTiles, kPer = D / 64;
    constexpr int64_t kSize = (int64_t)kRows * (D + 2);
    __shared__ float sums[kSplit][kJoinRows][D + 2];
    const int lane = threadIdx.x & 63, wave = uniform((int32_t)threadIdx.x >> 6);
    const Cut cut = cuts[blockIdx.x];
    if (cut.parts == 0) return;
    const int64_t worker = cut.worker;
    const int32_t group = a.num_q_heads / a.b.cache.num_heads;
    const auto part = [&](int j) { return partials + (2 * (worker + (int64_t)j * a.team) + (j == 0 ? 1 : 0)) * kSize; };
    const auto row_of = [&](int32_t m) {
        const int32_t p = m / group;
        return (T*)a.out + ((cut.row + p) * a.num_q_heads + cut.head * group + m - p * group) * D;
    };
    const int row = (int)blockIdx.y * kJoinRows + (wave & (kJoinRows - 1)), split = wave / kJoinRows;
    const int32_t m = cut.first + row;
    if (cut.parts <= kFewParts) {
        if (m >= cut.pairs || split > 0) return;
        float top[kFewParts], o[kPer];
        float best = -INFINITY, total = 0.0f;
#pragma unroll
        for (int j = 0; j < kFewParts; ++j) {
            top[j] = j < cut.parts ? part(j)[kRows * D + row] : -INFINITY;
            best = fmaxf(best, top[j]);
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] = 0.0f;
#pragma unroll
        for (int j = 0; j < kFewParts; ++j) {
            if (j >= cut.parts) break;
            const float f = top[j] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top[j] - best);
            const float* x = part(j);
            total = fmaf(f, x[kRows * (D + 1) + row], total);
#pragma unroll
            for (int e = 0; e < kPer; ++e) o[e] = fmaf(f, x[row * D + kPer * lane + e], o[e]);
        }
        const float over = best == -INFINITY ? 0.0f : 1.0f / total;
        T* dst = row_of(m);
#pragma unroll
        for (int e = 0; e < kPer; ++e) dst[kPer * lane + e] = (T)(o[e] * over);
        return;
    }
    float best = -INFINITY, total = 0.0f, o[kPer];
    const int32_t from = m < cut.pairs ? cut.parts * split / kSplit : 0;
    const int32_t to = m < cut.pairs ? cut.parts * (split + 1) / kSplit : 0;
    for (int32_t j = from + lane; j < to; j += 64) best = fmaxf(best, part(j)[kRows * D + row]);
    for (int s = 32; s > 0; s >>= 1) best = fmaxf(best, __shfl_xor(best, s));
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] = 0.0f;
    for (int32_t j0 = from; j0 < to; j0 += 64) {
        const int32_t here = min(64, to - j0);
        float f = 0.0f;
        if (lane < here) {
            const float* x = part(j0 + lane);
            const float top = x[kRows * D + row];
            f = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - best);
            total = fmaf(f, x[kRows * (D + 1) + row], total);
        }
        for (int32_t x = 0; x < here; x += kPartsAhead) {
            float y[kPartsAhead][kPer];
#pragma unroll
            for (int c = 0; c < kPartsAhead; ++c) {
                const float* from = part(j0 + min(x + c, here - 1)) + row * D + kPer * lane;
#pragma unroll
                for (int e = 0; e < kPer; ++e) y[c][e] = from[e];
            }
#pragma unroll
            for (int c = 0; c < kPartsAhead; ++c) {
                const float weight = __shfl(f, min(x + c, 63));
#pragma unroll
                for (int e = 0; e < kPer; ++e) o[e] = fmaf(weight, x + c < here ? y[c][e] : 0.0f, o[e]);
            }
        }
    }
    for (int s = 32; s > 0; s >>= 1) total += __shfl_xor(total, s);
    float* const mine = &sums[split][wave & (kJoinRows - 1)][0];
#pragma unroll
    for (int e = 0; e < kPer; ++e) mine[kPer * lane + e] = o[e];
    if (lane == 0) {
        mine[D] = best;
        mine[D + 1] = total;
    }
    __syncthreads();
    if (split > 0 || m >= cut.pairs) return;
    float all = -INFINITY;
#pragma unroll
    for (int x = 0; x < kSplit; ++x) all = fmaxf(all, sums[x][wave][D]);
    total = 0.0f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] = 0.0f;
#pragma unroll
    for (int x = 0; x < kSplit; ++x) {
        const float top = sums[x][wave][D], f = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - all);
        total = fmaf(f, sums[x][wave][D + 1], total);
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] = fmaf(f, sums[x][wave][kPer * lane + e], o[e]);
    }
    const float over = all == -INFINITY ? 0.0f : 1.0f / total;
    T* dst = row_of(m);
#pragma unroll
    for (int e = 0; e < kPer; ++e) dst[kPer * lane + e] = (T)(o[e] * over);
}

}  // namespace

namespace {

// 16-row tiles of an item: the (row, head) pairs of an average block spread evenly over the fewest
// items, of as many tiles as the registers hold.
int tiles_of(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t num_requests,
             int64_t total_rows) {
    const int64_t most = head_dim == 64 ? 4 : head_dim == 128 ? 3 : 2;
    const int64_t pairs = (total_rows + num_requests - 1) / num_requests * (num_q_heads / num_kv_heads);
    const int64_t tiles = (pairs + 15) / 16, items = (tiles + most - 1) / most;
    return (int)((tiles + items - 1) / items);
}

// Workgroups of a stretch: one for every tile of an average block, all of which read its keys and
// values at the same time, up to those that an XCD holds.
int32_t team_of(int32_t num_q_heads, int32_t num_kv_heads, int32_t num_requests, int64_t total_rows, int tiles) {
    const int64_t pairs = (total_rows + num_requests - 1) / num_requests * (num_q_heads / num_kv_heads);
    const int64_t items = (pairs + 16 * tiles - 1) / (16 * tiles);
    return (int32_t)(items < kMostTeam ? items : kMostTeam);
}

size_t partial_bytes(int64_t wgs, int head_dim, int tiles) {
    return (size_t)(2 * wgs) * 16 * tiles * (head_dim + 2) * sizeof(float);
}

template <typename T, int D, int kTiles>
hipError_t attend(const AttentionArgs& a, void* workspace, int64_t wgs, hipStream_t stream) {
    float* const partials = (float*)workspace;
    Cut* const cuts = (Cut*)((char*)workspace + partial_bytes(wgs, D, kTiles));
    asd_attend_kernel<T, D, kTiles><<<(unsigned)wgs, kAttendThreads, 0, stream>>>(a, partials, cuts);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    const dim3 grid((unsigned)wgs, 16 * kTiles / kJoinRows);
    const int64_t items = (int64_t)a.b.num_requests * a.b.cache.num_heads;
    if (2 * kFewParts * items * a.team <= wgs)
        asd_attend_join_kernel<T, D, kTiles, 4><<<grid, kJoinRows * 4 * 64, 0, stream>>>(a, partials, cuts);
    else
        asd_attend_join_kernel<T, D, kTiles, 1><<<grid, kJoinRows * 64, 0, stream>>>(a, partials, cuts);
    return hipGetLastError();
}

template <typename T>
hipError_t attend_any(const AttentionArgs& a, void* workspace, int64_t wgs, int tiles, hipStream_t stream) {
    const int d = a.b.cache.head_dim;
    switch (tiles) {
        case 1:
            return d == 64    ? attend<T, 64, 1>(a, workspace, wgs, stream)
                   : d == 128 ? attend<T, 128, 1>(a, workspace, wgs, stream)
                              : attend<T, 256, 1>(a, workspace, wgs, stream);
        case 2:
            return d == 64    ? attend<T, 64, 2>(a, workspace, wgs, stream)
                   : d == 128 ? attend<T, 128, 2>(a, workspace, wgs, stream)
                              : attend<T, 256, 2>(a, workspace, wgs, stream);
        case 3:
            return d == 64 ? attend<T, 64, 3>(a, workspace, wgs, stream)
                           : attend<T, 128, 3>(a, workspace, wgs, stream);
        default: return attend<T, 64, 4>(a, workspace, wgs, stream);
    }
}

}  // namespace

size_t attention_workspace_bytes(int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                 int32_t num_requests, int64_t total_rows, int cus) {
    if (num_requests == 0) return 0;
    const int tiles = tiles_of(num_q_heads, num_kv_heads, head_dim, num_requests, total_rows);
    const int64_t wgs = (int64_t)cus * resident(head_dim, tiles);
    return partial_bytes(wgs, head_dim, tiles) + (size_t)wgs * sizeof(Cut);
}

hipError_t launch_block_attention(const AttentionArgs& a, bool bf16, void* workspace, int cus,
                                  hipStream_t stream) {
    const asd_paged_cache& c = a.b.cache;
    AttentionArgs b = a;
    page_divisor(c.page_size, &b.page_magic, &b.page_shift);
    const int tiles = tiles_of(a.num_q_heads, c.num_heads, c.head_dim, a.b.num_requests, a.b.total_rows);
    const int64_t wgs = (int64_t)cus * resident(c.head_dim, tiles);
    b.team = team_of(a.num_q_heads, c.num_heads, a.b.num_requests, a.b.total_rows, tiles);
    return bf16 ? attend_any<__bf16>(b, workspace, wgs, tiles, stream)
                : attend_any<_Float16>(b, workspace, wgs, tiles, stream);
}

}  // namespace asd
