// gfx950 kernels that draw a token from every logit row.
//
// Nothing is sorted as a whole: the running sum of the draw is taken in index order, and what the filters cut is
// found among the few tokens next to the cut.
//
// Pass 1 (scan) reads every row once from HBM, a wavefront a group of 1,024 logits at a
// time, and leaves the greatest logit of every 64 (a sub-block) and, for rows whose whole mass counts, the
// group's sum of exp((z - its greatest) / T) in binary64.
//
// Pass 2 (pick), a workgroup a row, works on those: without filters the draw falls into one group, which is
// read again; with them, a threshold that as many sub-block maxima reach as tokens are wanted bounds the
// candidates from below, only the sub-blocks whose maximum reaches it are read again, and the filters' cuts
// are found among the candidates, up to 2,048, by their order.
//
// Rows that keep more tokens than that (a nucleus of tens of thousands) are read again in parts by all workgroups: pass
// 3 sums their weights, coarsely, by bins of the logit, pass 4 lists the tokens of the bin that holds the cut and sums,
// group by group, what lies above it, and pass 5 (finish) finds the cut among the listed and draws.  Pass 6 (flat), one
// workgroup a row, takes what is left: calls too small for passes 3 to 5, top-k beyond 1,920, bins of more
// ties than a list holds, cuts that the coarse sums put into another bin than the exact ones.
//
// A sum in a fixed order is binary64; one whose order the hardware chooses is of whole numbers (Mass, Coarse).
//
// Bounds and measurements: pass 1 is memory's and the binary64 exponentials'; 2,112 rows of 151,936 float32
// (1.28 GB) take 267 us, 4.8 TB/s.  Pass 2 is latency and, with 1,400 candidates, arithmetic: 12 us for
// one row of 32,000 with top-k 50, 36 with top-k 1,000 of 129,280, 105 for the 2,112.  Passes 3 and 4 are
// the exponentials': 69 and 77 us for some 480 flat rows of the 2,112, 9 and 13 for 15 rows of 129,280 in bfloat16;
// pass 5 22 and 11 to 18.  In all 526-545 us by the box, 84-87 us for 67 rows of 129,280, 16.8 for one of 32,000 (a
// bisection over each row by one workgroup took 7,165, 584 and 202).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "asd_decode.h"

namespace asd {
namespace {

typedef unsigned long long u64;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kGroup = 1024, kSub = 64, kSubs = kGroup / kSub;

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
constexpr uint32_t kKeyNegInf = 0x007fffffu, kKeyInf = 0xff800000u, kKeyNan = 0xffffffffu;

// 2^x for x <= 0, to 2^-47: the Taylor polynomial of degree 11 of 2^r, |r| <= 1/2
// (the next term is (ln 2 / 2)^12 / 12! = 6e-15).  2^0 is 1 exactly; x below -1000 gives 2^-1000.
// Adding 1.5 2^52 rounds x to a whole number, which stands in the sum's low bits and goes into
// the result's exponent by one integer addition: conversions and ldexp run at a quarter of the rate.
__device__ __forceinline__ double power2_clamped(double x) {
    constexpr double kRound = 6755399441055744.0;
    x = fmax(x, -1000.0);
    const double t = x + kRound, r = x - (t - kRound);
    double p = 4.4455382718708114e-10;                 // ln(2)^k / k!, k = 11 .. 1
    p = fma(p, r, 7.0549116208011232e-09);
    p = fma(p, r, 1.0178086009239700e-07);
    p = fma(p, r, 1.3215486790144309e-06);
    p = fma(p, r, 1.5252733804059840e-05);
    p = fma(p, r, 1.5403530393381609e-04);
    p = fma(p, r, 1.3333558146428443e-03);
    p = fma(p, r, 9.6181291076284771e-03);
    p = fma(p, r, 5.5504108664821580e-02);
    p = fma(p, r, 2.4022650695910071e-01);
    p = fma(p, r, 6.9314718055994531e-01);
    p = fma(p, r, 1.0);
    const u64 bits = __builtin_bit_cast(u64, p);
    return __builtin_bit_cast(double, (u64)((uint32_t)(bits >> 32) + ((uint32_t)__builtin_bit_cast(u64, t) << 20)) << 32 |
                                          (uint32_t)bits);
}

// A row's weights, exp((z - top) / T).
struct Weights {
    double top, per;       // log2(e) / T
    float top_f;
    __device__ __forceinline__ Weights(float greatest, float t)
        : top((double)greatest), per(1.44269504088896340736 / (double)t), top_f(greatest) {}
    __device__ __forceinline__ double operator()(float z) const {
        const double x = ((double)z - top) * per, w = power2_clamped(x);
        return z == top_f ? 1.0 : !(x >= -1000.0) || z == -INFINITY || top_f == INFINITY ? 0.0 : w;
    }
};

// A sum of weights in whole numbers of 2^-64 of the greatest, so that it is the same in any order: `high` counts
// 2^-32 and `low`, which has a sign, 2^-64.  A weight adds 2^32 and 2^31 at most, so that the sums of 2^30 fit.
typedef unsigned __int128 u128;
struct Mass {
    u64 high, low;
    __device__ __forceinline__ Mass operator+(const Mass& o) const { return {high + o.high, low + o.low}; }
    __device__ __forceinline__ Mass operator-(const Mass& o) const { return {high - o.high, low - o.low}; }
    __device__ __forceinline__ Mass operator*(u64 n) const { return {high * n, low * n}; }
    __device__ __forceinline__ void operator+=(const Mass& o) { *this = *this + o; }
    __device__ __forceinline__ u128 value() const { return ((u128)high << 32) + (u128)(__int128)(long long)low; }
};
// A weight added to 2^20 is rounded to a multiple of 2^-32, which then stands in the sum's low bits; what it was
// rounded by, exact, gives the rest the same way.
__device__ __forceinline__ Mass mass_of(double weight) {
    constexpr double kHigh = 0x1p20, kLow = 0x1.8p-12;
    const double t = weight + kHigh, r = (weight - (t - kHigh)) + kLow;
    return {__builtin_bit_cast(u64, t) - __builtin_bit_cast(u64, kHigh),
            __builtin_bit_cast(u64, r) - __builtin_bit_cast(u64, kLow)};
}
__device__ __forceinline__ double real_of(u128 units) {
    return (double)(u64)(units >> 32) * 0x1p-32 + (double)(uint32_t)units * 0x1p-64;
}
// ceil(x 2^64) for 0 <= x < 2^30.
__device__ __forceinline__ u128 units_of(double x) {
    const double high = floor(x * 0x1p32);
    return ((u128)(u64)high << 32) + (u64)ceil((x * 0x1p32 - high) * 0x1p32);
}
__device__ __forceinline__ void add_to(u64* high, u64* low, const Mass& m) {
    atomicAdd(high, m.high);
    atomicAdd(low, m.low);
}

// Row parameters.
struct Row {
    float t, p, m;
    int32_t k;
    bool greedy, by_count, by_mass, by_floor;
    __device__ __forceinline__ Row(const SampleArgs& a, int64_t row) {
        t = a.temperature ? a.temperature[row] : 1.0f;
        k = a.top_k ? a.top_k[row] : 0;
        p = a.top_p ? a.top_p[row] : 1.0f;
        m = a.min_p ? a.min_p[row] : 0.0f;
        greedy = !(t > 0.0f);
        by_count = k > 0 && k < a.vocab;
        by_mass = p < 1.0f;
        by_floor = m > 0.0f;
        m = m < 1.0f ? m : 1.0f;
    }
};

// Rows that pass 2 leaves: to one workgroup each, or to be read in parts by many.
enum { kAlone = 0, kShared = 1 };

// A shared row's bins: of one width in the logit, counted up to the last one, which all from `high` on are in.
constexpr int kNearBins = 1024;
struct Near {
    float high, steps;     // steps: bins to a unit of the logit
    uint32_t top;          // key of the greatest logit
    uint32_t collected;    // tokens of the cut's bin that pass 4 listed, in the place of the row's sub-blocks
    double all;            // the row's mass
    Mass above;            // of the tokens above that bin
    __device__ __forceinline__ uint32_t bin(float x) const {
        return (uint32_t)(kNearBins - 1) - (uint32_t)fminf(fmaxf((high - x) * steps, 0.0f), (float)(kNearBins - 1));
    }
};

// What pass 1 leaves of a row: keys of its sub-blocks' maxima, keys and sums of its groups.
struct Stats {
    uint32_t* subs;        // [rows][groups * kSubs]
    uint32_t* tops;        // [rows][groups]
    double* sums;          // [rows][groups]
    uint32_t* queued;      // [2]: rows that pass 2 leaves, by kAlone and kShared,
    int32_t* queue[2];     // [rows]: and which
    int32_t groups;        // of the row that has most: its first vector may begin before it
    // where rows are shared out (shares_out), else null:
    Near* near;            // [rows]
    u64* bins;             // [rows][kNearBins]: weights by their bin
};

__device__ __forceinline__ void enqueue(const Stats& s, int to, int64_t row) {
    s.queue[to][atomicAdd(s.queued + to, 1u)] = (int32_t)row;
}

// A row as 16-byte vectors: its elements stand `shift` places behind the vector grid's origin.
template <typename T> struct Grid {
    const T* origin;       // 16-byte aligned, at most 15 bytes before the row
    int32_t shift;
    int64_t vocab;
    __device__ __forceinline__ Grid(const SampleArgs& a, int64_t row) : vocab(a.vocab) {
        const uintptr_t p = (uintptr_t)((const T*)a.logits + row * a.row_stride);
        shift = (int32_t)((p & 15) / sizeof(T));
        origin = (const T*)(p & ~(uintptr_t)15);
    }
    __device__ __forceinline__ int32_t groups() const { return (int32_t)((vocab + shift + kGroup - 1) / kGroup); }
    __device__ __forceinline__ bool has(int64_t at) const { return at >= shift && at < vocab + shift; }
    __device__ __forceinline__ float operator()(int64_t at) const { return (float)origin[at]; }
};

// The 16 / sizeof(T) logits of the vector that begins at grid place `at`; places outside the row -inf.
template <typename T>
__device__ __forceinline__ void unpack(u32x4 raw, float* x) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(raw[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = (float)__builtin_bit_cast(T, (unsigned short)(raw[e / 2] >> (16 * (e % 2))));
    }
}
template <typename T>
__device__ __forceinline__ u32x4 load_vector(const Grid<T>& z, int64_t at) {
    return at < z.vocab + z.shift ? *(const u32x4*)(z.origin + at) : u32x4{0, 0, 0, 0};
}
// The vector with -inf, or NaN, in the places outside the row.
template <typename T>
__device__ __forceinline__ u32x4 in_row(const Grid<T>& z, int64_t at, u32x4 raw, float fill = -INFINITY) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) raw[e] = z.has(at + e) ? raw[e] : __float_as_uint(fill);
    } else {
        const uint32_t none = __builtin_bit_cast(unsigned short, (T)fill);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!z.has(at + e)) raw[e / 2] = e % 2 ? (raw[e / 2] & 0xffffu) | none << 16 : (raw[e / 2] & 0xffff0000u) | none;
    }
    return raw;
}
__device__ __forceinline__ int32_t wave_of_block() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

template <int kCtrl>
__device__ __forceinline__ float dpp_max(float x) {
    const int y = __builtin_amdgcn_update_dpp(0, __float_as_int(x), kCtrl, 0xf, 0xf, true);
    return fmaxf(x, __int_as_float(y));
}
template <int kCtrl>
__device__ __forceinline__ double dpp_add(double x) {
    const u32x2 u = __builtin_bit_cast(u32x2, x);
    const u32x2 y = {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)u.x, kCtrl, 0xf, 0xf, true),
                     (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u.y, kCtrl, 0xf, 0xf, true)};
    return x + __builtin_bit_cast(double, y);
}
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kHalfMirror = 0x141, kMirror = 0x140;

__device__ __forceinline__ float across_rows_max(float x) {
    u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
// The sum over the wavefront, in every lane, in one order.
__device__ __forceinline__ double wave_sum(double x) {
    x = dpp_add<kXor1>(x);
    x = dpp_add<kXor2>(x);
    x = dpp_add<kHalfMirror>(x);
    x = dpp_add<kMirror>(x);
    u32x2 u = __builtin_bit_cast(u32x2, x);
    u32x2 a = __builtin_amdgcn_permlane16_swap(u.x, u.x, false, false);
    u32x2 b = __builtin_amdgcn_permlane16_swap(u.y, u.y, false, false);
    x = __builtin_bit_cast(double, u32x2{a.x, b.x}) + __builtin_bit_cast(double, u32x2{a.y, b.y});
    u = __builtin_bit_cast(u32x2, x);
    a = __builtin_amdgcn_permlane32_swap(u.x, u.x, false, false);
    b = __builtin_amdgcn_permlane32_swap(u.y, u.y, false, false);
    return __builtin_bit_cast(double, u32x2{a.x, b.x}) + __builtin_bit_cast(double, u32x2{a.y, b.y});
}

// Calls f(value, grid place) for every token of the row's groups g, g + step, ... below `stop`, by one
// wavefront; a group's end is told by end(group).
template <typename T, typename F, typename E>
__device__ __forceinline__ void over_groups(const Grid<T>& z, int32_t g, int32_t stop, int32_t step, F&& f, E&& end) {
    constexpr int kPer = 16 / sizeof(T), kLoads = kGroup / (64 * kPer);
    const int lane = threadIdx.x & 63;
    const int32_t groups = z.groups();
    if (g >= stop) return;
    u32x4 next[kLoads];
#pragma unroll
    for (int l = 0; l < kLoads; ++l) next[l] = load_vector(z, (int64_t)g * kGroup + (l * 64 + lane) * kPer);
    for (; g < stop; g += step) {
        u32x4 raw[kLoads];
#pragma unroll
        for (int l = 0; l < kLoads; ++l) raw[l] = next[l];
        if (g + step < stop) {
#pragma unroll
            for (int l = 0; l < kLoads; ++l)
                next[l] = load_vector(z, (int64_t)(g + step) * kGroup + (l * 64 + lane) * kPer);
        }
        const bool edge = g == 0 || g + 1 >= groups;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            float x[kPer];
            unpack<T>(raw[l], x);
            const int64_t at = (int64_t)g * kGroup + (l * 64 + lane) * kPer;
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (!edge || z.has(at + e)) f(x[e], at + e);
        }
        end(g);
    }
}

// ------------------------------------------------------------ pass 1

constexpr int kScanThreads = 256, kScanWaves = kScanThreads / 64;

template <int kType>
__global__ __launch_bounds__(kScanThreads) void asd_sample_scan_kernel(SampleArgs a, Stats s, int32_t per_wave,
                                                                       int32_t tiles) {
    typedef typename Element<kType>::T T;
    constexpr int kPer = 16 / sizeof(T), kLoads = kGroup / (64 * kPer);
    const int lane = threadIdx.x & 63, wave = wave_of_block();
    const int64_t row = blockIdx.x / tiles;
    const int32_t tile = (int32_t)(blockIdx.x - row * tiles);
    if (blockIdx.x == 0 && threadIdx.x < 2) s.queued[threadIdx.x] = 0;
    const Grid<T> z(a, row);
    const Row r(a, row);
    const bool whole = !r.greedy && !r.by_count;
    const double per = 1.44269504088896340736 / (double)r.t;
    // neighbouring wavefronts read neighbouring groups
    const int32_t groups = z.groups();
    int32_t g = (tile * per_wave) * kScanWaves + wave;
    const int32_t stop = min((tile + 1) * per_wave * kScanWaves, s.groups);
    u32x4 next[kLoads];
#pragma unroll
    for (int l = 0; l < kLoads; ++l) next[l] = load_vector(z, (int64_t)g * kGroup + (l * 64 + lane) * kPer);
    for (; g < stop; g += kScanWaves) {
        u32x4 raw[kLoads];
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            raw[l] = next[l];
            next[l] = load_vector(z, (int64_t)(g + kScanWaves) * kGroup + (l * 64 + lane) * kPer);
        }
        const int64_t base = (int64_t)g * kGroup;
        if (g == 0 || g + 1 >= groups) {         // some places are not in the row
#pragma unroll
            for (int l = 0; l < kLoads; ++l) raw[l] = in_row(z, base + (l * 64 + lane) * kPer, raw[l]);
        }
        float top = -INFINITY;
        bool any_nan = false;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            float x[kPer];
            unpack<T>(raw[l], x);
            float m = -INFINITY;
            bool nan = false;
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                nan |= x[e] != x[e];
                m = fmaxf(m, x[e]);
            }
            m = dpp_max<kXor1>(m);
            m = dpp_max<kXor2>(m);
            m = dpp_max<kHalfMirror>(m);
            if constexpr (kPer == 4) m = dpp_max<kMirror>(m);
            top = fmaxf(top, m);
            const u64 nans = __ballot(nan);
            any_nan |= nans != 0;
            constexpr int kLanes = kSub / kPer;              // of a sub-block
            if (lane % kLanes == 0) {
                const bool mine = (nans >> lane & ((1ull << kLanes) - 1)) != 0;
                s.subs[(row * s.groups + g) * kSubs + l * (64 / kLanes) + lane / kLanes] = mine ? kKeyNan : key_of(m);
            }
        }
        if constexpr (kPer == 8) top = dpp_max<kMirror>(top);
        top = across_rows_max(top);
        double sum = 0.0;
        if (whole) {
            // A finite greatest logit weighs 1, so that the 2^-1000 of tokens far below, -inf among
            // them, changes no sum; where it is +inf the tokens there share the weight.
            if (top > -INFINITY && top < INFINITY) {
                const double from = (double)top;
#pragma unroll
                for (int l = 0; l < kLoads; ++l) {
                    float x[kPer];
                    unpack<T>(raw[l], x);
#pragma unroll
                    for (int e = 0; e < kPer; ++e) sum += power2_clamped(((double)x[e] - from) * per);
                }
            } else if (top == INFINITY) {
#pragma unroll
                for (int l = 0; l < kLoads; ++l) {
                    float x[kPer];
                    unpack<T>(raw[l], x);
#pragma unroll
                    for (int e = 0; e < kPer; ++e)
                        sum += x[e] == INFINITY ? 1.0 : 0.0;
                }
            }
            sum = wave_sum(sum);
        }
        if (lane == 0) {
            s.tops[row * s.groups + g] = any_nan ? kKeyNan : key_of(top);
            s.sums[row * s.groups + g] = sum;
        }
    }
}

// ------------------------------------------------------------ workgroup sums

// The same for masses, and the sum over the lanes up to each one.
template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ u64 dpp(u64 x) {
    const u32x2 u = __builtin_bit_cast(u32x2, x);
    return __builtin_bit_cast(u64, u32x2{(uint32_t)__builtin_amdgcn_update_dpp(0, (int)u.x, kCtrl, kRows, 0xf, false),
                                         (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u.y, kCtrl, kRows, 0xf, false)});
}
__device__ __forceinline__ u64 wave_sum(u64 x) {
    x += dpp<kXor1>(x);
    x += dpp<kXor2>(x);
    x += dpp<kHalfMirror>(x);
    x += dpp<kMirror>(x);
    u32x2 u = __builtin_bit_cast(u32x2, x);
    u32x2 a = __builtin_amdgcn_permlane16_swap(u.x, u.x, false, false);
    u32x2 b = __builtin_amdgcn_permlane16_swap(u.y, u.y, false, false);
    u = __builtin_bit_cast(u32x2, __builtin_bit_cast(u64, u32x2{a.x, b.x}) + __builtin_bit_cast(u64, u32x2{a.y, b.y}));
    a = __builtin_amdgcn_permlane32_swap(u.x, u.x, false, false);
    b = __builtin_amdgcn_permlane32_swap(u.y, u.y, false, false);
    return __builtin_bit_cast(u64, u32x2{a.x, b.x}) + __builtin_bit_cast(u64, u32x2{a.y, b.y});
}
__device__ __forceinline__ u64 wave_scan(u64 x) {
    constexpr int kUp = 0x110, kLast15 = 0x142, kLast31 = 0x143;
    x += dpp<kUp + 1>(x);
    x += dpp<kUp + 2>(x);
    x += dpp<kUp + 4>(x);
    x += dpp<kUp + 8>(x);
    x += dpp<kLast15, 0xa>(x);
    return x + dpp<kLast31, 0xc>(x);
}
__device__ __forceinline__ Mass wave_sum(const Mass& m) { return {wave_sum(m.high), wave_sum(m.low)}; }
__device__ __forceinline__ Mass wave_scan(const Mass& m) { return {wave_scan(m.high), wave_scan(m.low)}; }
template <typename V> __device__ __forceinline__ V wave_scan(V run) {
    for (int x = 1; x < 64; x <<= 1) {
        const V up = __shfl_up(run, x);
        if ((int)(threadIdx.x & 63) >= x) run += up;
    }
    return run;
}

template <int kN> struct Block {
    static constexpr int kWaves = kN / 64;
    double d[kWaves];
    u64 u[kWaves];
    Mass m[kWaves];

    __device__ __forceinline__ uint32_t max(uint32_t v) {
        for (int x = 32; x > 0; x >>= 1) v = ::max(v, (uint32_t)__shfl_xor((int)v, x));
        __syncthreads();
        if ((threadIdx.x & 63) == 0) u[threadIdx.x >> 6] = v;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) v = ::max(v, (uint32_t)u[w]);
        return v;
    }
    __device__ __forceinline__ uint32_t min(uint32_t v) { return ~max(~v); }
    __device__ __forceinline__ uint32_t any(uint32_t v) {
        for (int x = 32; x > 0; x >>= 1) v |= (uint32_t)__shfl_xor((int)v, x);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) u[threadIdx.x >> 6] = v;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) v |= (uint32_t)u[w];
        return v;
    }
    __device__ __forceinline__ uint32_t count(uint32_t v) {
        for (int x = 32; x > 0; x >>= 1) v += (uint32_t)__shfl_xor((int)v, x);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) u[threadIdx.x >> 6] = v;
        __syncthreads();
        uint32_t sum = 0;
        for (int w = 0; w < kWaves; ++w) sum += (uint32_t)u[w];
        return sum;
    }
    __device__ __forceinline__ double sum(double v) {
        v = wave_sum(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) d[threadIdx.x >> 6] = v;
        __syncthreads();
        double all = 0.0;
        for (int w = 0; w < kWaves; ++w) all += d[w];
        return all;
    }
    __device__ __forceinline__ Mass sum(Mass v) {
        v = wave_sum(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) m[threadIdx.x >> 6] = v;
        __syncthreads();
        Mass all{0, 0};
        for (int w = 0; w < kWaves; ++w) all += m[w];
        return all;
    }
    // The sum of a number that each wavefront has, with one barrier: the place alternates with `turn`, which the
    // caller counts up, so that a wavefront that is ahead does not write what another still reads.
    u64 votes_of[2][kWaves];
    __device__ __forceinline__ u64 votes(u64 of_wave, int turn) {
        if ((threadIdx.x & 63) == 0) votes_of[turn & 1][threadIdx.x >> 6] = of_wave;
        __syncthreads();
        u64 sum = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += votes_of[turn & 1][w];
        return sum;
    }
    // sum over the threads before this one, and over all
    template <typename V>
    __device__ __forceinline__ V before(V v, V* box, V* total) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const V run = wave_scan(v);
        __syncthreads();
        if (lane == 63) box[wave] = run;
        __syncthreads();
        V mine{}, all{};
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) mine += box[w];
            all += box[w];
        }
        *total = all;
        return mine + (run - v);
    }
};

// The first of wavefront 0's elements at which the running sum from `run` on passes `target`, lane
// after lane, 16 to a lane from grid place `base`; the last one with a weight where rounding
// leaves none.  Returns the grid place (every lane), and its weight.
template <typename W>
__device__ __forceinline__ int64_t draw_in_group(int64_t base, W&& weight, double run, double target, double* w) {
    const int lane = threadIdx.x & 63;
    double mine = 0.0;
#pragma unroll 4
    for (int e = 0; e < 16; ++e) mine += weight(base + lane * 16 + e);
    double upto = mine;
    for (int x = 1; x < 64; x <<= 1) {
        const double up = __shfl_up(upto, x);
        if (lane >= x) upto += up;
    }
    const u64 passes = __ballot(run + upto > target), some = __ballot(mine > 0.0);
    const int at = passes ? __builtin_ctzll(passes) : 63 - __builtin_clzll(some);
    int64_t place = -1;
    double last = 0.0;
    if (lane == at) {
        double sum = run + (upto - mine);
        for (int e = 0; e < 16; ++e) {
            const double x = weight(base + lane * 16 + e);
            sum += x;
            if (x > 0.0) {
                place = base + lane * 16 + e;
                last = x;
                if (sum > target) break;
            }
        }
    }
    *w = __shfl(last, at);
    return __shfl((long long)place, at);
}

__device__ __forceinline__ float inside_unit(float u) {
    return u >= 1.0f ? 0x1.fffffep-1f : u > 0.0f ? u : 0.0f;
}

// ------------------------------------------------------------ pass 2

constexpr int kPickThreads = 512, kPickWaves = kPickThreads / 64, kListed = 2048, kHeld = 8;
constexpr int kMostSubs = kPickThreads * kHeld;          // sub-block maxima held in registers
constexpr int kFewest = 192;                             // sub-blocks that candidates come from without top-k
constexpr int kRanked = kListed / kPickThreads, kRankBins = 1024;
static_assert(kMostSubs / 2 * (kSub / 4) / 64 <= kRankBins, "the vectors' starts");
// Top-k takes its candidates from a threshold that k sub-blocks' maxima reach, for as many as this: in a row in no
// order -ln(1 - k / subs) / (k / subs) times as many do, 1.53 at 0.6.  Beyond, up to kMostK, from a histogram
// of the row.
__device__ __forceinline__ int32_t most_k(int32_t subs) { return min(subs * 3 / 5, 1200); }
constexpr int32_t kMostK = kListed - 128;

template <int kType>
__global__ __launch_bounds__(kPickThreads) void asd_sample_pick_kernel(SampleArgs a, Stats s) {
    typedef typename Element<kType>::T T;
    constexpr int kPer = 16 / sizeof(T);
    __shared__ Block<kPickThreads> block;
    __shared__ uint32_t key[kListed], place[kListed];
    __shared__ double weight[kListed];
    __shared__ union {
        int32_t wanted[kMostSubs / 2];                       // the sub-blocks to read, then
        u64 order[kListed];                                  // the candidates by their keys' bins, then
        double ranked[kListed];                              // the weights in order
    } share;
    int32_t* const wanted = share.wanted;
    __shared__ uint32_t starts[kRankBins + 1];               // by 64 vectors of those, then by bin
    __shared__ int32_t found;
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_of_block();
    const int64_t row = blockIdx.x;
    const Grid<T> z(a, row);
    const Row r(a, row);
    const int32_t groups = z.groups(), subs = groups * kSubs;
    const uint32_t* const sub = s.subs + row * s.groups * kSubs;
    const uint32_t* const tops = s.tops + row * s.groups;
    const double* const sums = s.sums + row * s.groups;
    const auto finish = [&](int64_t at, double prob) {
        a.out_token[row] = at < 0 ? -1 : (int32_t)(at - z.shift);
        if (a.out_prob) a.out_prob[row] = (float)prob;
    };

    uint32_t top = 0;
    for (int32_t g = tid; g < groups; g += kPickThreads) top = max(top, tops[g]);
    top = block.max(top);
    if (top == kKeyNan || top == kKeyNegInf) {
        if (tid == 0) {
            finish(-1, 0.0);
            atomicOr(a.error_word, kDecodeErrSample);
        }
        return;
    }
    if (r.greedy) {
        uint32_t first = ~0u;
        for (int32_t g = tid; g < groups && first == ~0u; g += kPickThreads)
            if (tops[g] == top) first = (uint32_t)g;
        first = block.min(first);
        if (wave == 0) {
            const uint32_t k = lane < kSubs ? sub[(int64_t)first * kSubs + lane] : 0;
            const int64_t at = (int64_t)first * kGroup + __builtin_ctzll(__ballot(k == top)) * kSub + lane;
            const u64 same = __ballot(z.has(at) && key_of(z(min(max(at, (int64_t)z.shift), z.vocab + z.shift - 1))) == top);
            if (lane == 0) finish(at + __builtin_ctzll(same), 1.0);
        }
        return;
    }
    const Weights w(value_of(top), r.t);
    const float u = inside_unit(a.uniform[row]);

    double all = 0.0;           // the row's weights, where they count
    const bool filtered = r.by_count || r.by_mass || r.by_floor;
    if (!r.by_count) {
        if (!filtered) {
            // the draw's group
            const int32_t each = (groups + kPickThreads - 1) / kPickThreads;
            const int32_t from = min(groups, tid * each), to = min(groups, from + each);
            double mine = 0.0;
            for (int32_t g = from; g < to; ++g) mine += sums[g] * w(value_of(tops[g]));
            const double before = block.before(mine, block.d, &all), target = (double)u * all;
            // the first thread whose share passes it; rounding may leave none: the last with a weight
            uint32_t passes = mine > 0.0 && before + mine > target ? (uint32_t)tid : ~0u;
            passes = block.min(passes);
            if (passes == ~0u) passes = block.max(mine > 0.0 ? (uint32_t)tid : 0u);
            if ((uint32_t)tid == passes) {
                double run = before;
                for (int32_t g = from; g < to; ++g) {
                    const double x = sums[g] * w(value_of(tops[g]));
                    if (x > 0.0) {
                        found = g;
                        weight[0] = run;        // of the tokens before the group
                    }
                    if (run + x > target) break;
                    run += x;
                }
            }
            __syncthreads();
            if (wave == 0) {
                double x;
                const int64_t at = draw_in_group(
                    (int64_t)found * kGroup,
                    [&](int64_t place) { return z.has(place) ? w(z(place)) : 0.0; }, weight[0], target, &x);
                if (lane == 0) finish(at, x / all);
            }
            return;
        }
        double mine = 0.0;
        for (int32_t g = tid; g < groups; g += kPickThreads) mine += sums[g] * w(value_of(tops[g]));
        all = block.sum(mine);
    }

    // Candidates: every token whose key reaches `least`; all of a short row.
    const int32_t need = r.by_count ? r.k : max(1, min(kFewest, subs / 2));
    const bool all_listed = z.vocab <= kListed, by_bins = !all_listed && r.by_count && r.k > most_k(subs);
    if (subs > kMostSubs || (by_bins && (r.k > kMostK || top >= kKeyInf))) {
        if (tid == 0) enqueue(s, kAlone, row);
        return;
    }
    uint32_t held[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = i * kPickThreads + tid < subs ? sub[i * kPickThreads + tid] : 0;
    int turn = 0;               // of the sums with one barrier
    // the least of the sub-blocks' maxima, but of those that hold nothing
    const auto lowest = [&] {
        uint32_t low = kKeyNan;
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (held[i] > kKeyNegInf) low = min(low, held[i]);
        return block.min(low);
    };
    uint32_t least = 0;
    if (by_bins) {
        // bins of one width in the logit, from the greatest down to as far below the least of the maxima
        const float high = value_of(top), per = 0.5f * kRankBins / (high - value_of(lowest()));
        for (int b = tid; b < kRankBins; b += kPickThreads) starts[b] = 0;
        __syncthreads();
        over_groups(
            z, wave, groups, kPickWaves,
            [&](float x, int64_t) {
                atomicAdd(&starts[(uint32_t)fminf(fmaxf((high - x) * per, 0.0f), (float)(kRankBins - 1))], 1u);
            },
            [](int32_t) {});
        __syncthreads();
        const int32_t one = (int32_t)starts[2 * tid], two = (int32_t)starts[2 * tid + 1];
        int32_t in_all;
        const int32_t before = block.before(one + two, (int32_t*)block.u, &in_all);
        if (before < need && before + one + two >= need) found = 2 * tid + (before + one < need);
        __syncthreads();
        // All of that bin and those above it.  A hundredth of a bin further, which is more than the roundings of
        // the bins' numbers; the difference's own rounding passes no logit.
        const float edge = high - ((float)found + 1.01f) / per;
        least = found < kRankBins - 1 && edge > -INFINITY ? key_of(edge) : 0;
    } else if (!all_listed) {
        // by its upper 16 bits, two at a time
        for (int bit = 30; bit >= 16; bit -= 2) {
            if ((least | 1u << bit) > top) continue;
            u64 n = 0;              // how many reach each of the three trials
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                if (i * kPickThreads >= subs) break;
#pragma unroll
                for (uint32_t c = 1; c < 4; ++c)
                    n += (u64)__popcll(__ballot(held[i] >= (least | c << bit))) << (20 * (c - 1));
            }
            n = block.votes(n, turn++);
            for (uint32_t c = 3; c > 0; --c)
                if ((uint32_t)(n >> (20 * (c - 1)) & 0xfffff) >= (uint32_t)need) {
                    least |= c << bit;
                    break;
                }
        }
    }
    least = max(least, kKeyNegInf);
    // the sub-blocks that reach it, in order: the counts of each held[i] of each wavefront, summed up
    static_assert(kHeld * kPickWaves == 64, "a lane a count");
    uint32_t* const counts = starts;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int c = __popcll(__ballot(held[i] >= least));
        if (lane == 0) counts[i * kPickWaves + wave] = c;
    }
    __syncthreads();
    int32_t upto = (int32_t)counts[lane];
    for (int x = 1; x < 64; x <<= 1) {
        const int32_t up = __shfl_up(upto, x);
        if (lane >= x) upto += up;
    }
    const int32_t blocks = __shfl(upto, 63);
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const u64 in = __ballot(held[i] >= least);
        const int32_t at = __shfl(upto, i * kPickWaves + wave) - __popcll(in >> lane);
        if (held[i] >= least && at < kMostSubs / 2) wanted[at] = i * kPickThreads + tid;
    }
    __syncthreads();
    // Their tokens, in order: a sweep that counts them, 64 vectors at a time, and one that lists them (the
    // second finds them in the L2); several loads of a wavefront are on the way at once.
    int32_t n = 0;
    constexpr int kLanes = kSub / kPer, kAhead = 8, kWaves = kPickWaves;
    const int32_t sweeps = (blocks * kLanes + 63) / 64;
    if (blocks <= kMostSubs / 2) {
        // No NaN is left here, so that the logits' own order is the keys'; one fills places that do not count.
        const float from = value_of(least);
        const auto sweep = [&](auto&& f) {
            for (int32_t b = wave; b < sweeps; b += kAhead * kWaves) {
                u32x4 raw[kAhead];
                uint32_t at[kAhead];
#pragma unroll
                for (int c = 0; c < kAhead; ++c) {
                    const int32_t v = (b + c * kWaves) * 64 + lane;
                    at[c] = v < blocks * kLanes ? (uint32_t)(wanted[v / kLanes] * kSub + v % kLanes * kPer) : ~0u;
                    raw[c] = load_vector(z, at[c]);
                }
#pragma unroll
                for (int c = 0; c < kAhead; ++c) {
                    if (b + c * kWaves >= sweeps) break;
                    if (at[c] < (uint32_t)z.shift || (int64_t)at[c] + kPer > z.vocab + z.shift)
                        raw[c] = in_row(z, at[c], raw[c], NAN);
                    float x[kPer];
                    unpack<T>(raw[c], x);
                    f(b + c * kWaves, at[c], x);
                }
            }
        };
        sweep([&](int32_t b, uint32_t, const float* x) {
            uint32_t c = 0;
#pragma unroll
            for (int e = 0; e < kPer; ++e) c += (uint32_t)__popcll(__ballot(x[e] >= from));
            if (lane == 0) starts[b] = c;
        });
        __syncthreads();
        for (int32_t b0 = 0; b0 < sweeps; b0 += kPickThreads) {
            const int32_t c = b0 + tid < sweeps ? (int32_t)starts[b0 + tid] : 0;
            int32_t total;
            const int32_t before = n + block.before(c, (int32_t*)block.u, &total);
            if (b0 + tid < sweeps) starts[b0 + tid] = (uint32_t)before;
            n += total;
        }
        __syncthreads();
        if (n <= kListed)
            sweep([&](int32_t b, uint32_t at, const float* x) {
                uint32_t to = starts[b];
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    const u64 in = __ballot(x[e] >= from);
                    to = __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, to));
                }
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (x[e] >= from) {
                        key[to] = key_of(x[e]);
                        place[to] = at + e;
                        ++to;
                    }
            });
    }
    // What is left to the passes over whole rows.  The mass is reached below `least` as a rule, so the bins of a
    // shared row begin there; they reach four times as far as the lowest sub-block's maximum, which in rows of
    // any spread leaves 1 in 300 tokens or fewer in a bin.
    const auto leave = [&] {
        const bool shared = s.near && !r.by_count && top < kKeyInf;
        if (shared) {
            const uint32_t low = lowest();
            for (int b = tid; b < kNearBins; b += kPickThreads) s.bins[row * kNearBins + b] = 0;
            if (tid == 0) {
                const float high = value_of(least), range = 4.0f * (high - value_of(low));
                s.near[row] = Near{high, range > 0.0f ? kNearBins / range : 0.0f, top, 0, all, Mass{0, 0}};
            }
        }
        if (tid == 0) enqueue(s, shared ? kShared : kAlone, row);
    };
    if (blocks > kMostSubs / 2 || n > kListed) {
        leave();
        return;
    }
    __syncthreads();
    double mine = 0.0;
    for (int i = tid; i < n; i += kPickThreads) mine += weight[i] = w(value_of(key[i]));
    const double floor = r.by_floor ? (double)r.m : 0.0, sum = block.sum(mine);
    if (!r.by_count && least != kKeyNegInf &&            // some tokens are no candidates
        !(r.by_mass && sum >= (double)r.p * all) && !(r.by_floor && w(value_of(least)) < floor)) {
        leave();
        return;
    }

    uint32_t rank[kRanked];
    if (r.by_count || r.by_mass) {
        // Their order: bins of the logit, from the greatest down and narrower where there are more, put them in
        // their places but for those that share a bin, which are compared with each other.  (Comparing each with each took 8 us of
        // a row's 14, cuts by bisection over the keys' bits 30 of 65 with 1,400 candidates.)
        uint32_t last = least;
        if (least == kKeyNegInf) {          // all of the row: from the least logit that has a weight
            last = kKeyNan;
            for (int i = tid; i < n; i += kPickThreads)
                if (key[i] > kKeyNegInf) last = min(last, key[i]);
            last = block.min(last);
        }
        const float low = value_of(last), per = 1.0f / (value_of(top) - low);
        const auto bin_of = [&](uint32_t k) {
            const float part = fminf(fmaxf((value_of(k) - low) * per, 0.0f), 1.0f);
            return (uint32_t)(kRankBins - 1) - (uint32_t)(sqrtf(part) * (float)(kRankBins - 1));
        };
        for (int b = tid; b < kRankBins; b += kPickThreads) starts[b] = 0;
        __syncthreads();
        uint32_t bin[kRanked];
#pragma unroll
        for (int c = 0; c < kRanked; ++c) {
            const int i = c * kPickThreads + tid;
            if (i >= n) break;
            bin[c] = bin_of(key[i]);
            rank[c] = atomicAdd(&starts[bin[c]], 1u);
        }
        __syncthreads();
        static_assert(kRankBins == 2 * kPickThreads, "two bins a thread");
        const int32_t one = (int32_t)starts[2 * tid], two = (int32_t)starts[2 * tid + 1];
        int32_t in_all;
        const int32_t first = block.before(one + two, (int32_t*)block.u, &in_all);
        starts[2 * tid] = (uint32_t)first;
        starts[2 * tid + 1] = (uint32_t)(first + one);
        if (tid == 0) starts[kRankBins] = (uint32_t)n;
        __syncthreads();
#pragma unroll
        for (int c = 0; c < kRanked; ++c) {
            const int i = c * kPickThreads + tid;
            if (i >= n) break;
            share.order[starts[bin[c]] + rank[c]] = (u64)key[i] << 32 | (uint32_t)~i;
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < kRanked; ++c) {
            const int i = c * kPickThreads + tid;
            if (i >= n) break;
            const u64 own = (u64)key[i] << 32 | (uint32_t)~i;
            const uint32_t from = starts[bin[c]], to = starts[bin[c] + 1];
            rank[c] = from;
            uint32_t j = from;
            for (; j + 4 <= to; j += 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e) rank[c] += share.order[j + e] > own;
            }
            for (; j < to; ++j) rank[c] += share.order[j] > own;
        }
        if (r.by_mass) {
            // the weights before each, by a sum in that order
            __syncthreads();
#pragma unroll
            for (int c = 0; c < kRanked; ++c) {
                const int i = c * kPickThreads + tid;
                if (i < n) share.ranked[rank[c]] = !r.by_count || rank[c] < (uint32_t)r.k ? weight[i] : 0.0;
            }
            __syncthreads();
            double of[kRanked], mine = 0.0, whole;
#pragma unroll
            for (int c = 0; c < kRanked; ++c) mine += of[c] = tid * kRanked + c < n ? share.ranked[tid * kRanked + c] : 0.0;
            double before = block.before(mine, block.d, &whole);
            if (r.by_count) all = whole;
#pragma unroll
            for (int c = 0; c < kRanked; ++c) {
                share.ranked[tid * kRanked + c] = before;
                before += of[c];
            }
            __syncthreads();
        }
    }
    const double goal = (double)r.p * all;
#pragma unroll
    for (int c = 0; c < kRanked; ++c) {
        const int i = c * kPickThreads + tid;
        if (i >= n) break;
        if (weight[i] < floor || (r.by_count && rank[c] >= (uint32_t)r.k) ||
            (r.by_mass && rank[c] != 0 && !(share.ranked[rank[c]] < goal)))
            weight[i] = 0.0;
    }
    __syncthreads();

    // The draw, in order: a thread takes neighbouring candidates.
    const int each = (n + kPickThreads - 1) / kPickThreads, from = min(n, tid * each), to = min(n, from + each);
    mine = 0.0;
    for (int i = from; i < to; ++i) mine += weight[i];
    double total;
    const double before = block.before(mine, block.d, &total), target = (double)u * total;
    uint32_t passes = block.min(mine > 0.0 && before + mine > target ? (uint32_t)tid : ~0u);
    if (passes == ~0u) passes = block.max(mine > 0.0 ? (uint32_t)tid : 0u);
    if ((uint32_t)tid == passes) {
        double run = before, x = 0.0;
        int at = from;
        for (int i = from; i < to; ++i) {
            run += weight[i];
            if (weight[i] > 0.0) {
                at = i;
                x = weight[i];
                if (run > target) break;
            }
        }
        finish((int64_t)place[at], x / total);
    }
}

// ------------------------------------------------------------ whole rows

// ceil and floor of f * total for a float 0 <= f < 1 and a whole number below 2^95, exactly.
__device__ __forceinline__ u128 share(float f, u128 total, bool up) {
    if (!(f > 0.0f)) return 0;
    int e;
    const uint32_t m = (uint32_t)ldexpf(frexpf(f, &e), 24);   // f = m 2^(e - 24)
    const int shift = 24 - e;
    const u128 x = total * m;
    if (shift >= 120) return up && x != 0;
    return (x + (up ? ((u128)1 << shift) - 1 : 0)) >> shift;
}

// Coarse whole numbers, of 2^-bits of the greatest weight, for bins: a row's sum of them fits 62 bits.  What they
// say of a cut's place is checked by exact sums.
struct Coarse {
    double carrier;                 // as in mass_of; a weight below half a unit gives 0
    __device__ __forceinline__ explicit Coarse(int bits) : carrier((double)(1ull << (52 - bits))) {}
    __device__ __forceinline__ u64 operator()(double weight) const {
        return __builtin_bit_cast(u64, weight + carrier) - __builtin_bit_cast(u64, carrier);
    }
};

// The fewest tokens of `one` unit each, one at least, that make up `want`.
__device__ __forceinline__ u64 ties_for(u128 want, u128 one) {
    u64 n = 0;
    for (int bit = 30; bit >= 0; --bit)
        if (one * (n | 1ull << bit) < want) n |= 1ull << bit;
    return one > 0 ? n + 1 : 1;
}

// A row's weights.  Where the greatest logit is finite no token needs care: -inf gives 2^-1000, which is no unit.
struct Reals {
    Weights w;
    bool finite;
    __device__ __forceinline__ Reals(const Weights& w, uint32_t top) : w(w), finite(top < kKeyInf) {}
    __device__ __forceinline__ double operator()(float z) const {
        return finite ? power2_clamped(((double)z - w.top) * w.per) : w(z);
    }
};

// ------------------------------------------------------------ passes 3 and 4

// Rows that keep more tokens than pass 2 holds, by mass alone: every row in parts, all workgroups of the launch
// taking parts in turn.  Pass 3 sums the weights, coarsely, by bins of the logit.  Pass 4 finds the bin in which the
// mass is reached, sums each group's weights above it and lists the bin's own tokens.  (Where the rounding named a
// bin beside the cut's, pass 5 sees that and leaves the row to pass 6.)
constexpr int kPartThreads = 256, kPartWaves = kPartThreads / 64, kPartList = 1024;

// Whether rows are shared out: where pass 2 can hold their sub-blocks, and they are long, or many, enough to
// pay for three more launches, 6 us where no row is flat.  One flat row of 32,000 takes 67 us alone, one of
// 65,000 102 us, one of 151,936 56 us shared out, and 16 of 32,000 so 45.
bool shares_out(int64_t vocab, int64_t rows) {
    return vocab > (rows < 8 ? 65536 : 8192) && vocab + 7 <= (int64_t)kMostSubs * kSub;
}

// Shared tokens of a row that its list has room for, in the place of its sub-blocks' maxima.
__device__ __forceinline__ uint32_t list_room(const Stats& s) { return (uint32_t)s.groups * (kSubs / 2); }

template <int kType, bool kSurvey>
__global__ __launch_bounds__(kPartThreads) void asd_sample_part_kernel(SampleArgs a, Stats s, int bits) {
    typedef typename Element<kType>::T T;
    __shared__ Block<kPartThreads> block;
    __shared__ u64 box[kSurvey ? kPartList : kNearBins];      // listed tokens, or the part's bins
    __shared__ int32_t found;
    __shared__ uint32_t listed, start;
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_of_block();
    const uint32_t rows = s.queued[kShared];
    if (rows == 0) return;
    // parts of 4 groups at least, and two to a workgroup where there are enough
    const uint32_t parts = max(1u, min((2 * gridDim.x + rows - 1) / rows, (uint32_t)s.groups / kPartWaves));
    for (int64_t unit = blockIdx.x; unit < (int64_t)rows * parts; unit += gridDim.x) {
        const int64_t row = s.queue[kShared][unit / parts];
        const uint32_t part = (uint32_t)(unit % parts);
        const Grid<T> z(a, row);
        const Row r(a, row);
        if (!kSurvey && !r.by_mass) continue;        // min-p alone: no bin to find
        Near* const mine = s.near + row;
        const Near near{mine->high, mine->steps, mine->top, 0, 0.0, Mass{0, 0}};
        u64* const bins = s.bins + row * kNearBins;
        const Reals weight_of(Weights(value_of(near.top), r.t), near.top);
        const int64_t groups = z.groups();
        const int32_t from = (int32_t)(part * groups / parts), to = (int32_t)((part + 1) * groups / parts);
        if constexpr (!kSurvey) {
            for (int b = tid; b < kNearBins; b += kPartThreads) box[b] = 0;
            __syncthreads();
            const Coarse coarse(bits);
            over_groups(
                z, from + wave, to, kPartWaves,
                [&](float x, int64_t) { atomicAdd(&box[near.bin(x)], coarse(weight_of(x))); }, [](int32_t) {});
            __syncthreads();
            for (int b = tid; b < kNearBins; b += kPartThreads)
                if (box[b] != 0) atomicAdd(&bins[b], box[b]);
            __syncthreads();
        } else {
            if (tid == 0) listed = 0;
            int32_t bin = -1;            // of the cut: without one all tokens are above
            if (r.by_mass) {
                // from the last bin down
                constexpr int kEach = kNearBins / kPartThreads;
                u64 each[kEach], sum = 0, total;
#pragma unroll
                for (int c = 0; c < kEach; ++c) sum += each[c] = bins[kNearBins - 1 - (tid * kEach + c)];
                u64 have = block.before(sum, block.u, &total);
                const u64 want = max((u64)1, (u64)share(r.p, total, true));
                if (have < want && have + sum >= want) {
#pragma unroll
                    for (int c = 0; c < kEach; ++c) {
                        if (have < want && have + each[c] >= want) found = kNearBins - 1 - (tid * kEach + c);
                        have += each[c];
                    }
                }
                __syncthreads();
                bin = found;
            } else {
                __syncthreads();
            }
            const double floor = r.by_floor ? (double)r.m : 0.0;
            double above = 0.0, kept = 0.0;              // `kept`: of those above, what min-p keeps
            Mass all_above{0, 0};
            over_groups(
                z, from + wave, to, kPartWaves,
                [&](float x, int64_t at) {
                    const int32_t b = (int32_t)near.bin(x);
                    if (b > bin) {
                        const double y = weight_of(x);
                        above += y;
                        if (r.by_floor) kept += y >= floor ? y : 0.0;
                    } else if (b == bin) {
                        const uint32_t i = atomicAdd(&listed, 1u);
                        if (i < kPartList) box[i] = (u64)at << 32 | key_of(x);
                    }
                },
                [&](int32_t g) {
                    if (r.by_mass) all_above += mass_of(above = wave_sum(above));
                    if (r.by_floor) above = wave_sum(kept);
                    if (lane == 0) s.sums[row * s.groups + g] = above;
                    above = kept = 0.0;
                });
            if (r.by_mass && lane == 0) add_to(&mine->above.high, &mine->above.low, all_above);
            __syncthreads();
            // more than there is room for: a number that no list has
            if (tid == 0 && listed > 0) start = atomicAdd(&mine->collected, listed <= kPartList ? listed : 1u << 24);
            __syncthreads();
            const uint32_t n = min(listed, (uint32_t)kPartList);
            u64* const list = (u64*)(s.subs + row * s.groups * kSubs);
            for (uint32_t i = tid; i < n; i += kPartThreads)
                if (start + i < list_room(s)) list[start + i] = box[i];
            __syncthreads();
        }
    }
}

// ------------------------------------------------------------ pass 5

// A shared row's token from what passes 3 and 4 left of it, a workgroup a row and a thread a group: the cut
// among the listed tokens, in the order of their ranks, then the draw's group and its tokens in order.
constexpr int kFinishList = 1024, kFinishEach = kFinishList / kPartThreads;
static_assert(kMostSubs / kSubs <= kPartThreads, "a thread a group");

template <int kType>
__global__ __launch_bounds__(kPartThreads) void asd_sample_finish_kernel(SampleArgs a, Stats s) {
    typedef typename Element<kType>::T T;
    __shared__ Block<kPartThreads> block;
    __shared__ u64 order[kFinishList];
    __shared__ Mass ranked[kFinishList], kept_in[kPartThreads];
    __shared__ u128 pick_run;
    __shared__ int32_t pick;
    const int tid = threadIdx.x;
    const uint32_t rows = s.queued[kShared];
    for (uint32_t q = blockIdx.x; q < rows; q += gridDim.x) {
        __syncthreads();
        const int64_t row = s.queue[kShared][q];
        const Near near = s.near[row];
        const float u = inside_unit(a.uniform[row]);
        const int n = (int)min(near.collected, 1u << 24);
        // more in the cut's bin than fit, and u = 0, for which even a token of no unit is the first
        if (n > (int)min(list_room(s), (uint32_t)kFinishList) || u == 0.0f) {
            if (tid == 0) enqueue(s, kAlone, row);
            continue;
        }
        const Grid<T> z(a, row);
        const Row r(a, row);
        const Reals weight_of(Weights(value_of(near.top), r.t), near.top);
        const double floor = r.by_floor ? (double)r.m : 0.0;
        const auto kept_weight = [&](float x) -> Mass {
            const double y = weight_of(x);
            return y >= floor ? mass_of(y) : Mass{0, 0};
        };
        const int32_t groups = z.groups();
        kept_in[tid] = mass_of(tid < groups ? s.sums[row * s.groups + tid] : 0.0);
        uint32_t cut = 0, ties = 0;          // kept: greater keys, and the first `ties` tokens that have it
        const u64* const list = (const u64*)(s.subs + row * s.groups * kSubs);
        uint32_t key[kFinishEach], place[kFinishEach];
        if (r.by_mass) {
#pragma unroll
            for (int c = 0; c < kFinishEach; ++c) {
                const int i = c * kPartThreads + tid;
                const u64 x = i < n ? list[i] : 0;
                key[c] = (uint32_t)x;
                place[c] = (uint32_t)(x >> 32);
                order[i] = i < n ? (u64)key[c] << 32 | (uint32_t)~place[c] : 0;
                ranked[i] = Mass{0, 0};
            }
            __syncthreads();
            uint32_t rank[kFinishEach];
#pragma unroll
            for (int c = 0; c < kFinishEach; ++c) {
                rank[c] = 0;
                if (c * kPartThreads >= n) break;
                const u64 own = order[c * kPartThreads + tid];
                for (int i = 0; i < n; i += 16) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) rank[c] += order[i + e] > own;
                }
                if (c * kPartThreads + tid < n) ranked[rank[c]] = mass_of(weight_of(value_of(key[c])));
            }
            __syncthreads();
            Mass of[kFinishEach], sum{0, 0}, whole;
#pragma unroll
            for (int c = 0; c < kFinishEach; ++c) sum += of[c] = ranked[tid * kFinishEach + c];
            Mass before = block.before(sum, block.m, &whole);
            // what is wanted of the list: some of it, and no more than it has, or the cut lies in another bin
            const u128 want = units_of((double)r.p * near.all), above = near.above.value();
            if (want <= above || want - above > whole.value()) {
                if (tid == 0) enqueue(s, kAlone, row);
                continue;
            }
            const u128 rest = want - above;
#pragma unroll
            for (int c = 0; c < kFinishEach; ++c) {
                ranked[tid * kFinishEach + c] = before;
                before += of[c];
            }
            __syncthreads();
            uint32_t least = ~0u, same = 0;
            bool kept[kFinishEach];
#pragma unroll
            for (int c = 0; c < kFinishEach; ++c) {
                kept[c] = c * kPartThreads + tid < n && ranked[rank[c]].value() < rest;
                if (kept[c]) {
                    least = min(least, key[c]);
                    Mass* const to = &kept_in[place[c] / kGroup];
                    add_to(&to->high, &to->low, kept_weight(value_of(key[c])));
                }
            }
            cut = block.min(least);
#pragma unroll
            for (int c = 0; c < kFinishEach; ++c) same += kept[c] && key[c] == cut;
            ties = block.count(same);
        }
        __syncthreads();
        const Mass mine = kept_in[tid];
        Mass sum_of_all;
        const u128 before = block.before(mine, block.m, &sum_of_all).value(), all = sum_of_all.value();
        const u128 target = share(u, all, false);
        if (before <= target && before + mine.value() > target) {
            pick = tid;
            pick_run = before;
        }
        __syncthreads();
        const int64_t from = (int64_t)pick * kGroup;
        const double rest_of = real_of(target - pick_run);         // that the group's running sum has to exceed
        uint32_t seen = 0;                   // tokens that have the cut's key before the group's
        if (r.by_mass) {
#pragma unroll
            for (int c = 0; c < kFinishEach; ++c)
                seen += c * kPartThreads + tid < n && key[c] == cut && place[c] < (uint32_t)from;
            seen = block.count(seen);
        }
        // a thread four neighbouring tokens
        constexpr int kEach = kGroup / kPartThreads;
        uint32_t k[kEach], tied = 0, all_tied;
        float x[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int64_t at = from + tid * kEach + e;
            x[e] = z.has(at) ? z(at) : -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            k[e] = z.has(from + tid * kEach + e) ? key_of(x[e]) : 0;
            tied += r.by_mass && k[e] == cut;
        }
        seen += block.before(tied, (uint32_t*)block.u, &all_tied);
        double y[kEach], sum = 0.0, total;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const bool kept = k[e] > cut || (r.by_mass && k[e] == cut && seen++ < ties);
            const double weight = kept ? weight_of.w(x[e]) : 0.0;      // (-inf: none at all)
            sum += y[e] = weight >= floor ? weight : 0.0;
        }
        // the first thread whose tokens pass it; rounding may leave none: the last with a weight
        double run = block.before(sum, block.d, &total);
        uint32_t passes = block.min(sum > 0.0 && run + sum > rest_of ? (uint32_t)tid : ~0u);
        if (passes == ~0u) passes = block.max(sum > 0.0 ? (uint32_t)tid : 0u);
        if ((uint32_t)tid == passes) {
            int at = 0;
            double weight = 0.0;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                if (y[e] > 0.0 && !(weight > 0.0 && run > rest_of)) {
                    at = e;
                    weight = y[e];
                }
                run += y[e];
            }
            a.out_token[row] = (int32_t)(from + tid * kEach + at - z.shift);
            if (a.out_prob) a.out_prob[row] = (float)(weight / real_of(all));
        }
    }
}

// ------------------------------------------------------------ pass 6

constexpr int kFlatThreads = 512, kFlatWaves = kFlatThreads / 64, kBins = 4096, kCollected = 8192, kSpans = kFlatThreads;

// A whole row by one workgroup: histograms of it give the bin that holds the cut, a second reading lists that bin
// and sums what lies above it.  Each reading is the exponentials' time on one compute unit, some 40 us for
// 129,280 logits.  Spans (1,024 tokens each up to 2^19 tokens a row) hold what is kept of them.  A call of 8,000
// logits with top-p takes 41 us, one of 32,000 67.  (512 threads: 1,024, whose registers did not hold everything, took
// 1.6 and 1.3 times as long.)
template <int kType>
__device__ __forceinline__ void flat_row(const SampleArgs& a, const Stats& s, int bits, int64_t row) {
    typedef typename Element<kType>::T T;
    __shared__ Block<kFlatThreads> block;
    __shared__ u64 bin_high[kBins], bin_low[kBins];          // Mass by bin
    __shared__ uint32_t bin_count[kBins];
    __shared__ uint32_t key[kCollected], place[kCollected];
    __shared__ Mass span_sum[kSpans];
    __shared__ uint32_t span_ties[kSpans];
    __shared__ uint32_t collected;
    __shared__ u128 pick[2];
    __shared__ u64 pick_ties;
    __shared__ Mass in_all;                                  // that a reading of the row summed up
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_of_block();
    const Grid<T> z(a, row);
    const Row r(a, row);
    const int32_t groups = z.groups(), per_span = (groups + kSpans - 1) / kSpans;
    const int32_t spans = (groups + per_span - 1) / per_span;
    uint32_t top = 0;
    for (int32_t g = tid; g < groups; g += kFlatThreads) top = max(top, s.tops[row * s.groups + g]);
    top = block.max(top);
    const Weights w(value_of(top), r.t);
    const Reals real(w, top);
    const double floor = r.by_floor ? (double)r.m : 0.0;
    const auto weight_of = [&](float z) -> Mass { return mass_of(real(z)); };
    const auto kept_weight = [&](float z) -> Mass {
        const double x = real(z);
        return x >= floor ? mass_of(x) : Mass{0, 0};
    };

    const auto over = [&](auto&& f, auto&& end) { over_groups(z, wave, groups, kFlatWaves, f, end); };
    const auto nothing = [](int32_t) {};

    // What every span holds: the weights of the tokens whose order exceeds `at_order`, less what min-p drops (all of
    // them in in_all), and, of those that have it, the tokens themselves (key and place), or, where the order is
    // the whole key, how many there are.
    const auto survey = [&](auto&& order, uint32_t at_order, bool whole_key, uint32_t limit) {
        for (int i = tid; i < kSpans; i += kFlatThreads) {
            span_sum[i] = Mass{0, 0};
            span_ties[i] = 0;
        }
        if (tid == 0) {
            collected = 0;
            in_all = Mass{0, 0};
        }
        __syncthreads();
        double above = 0.0, kept = 0.0;              // `kept`: of those above, what min-p keeps
        Mass of_wave{0, 0};
        uint32_t same = 0;
        over(
            [&](float x, int64_t at) {
                const uint32_t b = order(x);
                if (b > at_order) {
                    const double y = real(x);
                    above += y;
                    if (r.by_floor) kept += y >= floor ? y : 0.0;
                } else if (b == at_order) {
                    const uint32_t k = key_of(x);
                    if (k < limit) return;
                    if (whole_key) {
                        ++same;
                    } else {
                        const uint32_t i = atomicAdd(&collected, 1u);
                        if (i < kCollected) {
                            key[i] = k;
                            place[i] = (uint32_t)at;
                        }
                    }
                }
            },
            [&](int32_t g) {
                above = wave_sum(above);
                of_wave += mass_of(above);
                if (r.by_floor) above = wave_sum(kept);
                for (int x = 32; whole_key && x > 0; x >>= 1) same += (uint32_t)__shfl_xor((int)same, x);
                if (lane == 0) {
                    Mass* const span = &span_sum[g / per_span];
                    add_to(&span->high, &span->low, mass_of(above));
                    if (whole_key) atomicAdd(&span_ties[g / per_span], same);
                }
                above = kept = 0.0;
                same = 0;
            });
        if (lane == 0) add_to(&in_all.high, &in_all.low, of_wave);
        __syncthreads();
    };
    const auto clear_bins = [&]() {
        for (int b = tid; b < kBins; b += kFlatThreads) {
            bin_high[b] = bin_low[b] = 0;
            bin_count[b] = 0;
        }
        if (tid == 0) in_all = Mass{0, 0};
        __syncthreads();
    };
    // The bin in which `want` is reached, from the last one down, and what is still wanted of it: eight bins a thread.
    enum { kCounts, kCoarsely, kFinely };
    const auto find_bin = [&](int kind, u128* want) -> uint32_t {
        constexpr int kEach = kBins / kFlatThreads;
        const auto of = [&](int i) {
            const int b = kBins - 1 - (kEach * tid + i);
            return kind == kFinely ? Mass{bin_high[b], bin_low[b]} : Mass{0, kind == kCounts ? bin_count[b] : bin_high[b]};
        };
        Mass mine{0, 0}, total;
#pragma unroll
        for (int i = 0; i < kEach; ++i) mine += of(i);
        u128 have = block.before(mine, block.m, &total).value();
        if (tid == 0) {
            pick[0] = 0;
            pick[1] = *want;
        }
        __syncthreads();
        if (have < *want && have + mine.value() >= *want) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const u128 upto = have + of(i).value();
                if (have < *want && upto >= *want) {
                    pick[0] = (u128)(kBins - 1 - (kEach * tid + i));
                    pick[1] = *want - have;
                }
                have = upto;
            }
        }
        __syncthreads();
        const uint32_t bin = (uint32_t)pick[0];
        *want = pick[1];
        __syncthreads();
        return bin;
    };
    // Keys above `cut` are kept, and the first `ties` tokens that have it; stage 0 cuts by count, stage 1 by
    // mass among what stage 0 left.
    uint32_t cut = 0;
    u64 ties = ~0ull;
    // Bins of 1/64 octave of the weight, the last one for all below 2^-64: tokens spread over many of them, so
    // that few add to one at a time.  (Leading bits of the keys put a row of N(0, 2) into some
    // sixty: its histogram alone took 70 us.)
    const float steps = (float)(64.0 * w.per);
    const auto near_top = [&](float x) -> uint32_t {
        return (uint32_t)(kBins - 1) - (uint32_t)fminf((w.top_f - x) * steps, (float)(kBins - 1));
    };
    for (int stage = 0; stage < 2; ++stage) {
        if (!(stage == 0 ? r.by_count : r.by_mass)) continue;
        const bool by_weight = stage == 1;
        const uint32_t limit = cut;
        const u64 limit_ties = ties;
        const Mass limit_weight = limit ? weight_of(value_of(limit)) : Mass{0, 0};
        const Mass limit_mass = by_weight && limit != 0 ? limit_weight * limit_ties : Mass{0, 0};
        const bool limited = limit_mass.value() != 0;
        const auto worth = [&](uint32_t k) -> Mass {     // of a token beyond the limit's
            return !by_weight ? Mass{0, 1} : k > limit ? weight_of(value_of(k)) : Mass{0, 0};
        };
        u128 want = (u128)(uint32_t)r.k;
        bool listed = false, limit_in = false;        // a list, and the limit's tokens in it
        if (top < kKeyInf) {
            clear_bins();
            const Coarse coarse(bits);
            double part = 0.0;
            Mass of_wave{0, 0};
            over(
                [&](float x, int64_t) {
                    const uint32_t b = near_top(x);
                    if (!by_weight) {
                        atomicAdd(&bin_count[b], 1u);
                    } else if (limit == 0 || key_of(x) > limit) {
                        const double y = real(x);
                        atomicAdd(&bin_high[b], coarse(y));
                        part += y;
                    }
                },
                [&](int32_t) {
                    if (!by_weight) return;
                    of_wave += mass_of(wave_sum(part));
                    part = 0.0;
                });
            if (lane == 0) add_to(&in_all.high, &in_all.low, of_wave);
            __syncthreads();
            // of the tokens at the limit only those count that stage 0 kept
            if (limited && tid == 0) bin_high[near_top(value_of(limit))] += coarse(real(value_of(limit))) * limit_ties;
            __syncthreads();
            u128 rest = want;
            if (by_weight) {
                want = max((u128)1, share(r.p, (in_all + limit_mass).value(), true));
                Mass mine{0, 0};
                for (int b = tid; b < kBins; b += kFlatThreads) mine.low += bin_high[b];
                rest = max((u128)1, share(r.p, block.sum(mine).value(), true));
            }
            const uint32_t bin = find_bin(by_weight ? kCoarsely : kCounts, &rest);
            const u64 in_bin = bin_high[bin];
            survey(near_top, bin, false, limit);
            listed = collected <= (uint32_t)kCollected;
            limit_in = limited && near_top(value_of(limit)) == bin;
            if (listed && by_weight) {
                // Some of the listed has to be wanted, and no more than there is, or the cut lies in another bin.
                // (Each of a bin's coarse weights is half a unit off at most.)
                const u128 above = in_all.value();
                listed = want > above;
                rest = want - above;
                if (listed && rest > (u128)(in_bin - min(in_bin, (u64)collected)) << (64 - bits)) {
                    Mass mine{0, 0};
                    for (int i = tid; i < (int)collected; i += kFlatThreads) mine += worth(key[i]);
                    Mass of_list = block.sum(mine);
                    if (limit_in) of_list += limit_mass;
                    listed = rest <= of_list.value();
                }
            }
            if (listed) want = rest;
        }
        uint32_t prefix = 0;            // of the cut's key, from bit `shift` up
        int shift = 32;
        if (!listed) {
            // More tokens in one bin than the list holds, or another bin: by the keys' bits.
            __syncthreads();
            if (by_weight && !(top < kKeyInf)) {
                Mass mine{0, 0};
                over([&](float x, int64_t) { if (key_of(x) > limit) mine += weight_of(x); }, nothing);
                want = max((u128)1, share(r.p, (block.sum(mine) + limit_mass).value(), true));
            }
            u64 in_bin = ~0ull;
            while (shift > 0 && in_bin > (u64)kCollected) {
                const int low = shift == 32 ? 20 : shift == 20 ? 8 : 0;
                const uint32_t mask = (1u << (shift - low)) - 1;
                clear_bins();
                over(
                    [&](float x, int64_t) {
                        const uint32_t k = key_of(x);
                        if (k < limit || (shift < 32 && k >> shift != prefix)) return;
                        const uint32_t b = k >> low & mask;
                        if (by_weight && k > limit) add_to(&bin_high[b], &bin_low[b], weight_of(x));
                        atomicAdd(&bin_count[b], 1u);
                    },
                    nothing);
                __syncthreads();
                if (limited && (shift == 32 || limit >> shift == prefix) && tid == 0) {
                    bin_high[limit >> low & mask] += limit_mass.high;
                    bin_low[limit >> low & mask] += limit_mass.low;
                }
                __syncthreads();
                const uint32_t bin = find_bin(by_weight ? kFinely : kCounts, &want);
                in_bin = bin_count[bin];
                prefix = (shift == 32 ? 0u : prefix << (shift - low)) | bin;
                shift = low;
                __syncthreads();
            }
            survey([&](float x) { return key_of(x) >> shift; }, prefix, shift == 0, limit);
            listed = shift > 0;
            limit_in = limited && listed && limit >> shift == prefix;
        }
        if (listed) {
            // the cut among the listed tokens
            const int n = min((int)collected, kCollected);
            if (n <= kFlatThreads) {
                // A token's rank by comparing it with each, then the mass before it by a sum over the
                // tokens in that order.  Those that have the limit's key come last, and the first
                // limit_ties of them count.
                const uint32_t k = tid < n ? key[tid] : 0;
                u64* const order = bin_high;                 // done with
                Mass* const ranked = (Mass*)bin_low;
                Mass* const sums = ranked + kFlatThreads;
                const u64 own = tid < n ? (u64)k << 32 | (uint32_t)~place[tid] : 0;
                order[tid] = own;
                ranked[tid] = Mass{0, 0};
                __syncthreads();
                uint32_t rank = 0;
                if (wave * 64 < n) {
                    for (int i = 0; i < n; i += 16) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) rank += order[i + e] > own;
                    }
                }
                u128 before = rank;
                bool counts = true;
                if (by_weight) {
                    const uint32_t more = block.count(k > limit);
                    counts = k > limit || rank - more < limit_ties;
                    if (tid < n) ranked[rank] = k > limit ? weight_of(value_of(k)) : counts ? limit_weight : Mass{0, 0};
                    __syncthreads();
                    Mass all;
                    sums[tid] = block.before(ranked[tid], block.m, &all);
                    __syncthreads();
                    if (tid < n) before = sums[rank].value();
                }
                const bool kept = tid < n && before < want && counts;
                prefix = block.min(kept ? k : ~0u);
                ties = block.count(kept && k == prefix);
                cut = prefix;
            } else {
                // The greatest of their keys that is reached, by those bits in which they differ.
                uint32_t differ = 0;
                for (int i = tid; i < n; i += kFlatThreads) differ |= key[i] ^ key[0];
                differ = block.any(differ);
                prefix = key[0] & ~differ;
                for (; differ != 0; differ &= ~(1u << (31 - __builtin_clz(differ)))) {
                    const uint32_t trial = prefix | 1u << (31 - __builtin_clz(differ));
                    bool reached;
                    if (by_weight) {
                        Mass mine{0, 0};
                        for (int i = tid; i < n; i += kFlatThreads)
                            if (key[i] >= trial) mine += worth(key[i]);
                        Mass reach = block.sum(mine);
                        if (limit_in && trial <= limit) reach += limit_mass;
                        reached = reach.value() >= want;
                    } else {
                        uint32_t mine = 0;
                        for (int i = tid; i < n; i += kFlatThreads) mine += key[i] >= trial;
                        reached = block.count(mine) >= want;
                    }
                    if (reached) prefix = trial;
                }
                Mass mine{0, 0};
                for (int i = tid; i < n; i += kFlatThreads)
                    if (key[i] > prefix) mine += worth(key[i]);
                want -= min(want, block.sum(mine).value());
                const u64 m = ties_for(want, by_weight ? weight_of(value_of(prefix)).value() : 1);
                ties = by_weight && prefix == limit ? min(m, limit_ties) : m;
                cut = prefix;
            }
            for (int i = tid; i < n; i += kFlatThreads) {
                const int32_t span = (int32_t)(place[i] / (uint32_t)kGroup) / per_span;
                if (key[i] > cut) {
                    add_to(&span_sum[span].high, &span_sum[span].low, kept_weight(value_of(key[i])));
                } else if (key[i] == cut) {
                    atomicAdd(&span_ties[span], 1u);
                }
            }
            __syncthreads();
        } else {
            cut = prefix;
            const u64 m = ties_for(want, by_weight ? weight_of(value_of(cut)).value() : 1);
            ties = by_weight && cut == limit ? min(m, limit_ties) : m;
        }
    }
    if (!r.by_count && !r.by_mass) survey([](float x) { return key_of(x); }, 0, true, 0);
    const Mass cut_weight = cut != 0 ? kept_weight(value_of(cut)) : Mass{0, 0};
    const u64 here = tid < spans ? span_ties[tid] : 0;
    u64 all_ties;
    const u64 ties_before = block.before(here, block.u, &all_ties);
    const u64 kept_ties = ties_before < ties ? min(here, ties - ties_before) : 0;
    const Mass sum = tid < spans ? span_sum[tid] + cut_weight * kept_ties : Mass{0, 0};
    Mass total;
    const u128 before = block.before(sum, block.m, &total).value(), all = total.value();
    const float u = inside_unit(a.uniform[row]);
    if (u == 0.0f) {
        // the first kept token, which may weigh less than a unit
        uint32_t first = ~0u;
        double weight = 0.0;
        over(
            [&](float x, int64_t at) {
                if (key_of(x) < cut || first != ~0u) return;
                const double y = w(x);
                if (y > 0.0 && y >= floor) {
                    first = (uint32_t)at;
                    weight = y;
                }
            },
            nothing);
        const uint32_t place = block.min(first);
        if (first == place) {
            a.out_token[row] = (int32_t)(place - (uint32_t)z.shift);
            if (a.out_prob) a.out_prob[row] = (float)(weight / real_of(all));
        }
        return;
    }
    const u128 target = share(u, all, false);            // the running sum has to exceed it
    if (before <= target && before + sum.value() > target) {
        pick[0] = (u128)tid;
        pick[1] = before;
        pick_ties = ties_before;
    }
    __syncthreads();
    // The span's tokens in order, two to a thread, up to the first at which the running sum passes the rest; rounding
    // may leave none: the last with a weight.
    const double rest = real_of(target - pick[1]);
    double run = 0.0, weight = 0.0, part;
    u64 seen = pick_ties;
    uint32_t passes = ~0u, last = 0;
    const int64_t from = (int64_t)pick[0] * per_span * kGroup;
    const int64_t to = min(from + (int64_t)per_span * kGroup, z.vocab + z.shift);
    for (int64_t first = from; first < to && passes == ~0u; first += 2 * kFlatThreads) {
        const int64_t at = first + 2 * tid;
        float x[2];
        uint32_t k[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const bool in = at + e < to && z.has(at + e);
            x[e] = in ? z(at + e) : -INFINITY;
            k[e] = in ? key_of(x[e]) : 0;
        }
        u64 tied;
        u64 rank = seen + block.before((u64)(k[0] == cut) + (u64)(k[1] == cut), block.u, &tied);
        double y[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            y[e] = k[e] > cut || (k[e] != 0 && k[e] == cut && rank++ < ties) ? w(x[e]) : 0.0;
            if (y[e] < floor) y[e] = 0.0;
        }
        double upto = run + block.before(y[0] + y[1], block.d, &part);
        bool mine = false;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            upto += y[e];
            if (y[e] > 0.0 && !mine) {
                last = (uint32_t)(at + e);
                weight = y[e];
                mine = upto > rest;
            }
        }
        passes = block.min(mine ? last : ~0u);
        run += part;
        seen += tied;
    }
    const uint32_t drawn = passes != ~0u ? passes : block.max(last);
    if (last == drawn && weight > 0.0) {
        a.out_token[row] = (int32_t)(drawn - (uint32_t)z.shift);
        if (a.out_prob) a.out_prob[row] = (float)(weight / real_of(all));
    }
}

template <int kType>
__global__ __launch_bounds__(kFlatThreads) void asd_sample_flat_kernel(SampleArgs a, Stats s, int bits) {
    const uint32_t rows = s.queued[kAlone];
    for (uint32_t q = blockIdx.x; q < rows; q += gridDim.x) {
        flat_row<kType>(a, s, bits, s.queue[kAlone][q]);
        __syncthreads();
    }
}

int32_t most_groups(int64_t vocab) { return (int32_t)((vocab + 7 + kGroup - 1) / kGroup); }

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

template <int kType>
hipError_t sample(const SampleArgs& a, const Stats& s, int32_t per_wave, int bits, int cus, hipStream_t stream) {
    const int32_t tiles = (s.groups + per_wave * kScanWaves - 1) / (per_wave * kScanWaves);
    asd_sample_scan_kernel<kType><<<(unsigned)(a.rows * tiles), kScanThreads, 0, stream>>>(a, s, per_wave, tiles);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    asd_sample_pick_kernel<kType><<<(unsigned)a.rows, kPickThreads, 0, stream>>>(a, s);
    if ((err = hipGetLastError()) != hipSuccess) return err;
    if (s.near) {
        const unsigned grid = (unsigned)cus * 4;
        asd_sample_part_kernel<kType, false><<<grid, kPartThreads, 0, stream>>>(a, s, bits);
        if ((err = hipGetLastError()) != hipSuccess) return err;
        asd_sample_part_kernel<kType, true><<<grid, kPartThreads, 0, stream>>>(a, s, bits);
        if ((err = hipGetLastError()) != hipSuccess) return err;
        asd_sample_finish_kernel<kType>
            <<<(unsigned)(a.rows < grid ? a.rows : grid), kPartThreads, 0, stream>>>(a, s);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    asd_sample_flat_kernel<kType>
        <<<(unsigned)(a.rows < cus ? a.rows : cus), kFlatThreads, 0, stream>>>(a, s, bits);
    return hipGetLastError();
}

// The workspace's parts, from `base` on (which may be null to add them up).
size_t lay_out(int64_t vocab, int64_t rows, char* base, Stats* s) {
    const size_t n = (size_t)rows, groups = (size_t)most_groups(vocab) * n;
    size_t at = 0;
    const auto part = [&](size_t bytes) {
        char* const p = (char*)((uintptr_t)base + at);
        at += align256(bytes);
        return p;
    };
    *s = Stats{};
    s->groups = most_groups(vocab);
    s->sums = (double*)part(groups * sizeof(double));
    s->subs = (uint32_t*)part(groups * kSubs * sizeof(uint32_t));
    s->tops = (uint32_t*)part(groups * sizeof(uint32_t));
    s->queued = (uint32_t*)part(2 * sizeof(uint32_t));
    s->queue[kAlone] = (int32_t*)part(n * sizeof(int32_t));
    if (shares_out(vocab, rows)) {
        s->queue[kShared] = (int32_t*)part(n * sizeof(int32_t));
        s->near = (Near*)part(n * sizeof(Near));
        s->bins = (u64*)part(n * kNearBins * sizeof(u64));
    }
    return at;
}

// Rows of a launch: more are drawn by several, one after the other in the same workspace.
constexpr int64_t kMostRows = (int64_t)1 << 20;

template <int kType> hipError_t sample_rows(const SampleArgs& a, void* workspace, int cus, hipStream_t stream) {
    int bits = 62;
    while (((int64_t)1 << (62 - bits)) < a.vocab) --bits;
    if (bits > 50) bits = 50;
    Stats s;
    lay_out(a.vocab, a.rows, (char*)workspace, &s);
    // groups a wavefront takes: as many as leave eight workgroups to a compute unit, eight at most
    // (4, 16 and 32 took 1.01, 1.03 and 1.2 times as long for 2,112 rows of 151,936)
    int64_t per_wave = (int64_t)s.groups * a.rows / ((int64_t)cus * 8 * kScanWaves);
    per_wave = per_wave < 1 ? 1 : per_wave > 8 ? 8 : per_wave;
    return sample<kType>(a, s, (int32_t)per_wave, bits, cus, stream);
}

}  // namespace

size_t sample_workspace_bytes(int64_t vocab, int64_t rows, int) {
    Stats s;
    return lay_out(vocab, rows < kMostRows ? rows : kMostRows, nullptr, &s);
}

hipError_t launch_sample(const SampleArgs& a, asd_dtype dtype, void* workspace, int cus, hipStream_t stream) {
    for (int64_t row = 0; row < a.rows; row += kMostRows) {
        SampleArgs b = a;
        b.rows = a.rows - row < kMostRows ? a.rows - row : kMostRows;
        b.logits = (const char*)a.logits + row * a.row_stride * (dtype == ASD_F32 ? 4 : 2);
        if (a.temperature) b.temperature += row;
        if (a.top_k) b.top_k += row;
        if (a.top_p) b.top_p += row;
        if (a.min_p) b.min_p += row;
        b.uniform += row;
        b.out_token += row;
        if (a.out_prob) b.out_prob += row;
        const hipError_t err = dtype == ASD_F32    ? sample_rows<ASD_F32>(b, workspace, cus, stream)
                               : dtype == ASD_BF16 ? sample_rows<ASD_BF16>(b, workspace, cus, stream)
                                                   : sample_rows<ASD_F16>(b, workspace, cus, stream);
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

}  // namespace asd
