// Places of a sequence's tokens in its page table, as the attention kernels walk over them.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define ASD_BOTH __host__ __device__ __forceinline__
#else
#define ASD_BOTH inline
#endif

namespace asd {

// A token's number.  Without sign: a sequence may have 2^31 - 1 tokens, and the strips that are asked for
// ahead of its last one begin behind them, where a signed number would wrap to one before the end.
typedef uint32_t Token;

constexpr Token kStrip = 32;              // tokens a wavefront takes at a time
constexpr int kAttendWaves = 4;
constexpr Token kUnit = kStrip * kAttendWaves;

struct Tokens {
    Token end;                            // there are 0 .. end - 1, at least one
    uint32_t page_size, magic;
    int32_t shift;

    // t / page_size = (2 t magic / 2^32) >> shift for t < 2^31: with 2^shift >= page_size and
    // magic = ceil(2^(31 + shift) / page_size) the excess stays below 1 / page_size.
    ASD_BOTH Token page(Token t) const { return (Token)((uint64_t)(2 * t) * magic >> 32) >> shift; }
    ASD_BOTH bool has(Token t) const { return t < end; }
    // The token's entry of the page table; of those behind the last one, its.
    ASD_BOTH Token entry(Token t) const { return page(t < end ? t : end - 1); }
    // Its place in that page, where it is there.
    ASD_BOTH Token slot(Token t) const { return t - page(t) * page_size; }
};

inline void page_divisor(int32_t page_size, uint32_t* magic, int32_t* shift) {
    *shift = 0;
    while (((int64_t)1 << *shift) < page_size) ++*shift;
    *magic = (uint32_t)((((uint64_t)1 << (31 + *shift)) + page_size - 1) / page_size);
}

// How many tokens from a strip's first one on row p of a chain sees, 32 at most; `past` is the strip's first
// token, counted from the block's.
ASD_BOTH int32_t chain_sees(int32_t p, int32_t past) {
    const int32_t n = p + 1 - (past > -(int32_t)kStrip ? past : -(int32_t)kStrip);
    return n < 0 ? 0 : n > (int32_t)kStrip ? (int32_t)kStrip : n;
}

}  // namespace asd
