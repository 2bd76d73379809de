// The attention kernels' walk over a sequence of `end` tokens, from its unit `from` on, with the kernels' own
// index arithmetic: every token is visited once, every entry of the page table that is read is there, every
// token that counts as there has its own page and slot, and every loop ends.
#include <stdio.h>
#include <stdlib.h>

#include <initializer_list>

#include "asd_tokens.h"

using namespace asd;

static long failures = 0;

static void fail(const char* what, long long end, long long page_size, long long at) {
    if (++failures <= 20) printf("%s: %lld tokens, pages of %lld, at %lld\n", what, end, page_size, at);
}

static void strip_is_sound(const Tokens& s, int64_t entries, int64_t first, Token strip) {
    for (Token lane = 0; lane < kStrip; ++lane) {
        const int64_t real = first + lane;
        const Token t = strip + lane;
        const int64_t last = s.end - (int64_t)1;
        const int64_t page = (real < last ? real : last) / s.page_size;
        if ((int64_t)s.entry(t) != page || page >= entries) fail("entry", s.end, s.page_size, real);
        if (s.has(t) != (real <= last)) fail("has", s.end, s.page_size, real);
        if (s.has(t) && (int64_t)s.slot(t) != real % s.page_size) fail("slot", s.end, s.page_size, real);
    }
}

static void walk(int64_t end, int64_t page_size, int64_t units_back) {
    Tokens s;
    s.end = (Token)end;
    s.page_size = (uint32_t)page_size;
    page_divisor((int32_t)page_size, &s.magic, &s.shift);
    const int64_t entries = (end + page_size - 1) / page_size, units = (end + kUnit - 1) / kUnit;
    const int64_t from = units > units_back ? units - units_back : 0;
    const Token strip_end = (Token)(units * kUnit < end ? units * kUnit : end);
    int64_t visited = 0;
    for (int wave = 0; wave < kAttendWaves; ++wave) {
        int64_t real = from * kUnit + wave * kStrip;
        long turns = 0;
        for (Token strip = (Token)(from * kUnit) + wave * kStrip; strip < strip_end; strip += kUnit, real += kUnit) {
            if (++turns > units_back + 1) {
                fail("no end", end, page_size, real);
                break;
            }
            for (int ahead = 0; ahead < 3; ++ahead)
                strip_is_sound(s, entries, real + ahead * (int64_t)kUnit, strip + ahead * kUnit);
            for (Token lane = 0; lane < kStrip; ++lane) visited += s.has(strip + lane);
        }
    }
    if (visited != end - from * (int64_t)kUnit) fail("visited", end, page_size, visited);
}

int main() {
    const int64_t top = 0x7fffffff;
    for (int64_t end = top; end > top - 700; --end)
        for (int64_t size : {(int64_t)1, (int64_t)2, (int64_t)7, (int64_t)16, (int64_t)24, (int64_t)126,
                             (int64_t)65537, (int64_t)1 << 20, (int64_t)1 << 30, top - 1, top})
            walk(end, size, 6);
    srand(5);
    for (int i = 0; i < 20000; ++i) {
        const int64_t end = 1 + (int64_t)rand() * (i % 3 == 0 ? 1 : 0) % top + rand() % 3000;
        walk(end < top ? end : top, 1 + rand() % (i % 2 ? 4000 : 1 << 30), 5);
    }
    // rows of a chain: row p sees `past` tokens fewer than p + 1
    for (int64_t past : {-(top - 1), -(top - 5), -(int64_t)100, (int64_t)-33, (int64_t)-32, (int64_t)-31, (int64_t)-1,
                         (int64_t)0, (int64_t)1, (int64_t)31, (int64_t)32, (int64_t)33, (int64_t)5000})
        for (int32_t p : {0, 1, 2, 30, 31, 32, 63, 64, 5000}) {
            const int64_t n = p + 1 - past, want = n < 0 ? 0 : n > 32 ? 32 : n;
            if (chain_sees(p, (int32_t)past) != want) fail("chain", p, past, want);
        }
    printf("%ld failures\n", failures);
    return failures != 0;
}
