// A paged cache of 8 bits: its numbers' powers of two, and which blocks of it a call adds to.  Runs on the CPU too.
#pragma once
#include <string.h>

#include "pages.h"

namespace cf {

constexpr int kBlock8 = 16;              // tokens that share a scale (CF_KV8_BLOCK)
constexpr int kLeast8 = -110;            // exponent of the least scale that is written: below it e4m3 times it would leave bf16's normal numbers
constexpr int kMost8 = 120;              // of the largest that a block of finite fp32 elements needs

CF_BOTH unsigned bits_of(float x)
{
    unsigned u;
    memcpy(&u, &x, 4);
    return u;
}
CF_BOTH float float_of(unsigned u)
{
    float x;
    memcpy(&x, &u, 4);
    return x;
}
CF_BOTH float power8(int e) { return float_of((unsigned)(e + 127) << 23); }      // 2^e, -126 .. 127

// The least e from kLeast8 on with most <= 448 * 2^e, for a finite most >= 0:  most = 1.f * 2^E,  448 = 1.75 * 2^8.
CF_BOTH int exponent_for(float most)
{
    const unsigned u = bits_of(most);
    return at_least(kLeast8, (int)(u >> 23) - 127 - 8 + ((u & 0x7fffff) > 0x600000));
}
// The exponent that a scale in the pages stands for, -127 .. 127, or 128: NaN.
CF_BOTH int exponent_of(float scale) { return (int)(bits_of(scale) >> 23 & 255) - 127; }
// What a scale multiplies with: its exponent alone (as the conversion instructions of the matrix kernels take it).
CF_BOTH float factor8(float scale)
{
    const unsigned e = bits_of(scale) >> 23 & 255;
    return float_of(e == 0 ? 0x400000u : e == 255 ? 0x7fc00000u : e << 23);
}
// 2^-e, by which elements are multiplied that a block of exponent e, kLeast8 .. 128, takes (128: NaN whatever they are).
CF_BOTH float inverse8(int e) { return factor8(power8(-at_most(127, e))); }

// Workgroup id of `all` (an even number) does one or the other half of a pair, 8 pairs in 16 workgroups: halves are 8 workgroups apart (behind the last 16, as
// many as are left there).
struct HeadPair {
    int pair, second;
    CF_BOTH HeadPair(int id, int all)
    {
        const int whole = all & ~15, half = id < whole ? 8 : (all - whole) / 2, begin = id < whole ? id & ~15 : whole;
        second = id - begin >= half;
        pair = begin / 2 + (id - begin) - (second ? half : 0);
    }
};

// The blocks of 16 keys that a sequence's new rows go into, [first, first + n), and those of all sequences in one list: sequence g's from place
// first(cu_seqlens_q[g], g) on.  Lq rows touch (Lq + 14) / 16 + 1 blocks at most, and two sequences' places are Lq / 16 + 2, rounded either way, apart; or, where
// that makes fewer places in all (single tokens), a place for each row, since Lq rows touch no more than Lq blocks.
struct BlockPlaces {
    bool of_rows;
    CF_BOTH BlockPlaces(int64_t tokens, int64_t seqs) : of_rows(tokens < tokens / kBlock8 + 2 * seqs) {}
    CF_BOTH int first(int begin, int seq) const { return of_rows ? begin : begin / kBlock8 + 2 * seq; }
    CF_BOTH int64_t all(int64_t tokens, int64_t seqs) const { return of_rows ? tokens : tokens / kBlock8 + 2 * seqs; }
};
struct NewBlocks {
    int begin, end;                      // positions of the new rows
    int first, n;
    CF_BOTH NewBlocks(const NewRows &rows) : begin(at_least(0, rows.first_position)), end(rows.first_position + rows.lq), first(begin / kBlock8), n(0)
    {
        if (end > begin) n = (end - 1) / kBlock8 - first + 1;
    }
};

}  // namespace cf
