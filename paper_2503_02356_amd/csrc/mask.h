// Which keys a query sees.  Position of query row i of a segment: p = i + (Lk - Lq).
//   CausalMask  keys j <= p
//   WindowMask  of these the last `window` ones and the first `sinks` ones:  j <= p and (j > p - window or j < sinks)
// A row's visible keys are the sinks that lie before its window, then one stretch that ends at its position.  Kernels go over tiles of
// keys, so their lists of tiles have the same two parts.
// window is from 1 to 2^31 - 1, sinks from 0 to the keys of a call (its entry points see to that).  Sums that could leave 32 bits with fewer than
// 2^31 - 128 keys have 64 (more keys are 256 GB of keys alone, at one head of 64).
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define CF_BOTH __host__ __device__ inline
#else
#define CF_BOTH inline
#endif

namespace cf {

struct CausalMask {
    static constexpr bool windowed = false;
};
struct WindowMask {
    static constexpr bool windowed = true;
    int window, sinks;
    // Rows that see at most this many keys have probabilities as large as those of a sequence's first rows.
    CF_BOTH bool few(int keys) const { return window + (int64_t)sinks <= keys; }
};

CF_BOTH int at_most(int a, int b) { return a < b ? a : b; }
CF_BOTH int at_least(int a, int b) { return a > b ? a : b; }

// The n visible keys of the row at a position, in ascending order.
template <typename Mask>
struct KeysOfRow;
template <>
struct KeysOfRow<CausalMask> {
    int n;
    CF_BOTH KeysOfRow(const CausalMask &, int position) : n(position + 1) {}
    CF_BOTH int key(int x) const { return x; }
};
template <>
struct KeysOfRow<WindowMask> {
    int n, sinks, gap;                               // keys between the sinks and the window
    CF_BOTH KeysOfRow(const WindowMask &m, int position)
    {
        const int first = at_least(0, position + 1 - m.window);
        sinks = at_most(m.sinks, first);
        gap = first - sinks;
        n = position + 1 - gap;
    }
    CF_BOTH int key(int x) const { return x < sinks ? x : x + gap; }
};

// The rows that see key j of a segment with `prefix` = Lk - Lq end here (they begin at row max(0, j - prefix)).
CF_BOTH int rows_that_see(const CausalMask &, int, int, int lq) { return lq; }
CF_BOTH int rows_that_see(const WindowMask &m, int j, int prefix, int lq)
{
    return j < m.sinks ? lq : (int)((int64_t)j + m.window - prefix < lq ? (int64_t)j + m.window - prefix : lq);
}

// The key tiles of `TILE` keys that rows at positions [first_position, keys) see, `keys` being one more than the last of them: tile t starts
// at key start(t), the one behind it at next(t, start(t)).
template <int TILE, typename Mask>
struct KeyTiles;
template <int TILE>
struct KeyTiles<TILE, CausalMask> {
    int n;
    CF_BOTH KeyTiles(const CausalMask &, int, int keys) : n((keys + TILE - 1) / TILE) {}
    CF_BOTH int start(int t) const { return t * TILE; }
    CF_BOTH int next(int, int start) const { return start + TILE; }
};
template <int TILE>
struct KeyTiles<TILE, WindowMask> {
    int n, sinks, gap;                               // tiles of sinks, tiles that nobody sees
    CF_BOTH KeyTiles(const WindowMask &m, int first_position, int keys)
    {
        const int first = at_least(0, first_position + 1 - m.window);
        sinks = (at_most(m.sinks, first) + TILE - 1) / TILE;
        gap = at_least(0, first / TILE - sinks);
        n = at_least((keys + TILE - 1) / TILE - gap, sinks);        // (keys: fewer than the positions where a cache holds fewer)
    }
    CF_BOTH int start(int t) const { return (t < sinks ? t : t + gap) * TILE; }
    CF_BOTH int next(int t, int) const { return start(t + 1); }
};

// The query tiles of `TILE` rows, [first, end), with a row that sees one of the keys [key, key_end) of a segment.
template <int TILE>
struct QueryTiles {
    int first, end;
    CF_BOTH QueryTiles(const CausalMask &, int key, int, int prefix, int lq) : first(at_least(0, key - prefix) / TILE), end((lq + TILE - 1) / TILE) {}
    CF_BOTH QueryTiles(const WindowMask &m, int key, int key_end, int prefix, int lq)
        : first(at_least(0, key - prefix) / TILE), end((at_least(0, key < m.sinks ? lq : rows_that_see(m, key_end - 1, prefix, lq)) + TILE - 1) / TILE)
    {
    }
};

}  // namespace cf
