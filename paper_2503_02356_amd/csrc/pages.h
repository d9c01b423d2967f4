// Keys and values in pages: where key j of a sequence stands, and which positions its rows have.  Whatever a table or a length holds, no
// index that leaves these functions is out of the pages.
#pragma once
#include "mask.h"

namespace cf {

struct PageTable {
    const int32_t *row;          // the sequence's row of the block table
    int pages, shift, n_pages;   // columns, log2 of a page's tokens, pages that there are
    CF_BOTH int capacity() const { return pages << shift; }
    // The page of key j, -1: none.
    CF_BOTH int page_of(int j) const
    {
        if (j < 0 || (j >> shift) >= pages) return -1;
        const int page = row[j >> shift];
        return page >= 0 && page < n_pages ? page : -1;
    }
    CF_BOTH int row_in_page(int j) const { return j & ((1 << shift) - 1); }
};

// The rows of a sequence: row i is row q0 + i of q, at position(i); a negative position, of a row that sees nothing, is -1.
struct NewRows {
    int q0, lq, first_position;
    CF_BOTH int position(int i) const { return at_least(-1, first_position + i); }
    CF_BOTH NewRows(int begin, int end, int kv_len) : q0(begin), lq(end - begin), first_position(at_least(kv_len, 0) - (end - begin)) {}
};

// Token-head rows of a sequence and a key/value head: row x is token x / G, head x % G of the group.  They go into tiles of BM; the tiles of all
// sequences have places, sequence g's from cu_seqlens_q[g] * G / BM + g on, which leaves room for its last, partly filled one.
CF_BOTH int first_place(int begin, int seq, int G, int BM) { return begin * G / BM + seq; }
CF_BOTH int64_t places_most(int64_t tokens, int64_t seqs, int64_t G, int64_t BM) { return tokens * G / BM + seqs; }
struct TileSpan {
    int row0, rows;              // first row of the tile at `place` among its sequence's, and how many it has (<= 0: none)
    CF_BOTH TileSpan(int place, int begin, int lq, int seq, int G, int BM)
        : row0((place - first_place(begin, seq, G, BM)) * BM), rows(at_most(BM, lq * G - row0))
    {
    }
};

// The keys that rows up to position `highest` may see: as many as the table has columns for.
CF_BOTH int keys_within(int highest, int pages, int shift) { return at_most(highest + 1, pages << shift); }

// Where the keys [0, last] of a sequence stand, for kernels that read a group of consecutive keys of one page at once (a multiple of 16 keys,
// aligned to its size, no larger than a page): the group's column of the table, looked at only where the page is used.
struct KeyPlaces {
    int shift, n_pages, last;
    CF_BOTH int column(int key) const { return at_most(key, last) >> shift; }
    CF_BOTH bool is_page(int entry) const { return (unsigned)entry < (unsigned)n_pages; }
    // Is there no key of the group from `key` on?  And the group's last row that may be read, counted from its first.
    CF_BOTH bool none(int entry, int key) const { return !is_page(entry) || key > last; }
    CF_BOTH int room(int key) const { return last - key; }
    // Bytes from the first page's first row.
    CF_BOTH int64_t offset(int page, int key, int64_t page_bytes, unsigned row_bytes) const
    {
        return page * page_bytes + (int64_t)(key & ((1 << shift) - 1)) * row_bytes;
    }
};

}  // namespace cf
