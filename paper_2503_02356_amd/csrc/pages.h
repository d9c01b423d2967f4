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

}  // namespace cf
