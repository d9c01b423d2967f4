// What the matrix kernels of the paged calls share: tiles of token-head rows, and where a tile's keys stand.
#pragma once
#include "mfma_common.h"
#include "paged.h"

namespace cf {
namespace {

// The call's arguments, loaded (again) where this is called.  What a workgroup needs only at its end would stand in scalar registers all the
// way, and there are too few of them: those of the loops over keys would go to and fro instead.
__device__ __forceinline__ const PagedArgs &arguments()
{
    auto p = (const CF_CONSTANT PagedArgs *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const PagedArgs *)p;
}

// A tile: up to BM token-head rows of a sequence and a key/value head.
struct TileRows {
    int seq, q0;                 // sequence, its first row of q
    int row0, rows;              // first row of the tile among the sequence's token-head rows, and how many it has
    int first_position;
    int G, kh;                   // query heads of a key/value head, key/value head
    int key0;                    // keys in one piece: the sequence's first row of them

    __device__ __forceinline__ int token(int x) const { return (row0 + x) / G; }
    __device__ __forceinline__ int position(int x) const { return at_least(-1, first_position + token(x)); }
    // row of q and head of the tile's row x
    __device__ __forceinline__ void find(int x, int64_t &row, int &head) const
    {
        const int i = token(x);
        row = q0 + i, head = kh * G + (row0 + x - i * G);
    }
    __device__ __forceinline__ int64_t flat(const PagedArgs &a, int x) const
    {
        int64_t row;
        int h;
        find(x, row, h);
        return row * a.p.n_q_heads + h;
    }
    __device__ __forceinline__ char *out(const PagedArgs &a, int x) const
    {
        int64_t row;
        int h;
        find(x, row, h);
        return (char *)a.p.o + (row * a.p.o_stride_tok + (int64_t)h * a.p.o_stride_head) * (a.p.dtype == CF_BF16 ? 2 : 4);
    }
    __device__ __forceinline__ void put_lse(const PagedArgs &a, int x, float lse) const
    {
        int64_t row;
        int h;
        find(x, row, h);
        if (a.p.lse) a.p.lse[(int64_t)h * a.p.n_tokens + row] = lse;
    }
};

// Tile `rank`, counted from the last one of the last sequence (places: pages.h).
// CHUNK: kv_lens holds the bounds of the sequences' keys, which stand in one piece.
template <int BM, bool CHUNK = false>
__device__ __forceinline__ bool find_tile(const PagedArgs &a, int rank, TileRows &t)
{
    const cf_attn_paged_params &p = a.p;
    const int32_t *cu = p.cu_seqlens_q;
    const int lane = threadIdx.x & 63, G = t.G;
    const int place = (int)places_most(p.n_tokens, p.n_seqs, G, BM) - 1 - rank;
    int lo = 0, hi = p.n_seqs;
    while (hi - lo > 64) {
        const int step = (hi - lo + 63) / 64, g = lo + lane * step;
        const unsigned long long before = __ballot(g < hi && first_place(cu[min(g, hi - 1)], g, G, BM) <= place);
        lo += (63 - __clzll((long long)before)) * step;      // (lane 0 always says yes)
        hi = min(hi, lo + step);
    }
    const int g = min(lo + lane, hi - 1);
    const int begin = cu[g], end = cu[g + 1], key0 = p.kv_lens[g], keys = CHUNK ? p.kv_lens[g + 1] - key0 : key0;
    const int last = 63 - __clzll((long long)__ballot(lo + lane < hi && first_place(begin, g, G, BM) <= place));
    t.seq = uniform(lo + last);
    const int q0 = __builtin_amdgcn_readlane(begin, last), q1 = __builtin_amdgcn_readlane(end, last);
    const NewRows rows(q0, q1, __builtin_amdgcn_readlane(keys, last));
    t.q0 = q0;
    t.key0 = CHUNK ? __builtin_amdgcn_readlane(key0, last) : 0;
    const TileSpan span(place, q0, rows.lq, t.seq, G, BM);
    t.row0 = span.row0, t.rows = span.rows;
    t.first_position = rows.first_position;
    return t.rows > 0;
}

// Where a workgroup's keys stand.  SIZE: bytes of an element.  CHUNK: in one piece, one page without end.
template <int SIZE, bool CHUNK = false>
struct KeySource : KeyPlaces {
    const CF_CONSTANT int32_t *table;        // the sequence's row (nothing writes it meanwhile: scalar loads, which no copy in flight holds up)
    unsigned row_bytes;
    int64_t page_bytes;
    const char *k, *v;           // of this head
    __device__ __forceinline__ KeySource(const PagedArgs &a, const TileRows &t, int keys)
        : KeyPlaces{a.shift, a.p.n_pages, keys - 1}, table((const CF_CONSTANT int32_t *)a.p.block_table + (int64_t)t.seq * a.p.table_stride),
          row_bytes((unsigned)(a.p.kv_stride_tok * SIZE)), page_bytes(a.p.page_stride * SIZE),
          k((const char *)a.p.k_pages + ((int64_t)t.key0 * a.p.kv_stride_tok + (int64_t)t.kh * a.p.kv_stride_head) * SIZE),
          v((const char *)a.p.v_pages + ((int64_t)t.key0 * a.p.kv_stride_tok + (int64_t)t.kh * a.p.kv_stride_head) * SIZE)
    {
    }
    // The table's entry for keys key .. (a group that lies in one page).  Looked at (is_page) only where the page is used, a tile later: the
    // load has come by then.
    __device__ __forceinline__ int entry(int key) const { return CHUNK ? 0 : table[column(key)]; }
    __device__ __forceinline__ bool is_page(int entry) const { return CHUNK || KeyPlaces::is_page(entry); }
    __device__ __forceinline__ bool none(int entry, int key) const { return !is_page(entry) || key > last; }
    __device__ __forceinline__ int page_of(int key) const
    {
        const int page = entry(key);
        return none(page, key) ? -1 : page;
    }
    __device__ __forceinline__ int64_t offset(int page, int key) const
    {
        if (CHUNK) return (int64_t)key * row_bytes;
        return KeyPlaces::offset(page, key, page_bytes, row_bytes);
    }
};

}  // namespace
}  // namespace cf
