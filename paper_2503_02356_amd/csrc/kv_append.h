// What the calls that rotate share (rotate.hip, kv_append8.hip): their arguments, their checks, one lane's part.
#pragma once
#include <hip/hip_runtime.h>

#include "chunkflow.h"
#include "rotation.h"

namespace cf {

struct TurnArgs {
    const float *inv_freq;
    int rot, interleaved, inverse;
    int units_shift;             // log2 of a row's units
    int n_tokens, n_seqs;
    int chunk;                   // lens: the bounds of the keys of a chunk's segments; else the sequences' lengths
    const int32_t *cu, *lens;
    const int32_t *table;        // pages (tensors that are paged)
    int64_t table_stride, page_stride;
    int pages, shift, n_pages;
    int per_group;               // heads
    int stream;                  // a call so large that its results go past the caches
    TurnTensor t[3];             // without heads: none
    __host__ __device__ int all_groups() const { return t[0].groups + t[1].groups + t[2].groups; }
    void group(int workgroups);  // chooses the groups of heads
};
hipError_t launch_turn_rows(const TurnArgs &a, hipStream_t s);

int check_rotation(const char *who, const cf_rotation &r, int D);
int check_append_rotation(const char *who, const cf_append_rotation *r, int dtype, int D);
int check_append(const cf_kv_append_params *p, const char *who, bool eight_bits);
int check_rows(const char *who, int n_tokens, int D);
TurnArgs turn_args(const cf_rotation *r, int D, int n_tokens, int n_seqs, const int32_t *cu, const int32_t *lens);
void queries_of(TurnArgs &a, const cf_append_rotation *r, int dtype);
void pages_of(TurnArgs &a, const cf_kv_append_params *p);

// Unit u of a row, of group `group` of the heads of all tensors.  where(seq, position): finds them.
template <bool INTERLEAVED, bool STREAM, typename Where>
__device__ __forceinline__ void turn_group(const TurnArgs &a, int row, int u, int group, Where where)
{
    int i = 0;
    if (group >= a.t[0].groups) {
        group -= a.t[0].groups, i = 1;
        if (group >= a.t[1].groups) group -= a.t[1].groups, i = 2;
    }
    const TurnTensor &t = a.t[i];
    const Unit unit(u, 16 << a.units_shift, a.rot, INTERLEAVED);
    const int h0 = group * a.per_group;
    int seq = 0, position = 0;
    auto place = [&]() -> int64_t {
        where(seq, position);
        if (!t.paged) return row * t.y_tok;
        const PageTable table{a.table + (int64_t)seq * a.table_stride, a.pages, a.shift, a.n_pages};
        const int page = table.page_of(position);
        return page < 0 ? -1 : (int64_t)page * a.page_stride + (int64_t)table.row_in_page(position) * t.y_tok;
    };
    turn_heads<INTERLEAVED, STREAM>(t, unit, row, h0, min(h0 + a.per_group, t.n_heads), place,
                                    [&](Turn &turn) { turn.set(a.inv_freq, unit, max(position, 0), a.inverse); });
}

// Workgroup `block` of 256 lanes, a lane to a unit of a row, of which there are `end`.
template <bool INTERLEAVED, bool STREAM>
__device__ __forceinline__ void turn_rows(const TurnArgs &a, int end, int group, int block)
{
    const int row = block * (256 >> a.units_shift) + (threadIdx.x >> a.units_shift), first = __builtin_amdgcn_readfirstlane(row);
    if (first >= end) return;
    const int r = min(row, end - 1);                 // (all lanes look for the sequences)
    const int seq_of_row = sequence_of(a.cu, a.n_seqs, first, r);
    if (row >= end) return;
    turn_group<INTERLEAVED, STREAM>(a, row, threadIdx.x & ((1 << a.units_shift) - 1), group, [&](int &seq, int &position) {
        seq = seq_of_row;
        const NewRows rows(a.cu[seq], a.cu[seq + 1], a.chunk ? a.lens[seq + 1] - a.lens[seq] : a.lens[seq]);
        position = rows.position(row - rows.q0);
    });
}

}  // namespace cf
