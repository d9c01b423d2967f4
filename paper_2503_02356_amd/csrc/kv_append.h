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
    TurnTensor t[3];             // without heads: none
    __host__ __device__ int all_groups() const { return t[0].groups + t[1].groups + t[2].groups; }
    void group();                // chooses the groups of heads
};
hipError_t launch_turn_rows(const TurnArgs &a, hipStream_t s);

int check_rotation(const char *who, const cf_rotation &r, int D);
int check_append_rotation(const char *who, const cf_append_rotation *r, int dtype, int D);
int check_append(const cf_kv_append_params *p, const char *who, bool eight_bits);
int check_rows(const char *who, int n_tokens, int D);
TurnArgs turn_args(const cf_rotation *r, int D, int n_tokens, int n_seqs, const int32_t *cu, const int32_t *lens);
void queries_of(TurnArgs &a, const cf_append_rotation *r, int dtype);
void pages_of(TurnArgs &a, const cf_kv_append_params *p);

// Unit u of a row, of group `group` of the heads of all tensors.
template <bool INTERLEAVED>
__device__ __forceinline__ void turn_group(const TurnArgs &a, int row, int u, int position, int seq, int group)
{
    int i = 0;
    if (group >= a.t[0].groups) {
        group -= a.t[0].groups, i = 1;
        if (group >= a.t[1].groups) group -= a.t[1].groups, i = 2;
    }
    const TurnTensor &t = a.t[i];
    const Unit unit(u, a.rot, INTERLEAVED);
    int64_t y_at = row * t.y_tok;
    if (t.paged) {
        const PageTable table{a.table + (int64_t)seq * a.table_stride, a.pages, a.shift, a.n_pages};
        const int page = table.page_of(position);
        if (page < 0) return;
        y_at = (int64_t)page * a.page_stride + (int64_t)table.row_in_page(position) * t.y_tok;
    }
    Turn turn;
    if (t.turned && unit.turned) turn.set(a.inv_freq + 8 * u, max(position, 0), a.inverse);
    const int h0 = group * a.per_group;
    turn_heads<INTERLEAVED>(t, turn, unit, row, y_at, h0, min(h0 + a.per_group, t.n_heads));
}

}  // namespace cf
