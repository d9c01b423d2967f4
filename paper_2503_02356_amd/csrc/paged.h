// What the kernels of the paged calls share: a call's arguments, one row pair by pair, the parts that a long cache is cut into.
#pragma once
#include <hip/hip_runtime.h>

#include "chunkflow.h"
#include "pages.h"
#include "scalar_rows.h"

namespace cf {

struct PagedArgs {
    cf_attn_paged_params p;
    WindowMask mask;             // no window: one of all keys
    int shift;                   // log2(page_size)
    // Parts of a tile's keys (tile: some rows of a sequence and a key/value head), each of so many key tiles of 64, by workgroups of their own:
    // parts > 1: row r = token * Hq + head of part x leaves its unnormalised result at part_o[(x * T * Hq + r) * D] and its maximum (log2
    // units) and sum at part_ml[r * parts + x]; a part without keys leaves the maximum -infinity.
    int parts, tiles_per_part;
    float *part_o;
    float2 *part_ml;
    __device__ __forceinline__ PageTable table(int seq) const
    {
        return PageTable{p.block_table + (int64_t)seq * p.table_stride, p.pages_per_seq, shift, p.n_pages};
    }
    __device__ __forceinline__ NewRows rows(int seq) const { return NewRows(p.cu_seqlens_q[seq], p.cu_seqlens_q[seq + 1], p.kv_lens[seq]); }
};

// One row's softmax over the visible keys of tiles [first, end) of `tiles` (TILE <= 64 keys, a lane to a key): maximum (natural units), sum and unnormalised result, element
// lane + 64 t.
template <typename T, int D>
struct RowSums {
    float m = -INFINITY, z = 0.f, acc[D / 64] = {};
};
// key0: row of the pages that the table counts from (0 but for keys in one piece).
template <typename T, int D, int UNROLL, int TILE, typename Q>
__device__ inline RowSums<T, D> paged_row(const PagedArgs &a, const PageTable &table, int position, int kh, const KeyTiles<TILE, WindowMask> &tiles,
                                          int first, int end, Q q, int key0 = 0)
{
    const cf_attn_paged_params &p = a.p;
    const int lane = threadIdx.x & 63;
    RowSums<T, D> r;
    for (int t = first; t < end; ++t) {
        const int j = tiles.start(t) + lane;
        const bool seen = lane < TILE && j <= position && (j > position - a.mask.window || j < a.mask.sinks);
        const int page = seen ? table.page_of(j) : -1;
        const int64_t at = (int64_t)max(page, 0) * p.page_stride + (int64_t)(key0 + table.row_in_page(j)) * p.kv_stride_tok + (int64_t)kh * p.kv_stride_head;
        float s = -INFINITY;
        if (page >= 0) {
            const T *k = (const T *)p.k_pages + at;
            float d = 0.f;
            for_elements<D, UNROLL>([&](int x) { d += q(x) * ld(k + x); });
            s = d * p.softmax_scale;
        }
        const unsigned long long some = __ballot(page >= 0);
        if (some == 0) continue;
        const float m_new = fmaxf(r.m, wave_max(s)), ref = m_new == -INFINITY ? 0.f : m_new;
        const float pr = page >= 0 ? expf(s - ref) : 0.f, corr = expf(r.m - ref);
        r.z = r.z * corr + wave_sum(pr);
        for (int x = 0; x < D / 64; ++x) r.acc[x] *= corr;
        for (unsigned long long left = some; left != 0; left &= left - 1) {
            const int jj = __ffsll((long long)left) - 1;
            const float pj = __shfl(pr, jj);
            const int64_t row = __shfl(at, jj);
            const T *v = (const T *)p.v_pages + row;
            for (int x = 0; x < D / 64; ++x) r.acc[x] += pj * ld(v + lane + 64 * x);
        }
        r.m = m_new;
    }
    return r;
}

constexpr int kMostParts = 64;       // (a lane of the joining wavefront to a part)
// bf16 matrix kernel (attn_paged_mfma.hip).  A windowed chunk of few rows goes by it too, as a cache of one page (launch_window_few).
hipError_t launch_paged_mfma(const PagedArgs &a, hipStream_t s);
int64_t paged_mfma_launch_size(const PagedArgs &a);      // work-items
// Cuts a call's keys into parts: sets parts and tiles_per_part.
void cut_paged_mfma(PagedArgs &a);
// fp32 matrix kernel (attn_paged_f32.hip): the same.
hipError_t launch_paged_f32(const PagedArgs &a, hipStream_t s);
int64_t paged_f32_launch_size(const PagedArgs &a);
void cut_paged_f32(PagedArgs &a);
// Joins the parts of every row (one call's parts > 1).
hipError_t launch_paged_join(const PagedArgs &a, hipStream_t s);

}  // namespace cf
