// What the kernels of the attention over a cache of 8 bits share: a call's arguments, one row pair by pair.
#pragma once
#include "paged.h"
#include "pages8.h"

namespace cf {

struct Paged8Args {
    PagedArgs a;                         // (first: arguments() of paged_tiles.h looks there)
    const float *k_scales, *v_scales;
    int64_t scale_page, scale_head;
    __device__ __forceinline__ int64_t scale_at(int page, int row_in_page, int kh) const
    {
        return (int64_t)page * scale_page + (int64_t)kh * scale_head + row_in_page / kBlock8;
    }
};

// paged_row of paged.h over 8 bits.
template <int D, int UNROLL, int TILE, typename Q>
__device__ inline RowSums<float, D> paged8_row(const Paged8Args &c, const PageTable &table, int position, int kh, const KeyTiles<TILE, WindowMask> &tiles,
                                               int first, int end, Q q)
{
    const PagedArgs &a = c.a;
    const cf_attn_paged_params &p = a.p;
    const int lane = threadIdx.x & 63;
    RowSums<float, D> r;
    for (int t = first; t < end; ++t) {
        const int j = tiles.start(t) + lane;
        const bool seen = lane < TILE && j <= position && (j > position - a.mask.window || j < a.mask.sinks);
        const int page = seen ? table.page_of(j) : -1;
        const int64_t at = (int64_t)max(page, 0) * p.page_stride + (int64_t)table.row_in_page(j) * p.kv_stride_tok + (int64_t)kh * p.kv_stride_head;
        const int64_t scale = c.scale_at(max(page, 0), table.row_in_page(j), kh);
        float s = -INFINITY, v_factor = 0.f;
        if (page >= 0) {
            const unsigned *k = (const unsigned *)((const char *)p.k_pages + at);
            float d = 0.f;
            for_elements<D / 4, UNROLL>([&](int x) {
                const int w = (int)k[x];
                d += q(4 * x) * __builtin_amdgcn_cvt_f32_fp8(w, 0);
                d += q(4 * x + 1) * __builtin_amdgcn_cvt_f32_fp8(w, 1);
                d += q(4 * x + 2) * __builtin_amdgcn_cvt_f32_fp8(w, 2);
                d += q(4 * x + 3) * __builtin_amdgcn_cvt_f32_fp8(w, 3);
            });
            s = d * factor8(c.k_scales[scale]) * p.softmax_scale;
            v_factor = factor8(c.v_scales[scale]);
        }
        const unsigned long long some = __ballot(page >= 0);
        if (some == 0) continue;
        const float m_new = fmaxf(r.m, wave_max(s)), ref = m_new == -INFINITY ? 0.f : m_new;
        const float pr = page >= 0 ? expf(s - ref) : 0.f, corr = expf(r.m - ref);
        r.z = r.z * corr + wave_sum(pr);
        for (int x = 0; x < D / 64; ++x) r.acc[x] *= corr;
        for (unsigned long long left = some; left != 0; left &= left - 1) {
            const int jj = __ffsll((long long)left) - 1;
            const float pj = __shfl(pr, jj), fj = __shfl(v_factor, jj);
            const char *v = (const char *)p.v_pages + __shfl(at, jj) + lane;
            for (int x = 0; x < D / 64; ++x) r.acc[x] += pj * (fj * __builtin_amdgcn_cvt_f32_fp8((int)(unsigned char)v[64 * x], 0));
        }
        r.m = m_new;
    }
    return r;
}

// Matrix kernels (attn_paged8_mfma.hip); as those of paged.h.
hipError_t launch_paged8_mfma(const Paged8Args &a, hipStream_t s);
int64_t paged8_mfma_launch_size(const PagedArgs &a);
void cut_paged8_mfma(PagedArgs &a);

}  // namespace cf
