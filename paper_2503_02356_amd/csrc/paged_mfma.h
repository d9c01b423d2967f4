// What the bf16 matrix kernels of the paged calls share (attn_paged_mfma.hip, attn_paged8_mfma.hip): the running softmax of a block of scores, a
// wavefront's rows over tiles of bf16 keys and values.
#pragma once
#include "paged_tiles.h"

namespace cf {
namespace {

using F = Mfma<16>;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLazy = 8.f;                 // log2 units a row maximum may exceed the running reference (attn_mfma_fwd.hip)

__device__ __align__(16) unsigned zeros[64];                 // a row of zeros

// The queries of the tile's row x, 8 elements from d on; a negative scale is put on them, a scale of 0 makes them 0 (the row maximum is
// taken before scaling, which needs a positive factor).
__device__ __forceinline__ bf16x8 query(const PagedArgs &a, const TileRows &t, int x, int d)
{
    int64_t row;
    int h;
    t.find(x, row, h);
    i32x4 w = *(const i32x4 *)((const char *)a.p.q + (row * a.p.q_stride_tok + (int64_t)h * a.p.q_stride_head + d) * 2);
    const int flip = a.p.softmax_scale < 0.f ? 0x80008000 : 0, keep = a.p.softmax_scale == 0.f ? 0 : -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (w[e] ^ flip) & keep;
    return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ float score_factor(const PagedArgs &a) { return a.p.softmax_scale == 0.f ? 1.f : fabsf(a.p.softmax_scale) * kLog2e; }

// Scores of a block of KB x 16 keys from key `start` on, for QB x 16 rows, become P: masks, the running softmax (m: maximum so far in log2 units,
// or rather its reference, see kLazy; l: this lane's part of the sum; o is rescaled with them).
// lowest, highest: positions of the wavefront's rows.  groups: hidden groups of 16 keys, a bit each.
template <int D, int KB, int QB>
__device__ __forceinline__ void settle(f32x4 (&s)[KB][QB], float (&m)[QB], float (&l)[QB], f32x4 (&o)[D / 16][QB], const int (&pos)[QB],
                                       const WindowMask &mask, int start, int lowest, int highest, unsigned groups, float c2)
{
    constexpr int NS = KB * F::R, DB = D / 16;
    const int group = F::group();
    if (start + 16 * KB - 1 > lowest) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int lim = pos[qb] - start - group * 4;
#pragma unroll
            for (int i = 0; i < NS; ++i)
                if (F::place(i) > lim) s[i / F::R][qb][i % F::R] = -INFINITY;
        }
    }
    if (start <= highest - mask.window && start + 16 * KB > mask.sinks) {
        const int from = mask.sinks - start - group * 4;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const unsigned gap = hidden_keys(mask, pos[qb]);
#pragma unroll
            for (int i = 0; i < NS; ++i)
                if ((unsigned)(F::place(i) - from) < gap) s[i / F::R][qb][i % F::R] = -INFINITY;
        }
    }
    if (groups != 0) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
            if (groups >> kb & 1) {
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                    for (int i = 0; i < F::R; ++i) s[kb][qb][i] = -INFINITY;
            }
    }
    // The running softmax, rescaled only where a maximum has grown by more than 2^kLazy; a row without a key so far has none.
    float mx2[QB];
    bool grow = false;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        float mx = s[0][qb][0];
#pragma unroll
        for (int i = 1; i < NS; ++i) mx = fmaxf(mx, s[i / F::R][qb][i % F::R]);
        mx2[qb] = mx * c2;
        grow = grow || mx2[qb] > m[qb] + kLazy;
    }
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const float mx = max_over_groups<16>(mx2[qb]), m_new = mx > m[qb] + kLazy ? mx : m[qb];
            const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[qb] - m_new);
            m[qb] = m_new;
            l[qb] *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db][qb] *= alpha;
        }
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const float ref = m[qb] == -INFINITY ? 0.f : m[qb];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / F::R][qb][i % F::R], c2, -ref));
            s[i / F::R][qb][i % F::R] = e;
            sum += e;
        }
        l[qb] += sum;
    }
}

// One block of KB x 16 keys, for QB x 16 rows: scores of a K tile, masks, the running softmax, P.
// RESIDUAL: P enters the second product with the bf16 rounding of what its own rounding leaves (16 bits and more).
template <int D, int KB, int QB, bool RESIDUAL>
struct Rows {
    static constexpr int KS = D / F::K, DB = D / 16;
    bf16x8 q[QB][KS];
    f32x4 o[DB][QB];
    float m[QB], l[QB];          // maximum so far (log2 units; its reference, see kLazy), this lane's part of the sum
    int pos[QB];                 // of the lane's row

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            m[qb] = -INFINITY, l[qb] = 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db][qb] = F::zero();
        }
    }
    __device__ __forceinline__ void scores(const char *k_tile, const LaneOffsets<D, 16> &lo, const WindowMask &mask, int start, int lowest, int highest,
                                           unsigned groups, float c2, f32x4 (&s)[KB][QB])
    {
        bf16x8 ka[KB][KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) ka[kb][ks] = lds_read_b128(k_tile + kb * (16 * 2 * D) + lo.row_unit[ks]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) s[kb][qb] = F::zero();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int x = 0; x < QB; ++x) {
                    const int qb = kb & 1 ? QB - 1 - x : x;
                    s[kb][qb] = F::mul(ka[kb][ks], q[qb][ks], s[kb][qb]);
                }
        settle<D, KB, QB>(s, m, l, o, pos, mask, start, lowest, highest, groups, c2);
    }
    __device__ __forceinline__ void values(const char *v_tile, const LaneOffsets<D, 16> &lo, const f32x4 (&s)[KB][QB])
    {
#pragma unroll
        for (int t = 0; t < KB * 16 / F::K; ++t) {
            bf16x8 pb[QB], rest[QB];
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = s[(8 * t + e) / F::R][qb][(8 * t + e) % F::R];
                pb[qb] = pack8(f);
                if (RESIDUAL) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] -= (float)pb[qb][e];
                    rest[qb] = pack8(f);
                }
            }
            const char *va = v_tile + t * (F::K * 2 * D);
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const bf16x8 x = lds_read_tr_pair(va + lo.tr_lo[db], va + lo.tr_hi(db));
#pragma unroll
                for (int y = 0; y < QB; ++y) {
                    const int qb = db & 1 ? QB - 1 - y : y;
                    o[db][qb] = F::mul(x, pb[qb], o[db][qb]);
                    if (RESIDUAL) o[db][qb] = F::mul(x, rest[qb], o[db][qb]);
                }
            }
        }
    }
};

__device__ __forceinline__ void scalar_loads_done() { __builtin_amdgcn_s_waitcnt(0xC07F); }      // lgkmcnt(0)

}  // namespace
}  // namespace cf
