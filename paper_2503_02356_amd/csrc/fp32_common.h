// Building blocks of the fp32 matrix kernels (v_mfma_f32_16x16x4_f32): 16 owned rows to a workgroup of 16 wavefronts, which take every 16th
// block of 16 rows of the other side.  Layouts: attn_fp32.hip.
#pragma once
#include <hip/hip_runtime.h>

#include "mfma_common.h"
#include "scalar_rows.h"

namespace cf {
namespace {

constexpr int NW = 16;           // wavefronts per workgroup
constexpr int RB = 16;           // rows per block
constexpr int kExactDeltaKeys = 64;      // rows that see at most so many keys: dQ takes delta from P and dP (as the scalar kernels do)
constexpr float kNoRow = 1e30f;  // LSE of a row past the end: P = 0 (finite, so that probability() takes no difference of infinities)
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

template <int D>
struct Shape {
    static constexpr int J = D / 16;         // float4 pieces of a row that a lane holds (quarter rows)
    static constexpr int NC = D / 64;        // 64-wide column groups of a result
    static constexpr int OS = D + 4;         // row stride of a partial result in LDS (spreads float4 rows over the banks)
    static constexpr int PART = RB * OS;     // floats of one wavefront's partial result
    static constexpr int OPERAND = RB * D * 4;   // bytes of 16 staged rows
    static constexpr int OPERANDS = 2 * OPERAND + RB * 4;    // what the backward stages: two operands, delta
    static constexpr bool BOTH_MEET = D == 64;   // LDS holds the partial results of dK and dV at once
};
template <int D>
using Acc = f32x4[D / 16];                   // [4 * c + e], register i: column 64 c + 4 * (4 * quarter + i) + e

// The lane, as a value that the compiler does not know to be the same for every item: what follows from it is formed where it is used.
template <int USE>
__device__ __forceinline__ int lane_again(int lane, int item)
{
    int x;
    asm("; lane %c3" : "=v"(x) : "0"(lane), "s"(item), "n"(USE));
    return x;
}

// Combines over the 16 lanes of a quarter (rotations inside a row of 16 lanes).
template <int N>
__device__ __forceinline__ float add_rotated(float x)
{
    return x + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x120 + N, 0xf, 0xf, false));
}
__device__ __forceinline__ float sum_over_16_lanes(float x) { return add_rotated<1>(add_rotated<2>(add_rotated<4>(add_rotated<8>(x)))); }

// This lane's quarter of a row: floats 16 j + 4 * quarter + 0..3.
template <int D>
__device__ __forceinline__ void load_row(const float *row, int quarter, f32x4 (&f)[D / 16])
{
#pragma unroll
    for (int j = 0; j < D / 16; ++j) f[j] = *(const f32x4 *)(row + 16 * j + 4 * quarter);
}
// The 16 owned rows into LDS, in operand order: piece c (floats 4 c .. 4 c + 3) of row r at [c * 16 + r].
template <int D, bool ANEW = false>
__device__ __forceinline__ void stage_rows(const float *base, int64_t stride, int row0, int last_row, f32x4 *dst)
{
    for (int t = ANEW ? wave_id() * 64 + fresh_lane() : threadIdx.x; t < RB * D / 4; t += NW * 64) {
        const int r = t / (D / 4), c = t % (D / 4);
        dst[c * RB + r] = *(const f32x4 *)(base + (int64_t)min(row0 + r, last_row) * stride + c * 4);
    }
}
// rows (A operand, from registers) x owned rows (B operand, from LDS), contraction over d.
template <int D>
__device__ __forceinline__ f32x4 row_product(const f32x4 (&a)[D / 16], const f32x4 *b, int lane)
{
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
        const f32x4 bj = b[j * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = mfma_f32(a[j][e], bj[e], acc);
    }
    return acc;
}
// Column operands of a 16-row block: whole rows per 16 lanes, step i of the contraction over the rows takes rows
// 4 * quarter + i, which is where register i of the other operand stands; lane % 16 = m holds columns 64 c + 4 m + e.
// Rows past last_row (relative to the block's first row, `block`) re-read last_row; the other operand is 0 there.
// (A scalar base that is known to be global memory and a 32-bit lane offset: a flat load would also wait for LDS.)
template <int D>
__device__ __forceinline__ void load_columns(const float *block, unsigned row_bytes, int last_row, int lane, f32x4 (&x)[4][D / 64])
{
    const int quarter = lane >> 4, m = lane & 15;
    const CF_GLOBAL char *base = (const CF_GLOBAL char *)uniform(block);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
            x[i][c] = *(const CF_GLOBAL f32x4 *)(base + ((unsigned)min(4 * quarter + i, last_row) * row_bytes + 16 * m + 256 * c));
}
// The same columns of rows that this wavefront already holds (load_row), turned around through its own piece of LDS.  In two
// parts: the rows may leave their registers in between.
__device__ __forceinline__ void lds_turn() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"), __builtin_amdgcn_wave_barrier(); }
template <int D>
__device__ __forceinline__ void put_rows(const f32x4 (&f)[D / 16], float *piece, int lane)
{
    lds_turn();                                      // (what stood there has been read)
#pragma unroll
    for (int j = 0; j < D / 16; ++j) *(f32x4 *)(piece + (lane & 15) * Shape<D>::OS + 16 * j + 4 * (lane >> 4)) = f[j];
    lds_turn();
}
// acc^T += X^T w
template <int D>
__device__ __forceinline__ void add_column_product(const f32x4 (&x)[4][D / 64], const f32x4 &w, Acc<D> &acc)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[4 * c + e] = mfma_f32(x[i][c][e], w[i], acc[4 * c + e]);
}
// acc^T += X^T w, X the rows that stand in this wavefront's piece of LDS
template <int D>
__device__ __forceinline__ void add_column_product(const float *piece, int lane, const f32x4 &w, Acc<D> &acc)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (D != 64) __builtin_amdgcn_sched_barrier(0);  // (all of X at once: 34 registers spilled)
        f32x4 x[D / 64];
#pragma unroll
        for (int c = 0; c < D / 64; ++c) x[c] = *(const f32x4 *)(piece + (4 * (lane >> 4) + i) * Shape<D>::OS + 4 * (lane & 15) + 64 * c);
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[4 * c + e] = mfma_f32(x[c][e], w[i], acc[4 * c + e]);
    }
}
// A wavefront's transposed result (lane % 16 = owned row) into its part of the LDS scratch.
template <int D>
__device__ __forceinline__ void write_part(const Acc<D> &acc, float *part, int lane)
{
    const int quarter = lane >> 4, r = lane & 15;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *(f32x4 *)(part + r * Shape<D>::OS + 64 * c + 16 * quarter + 4 * i) =
                f32x4{acc[4 * c][i], acc[4 * c + 1][i], acc[4 * c + 2][i], acc[4 * c + 3][i]};
}
template <int D>
__device__ __forceinline__ f32x4 sum_parts(const float *parts, int n, int row, int c)
{
    f32x4 s = *(const f32x4 *)(parts + row * Shape<D>::OS + c * 4);
    for (int w = 1; w < n; ++w) s += *(const f32x4 *)(parts + w * Shape<D>::PART + row * Shape<D>::OS + c * 4);
    return s;
}

// The last step of every kernel gives D / 4 consecutive lanes of a wavefront one row: visit(first lane of the row), by the whole
// wavefront, for every row that one of `lanes` has a part of.  (Rows whose result is not finite: see scalar_rows.h.)
template <int D>
__device__ __forceinline__ unsigned long long lanes_of_row(int lane) { return ((1ull << (D / 4)) - 1) << (lane / (D / 4) * (D / 4)); }
template <int D, typename Visit>
__device__ __forceinline__ void for_rows_of(unsigned long long lanes, Visit visit)
{
    static_assert(RB * (D / 4) <= NW * 64, "one step");
    while (lanes != 0) {
        const int first = __ffsll((long long)lanes) - 1;
        lanes &= ~lanes_of_row<D>(first);
        visit(first / (D / 4) * (D / 4));
    }
}
__device__ __forceinline__ bool finite(const f32x4 &x) { return cf::finite((x[0] + x[1]) + (x[2] + x[3])); }

}  // namespace
}  // namespace cf
