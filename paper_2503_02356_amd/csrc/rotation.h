// Rotation by positions, as the kernels of rotate.hip and kv_append8.hip make it.
//
// A lane has a unit of a row: 16 elements in two runs of 8, the 8 pairs of which it turns (or that are in no pair).  It takes the sines and
// cosines of its pairs once and turns its unit of several heads with them; since both elements of a pair are a lane's own, x may be y.
// The angle p * inv_freq / 2 pi is taken in 64 bits and its whole turns are dropped there: what is left has an error of 2^-25 of a turn
// (its rounding to fp32) for any position.  (In fp32 an angle of 2^18 radians would be off by 2^-6.)
#pragma once
#include <hip/hip_runtime.h>

#include "pages.h"
#include "scalar_rows.h"

namespace cf {

// Largest g with cu[g] <= row, for a row below cu[n]; `first`: the first row of the wavefront, the same in all its lanes, which all look on: 64
// bounds at a time.  Their own sequence is that one, one of the next, or lies behind a run of empty ones: looked for at twice the distance
// each time.
__device__ __forceinline__ int sequence_of(const int32_t *cu, int n, int first, int row)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, g = lo + lane * step;
        const unsigned long long before = __ballot(g < hi && cu[min(g, hi - 1)] <= first);
        lo += (63 - __clzll((long long)before)) * step;      // (lane 0 always says yes)
        hi = min(hi, lo + step);
    }
    int far = 1;
    while (far < n - lo && cu[lo + far] <= row) far *= 2;
    const int near = lo + far / 2;
    return near + find_segment(cu + near, min(far, n - lo) - far / 2, row);
}

__device__ __forceinline__ void load8(const unsigned short *p, float (&x)[8])
{
    const uint4 w = *(const uint4 *)p;
    const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
}
__device__ __forceinline__ void load8(const float *p, float (&x)[8])
{
    const float4 a = ((const float4 *)p)[0], b = ((const float4 *)p)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void store8(unsigned short *p, const float (&x)[8])
{
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    bf16x8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (__bf16)x[i];
    *(bf16x8 *)p = w;
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8])
{
    ((float4 *)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    ((float4 *)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Unit u of a row: elements at[0] .. + 7 and at[1] .. + 7, its pairs 8 u .. 8 u + 7 where it is turned.
struct Unit {
    int at[2];
    bool turned;
    __device__ __forceinline__ Unit(int u, int rot, bool interleaved) : turned(16 * u < rot)
    {
        const bool halves = turned && !interleaved;
        at[0] = halves ? 8 * u : 16 * u;
        at[1] = halves ? rot / 2 + 8 * u : 16 * u + 8;
    }
};

struct Turn {
    float c[8], s[8];
    // position >= 0; back: the other way round
    __device__ __forceinline__ void set(const float *inv_freq, int position, bool back)
    {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = inv_freq[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double turns = (double)f[i] * (double)position * 0.15915494309189533577;
            sincospif((float)(2.0 * (turns - rint(turns))), &s[i], &c[i]);
            if (back) s[i] = -s[i];
        }
    }
    __device__ __forceinline__ void pair(float &a, float &b, int i) const
    {
        const float x = a, y = b;
        a = x * c[i] - y * s[i];
        b = x * s[i] + y * c[i];
    }
    template <bool INTERLEAVED>
    __device__ __forceinline__ void apply(float (&a)[8], float (&b)[8]) const
    {
        if constexpr (INTERLEAVED) {
#pragma unroll
            for (int i = 0; i < 4; ++i) pair(a[2 * i], a[2 * i + 1], i), pair(b[2 * i], b[2 * i + 1], 4 + i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) pair(a[i], b[i], i);
        }
    }
};

// A tensor that is gone through head by head: x [rows][heads][D] to y, of rows or of places in the pages.
struct TurnTensor {
    const void *x;
    void *y;
    int64_t x_tok, x_head, y_tok, y_head;
    int n_heads, in_fp32, out_fp32;
    int turned, paged;           // (values of a cache are not turned)
    int groups;                  // of n heads each, a block of the grid's y to each
    __host__ void group(int per_group) { groups = (n_heads + per_group - 1) / per_group; }
};

// This lane's unit of heads [h0, h1) of row `row` of t, with a loop over `AT_ONCE` heads in flight.
template <typename In, typename Out, bool INTERLEAVED>
__device__ __forceinline__ void turn_heads(const TurnTensor &t, const Turn &turn, const Unit &unit, int64_t row, int64_t y_at, int h0, int h1)
{
    constexpr int AT_ONCE = 4;
    const In *x = (const In *)t.x + row * t.x_tok;
    Out *y = (Out *)t.y + y_at;
    if (!(t.turned && unit.turned) && t.x == t.y) return;        // in place
    for (int h = h0; h < h1; h += AT_ONCE) {
        float a[AT_ONCE][8], b[AT_ONCE][8];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const In *at = x + (int64_t)min(h + i, h1 - 1) * t.x_head;
            load8(at + unit.at[0], a[i]);
            load8(at + unit.at[1], b[i]);
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            if (h + i >= h1) break;
            if (t.turned && unit.turned) turn.apply<INTERLEAVED>(a[i], b[i]);
            Out *at = y + (int64_t)(h + i) * t.y_head;
            store8(at + unit.at[0], a[i]);
            store8(at + unit.at[1], b[i]);
        }
    }
}
template <bool INTERLEAVED>
__device__ __forceinline__ void turn_heads(const TurnTensor &t, const Turn &turn, const Unit &unit, int64_t row, int64_t y_at, int h0, int h1)
{
    if (!t.in_fp32) turn_heads<unsigned short, unsigned short, INTERLEAVED>(t, turn, unit, row, y_at, h0, h1);
    else if (!t.out_fp32) turn_heads<float, unsigned short, INTERLEAVED>(t, turn, unit, row, y_at, h0, h1);
    else turn_heads<float, float, INTERLEAVED>(t, turn, unit, row, y_at, h0, h1);
}

}  // namespace cf
