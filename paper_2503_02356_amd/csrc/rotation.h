// Rotation by positions, as the kernels of rotate.hip and kv_append8.hip make it.
//
// A lane has a unit of a row: 16 elements in two runs of 8, the 8 pairs of which it turns (or that are in no pair).  It takes the sines and
// cosines of its pairs once and turns its unit of several heads with them; since both elements of a pair are a lane's own, x may be y.
// The angle p * inv_freq loses its whole turns in twice 64 bits (angle.h): what is left has an error of 2^-25 of a turn (its rounding to
// fp32) for any position.  (In fp32 an angle of 2^18 radians would be off by 2^-6.)
// Bound by memory, one read and one write of every element, where a call is large; by its launch and one trip to memory where it is small.
#pragma once
#include <hip/hip_runtime.h>

#include "angle.h"
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

// Eight elements as they come from memory.
template <typename T>
struct Eight {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = ((const uint4 *)p)[i];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        const unsigned u[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 2) {
                x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
            } else {
                const unsigned v[4] = {w[1].x, w[1].y, w[1].z, w[1].w};
                x[i] = __uint_as_float(u[i]), x[4 + i] = __uint_as_float(v[i]);
            }
        }
    }
};

// STREAM: past the caches (results of a large call, which would only push its inputs out; figures at TurnArgs::group).
template <bool STREAM, typename V>
__device__ __forceinline__ void put(V *p, V w)
{
    if constexpr (STREAM) __builtin_nontemporal_store(w, p);
    else *p = w;
}
template <bool STREAM>
__device__ __forceinline__ void store8(unsigned short *p, const float (&x)[8])
{
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    bf16x8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (__bf16)x[i];
    put<STREAM>((bf16x8 *)p, w);
}
template <bool STREAM>
__device__ __forceinline__ void store8(float *p, const float (&x)[8])
{
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    put<STREAM>((f32x4 *)p, f32x4{x[0], x[1], x[2], x[3]});
    put<STREAM>((f32x4 *)p + 1, f32x4{x[4], x[5], x[6], x[7]});
}

// Unit u of a row: elements at[0] .. + 7 and at[1] .. + 7.  Pairs next to each other: a run in each half of the row, so that a wavefront's loads and stores
// take whole halves of rows.  Pairs of two halves: a run in each half of the part that is turned, or of the rest.
struct Unit {
    int at[2], first[2];         // first: the pairs that its first and last four are the beginning of
    bool turned[2];
    __device__ __forceinline__ Unit(int u, int D, int rot, bool interleaved)
    {
        const bool front = interleaved || 16 * u < rot;
        const int start = front ? 0 : rot, size = interleaved ? D : front ? rot : D - rot;
        at[0] = start + 8 * u - start / 2, at[1] = at[0] + size / 2;
        first[0] = interleaved ? at[0] / 2 : 8 * u, first[1] = interleaved ? at[1] / 2 : 8 * u + 4;
        turned[0] = at[0] < rot, turned[1] = interleaved ? at[1] < rot : turned[0];
    }
    __device__ __forceinline__ bool any() const { return turned[0] || turned[1]; }
};

struct Turn {
    float c[8], s[8];
    // position >= 0; back: the other way round
    __device__ __forceinline__ void set(const float *inv_freq, const Unit &unit, int position, bool back)
    {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = unit.turned[i / 4] ? inv_freq[unit.first[i / 4] + i % 4] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sincospif(half_turns(f[i], position), &s[i], &c[i]);
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
    __device__ __forceinline__ void apply(const Unit &unit, float (&a)[8], float (&b)[8]) const
    {
        if constexpr (INTERLEAVED) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (unit.turned[0]) pair(a[2 * i], a[2 * i + 1], i);
                if (unit.turned[1]) pair(b[2 * i], b[2 * i + 1], 4 + i);
            }
        } else if (unit.turned[0]) {
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

// This lane's unit of heads [h0, h1) of row `row` of t, AT_ONCE of them in flight, the first ones before `place` finds out where the results go (or that they go
// nowhere: -1) and `angles` what they are turned by.
template <typename In, typename Out, bool INTERLEAVED, bool STREAM, typename Place, typename Angles>
__device__ __forceinline__ void turn_heads(const TurnTensor &t, const Unit &unit, int64_t row, int h0, int h1, Place place, Angles angles)
{
    constexpr int AT_ONCE = 4;                       // (us, 2 / 4 / 8: 32768 rows of 64 + 8 heads there and back 530 / 527 / 531, 8192 of 28 + 4 60.5 / 58.1 / 60.8; one token into pages 5.3 each)
    const In *x = (const In *)t.x + row * t.x_tok;
    const bool turned = t.turned && unit.any();
    if (!turned && t.x == t.y) return;               // in place
    Eight<In> a[AT_ONCE], b[AT_ONCE];
    auto load = [&](int h) {
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const In *at = x + (int64_t)min(h + i, h1 - 1) * t.x_head;
            a[i].load(at + unit.at[0]);
            b[i].load(at + unit.at[1]);
        }
    };
    load(h0);
    const int64_t y_at = place();
    if (y_at < 0) return;
    Out *y = (Out *)t.y + y_at;
    Turn turn;
    if (turned) angles(turn);
    for (int h = h0;;) {
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            if (h + i >= h1) break;
            float p[8], q[8];
            a[i].get(p), b[i].get(q);
            if (t.turned) turn.apply<INTERLEAVED>(unit, p, q);
            Out *at = y + (int64_t)(h + i) * t.y_head;
            store8<STREAM>(at + unit.at[0], p);
            store8<STREAM>(at + unit.at[1], q);
        }
        h += AT_ONCE;
        if (h >= h1) return;
        load(h);
    }
}
template <bool INTERLEAVED, bool STREAM, typename Place, typename Angles>
__device__ __forceinline__ void turn_heads(const TurnTensor &t, const Unit &unit, int64_t row, int h0, int h1, Place place, Angles angles)
{
    if (!t.in_fp32) turn_heads<unsigned short, unsigned short, INTERLEAVED, STREAM>(t, unit, row, h0, h1, place, angles);
    else if (!t.out_fp32) turn_heads<float, unsigned short, INTERLEAVED, STREAM>(t, unit, row, h0, h1, place, angles);
    else turn_heads<float, float, INTERLEAVED, STREAM>(t, unit, row, h0, h1, place, angles);
}

}  // namespace cf
