// fp32 attention of new tokens over a paged cache, head_dim 64 and 128, any scale: the fp32 forward kernel of a chunk (attn_fp32.hip) over
// tiles of 16 token-head rows (row r of a sequence: token r / G, head r % G).  A workgroup of 8 wavefronts takes a tile and a part of its
// keys, its wavefronts every 8th block of 16 keys, straight from the pages into registers (a block lies in one page); their results meet in
// LDS in a fixed order, parts in a kernel behind this one.  A block of no page is passed over.
// Bound by the fp32 matrix rate where there are many rows (a prompt of 2000, 6/2 heads, D = 128: 76 us, 82 TFLOP/s), by the chain of a wavefront's
// blocks and the loads' latency where there are few (3 tokens and 2 chunks of 100 behind up to 700 keys: 13 us).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "fp32_common.h"
#include "paged_tiles.h"

namespace cf {
namespace {

// Wavefronts of a workgroup.  8: two workgroups to a compute unit, one multiplies while the other loads (append and attention, 6/2 heads, D = 128,
// us, 16 / 8 / 4 wavefronts: 3 tokens and 2 chunks of 100 behind up to 700 keys 27.9 / 18.7 / 21.0, 64 tokens behind 4000 134 / 103 / 118, a prompt of 2000
// 83.6 / 76.3 / 103).
constexpr int W = 8;
template <int D>
__global__ __launch_bounds__(W * 64, 4) void f32_paged_kernel(PagedArgs a)
{
    using S = Shape<D>;
    __shared__ f32x4 qs[S::J * 64];
    __shared__ __attribute__((aligned(16))) float parts[W * S::PART];
    __shared__ float m_s[W][RB], l_s[W][RB];
    const int lane = threadIdx.x & 63, wave = wave_id(), quarter = lane >> 4, col = lane & 15;
    TileRows t;
    t.G = a.p.n_q_heads / a.p.n_kv_heads;
    int id = blockIdx.x;
    t.kh = id % a.p.n_kv_heads;
    id /= a.p.n_kv_heads;
    const int part = id % a.parts;
    if (!find_tile<RB>(a, id / a.parts, t)) return;
    const int lowest = t.position(0), highest = t.position(t.rows - 1);
    const int keys = keys_within(highest, a.p.pages_per_seq, a.shift);
    const KeyTiles<RB, WindowMask> blocks(a.mask, lowest, keys);
    const int n = at_least(0, blocks.n), first = at_most(n, a.parts > 1 ? part * a.tiles_per_part : 0);
    const int end = a.parts > 1 && part + 1 < a.parts ? at_most(n, first + a.tiles_per_part) : n;
    const int64_t all = (int64_t)a.p.n_tokens * a.p.n_q_heads;
    if (first >= end && a.parts > 1) {               // no keys: what is left of the rows
        if (threadIdx.x < t.rows) a.part_ml[t.flat(a, threadIdx.x) * a.parts + part] = make_float2(-INFINITY, 0.f);
        return;
    }
    for (int i = threadIdx.x; i < RB * D / 4; i += W * 64) {
        const int r = i / (D / 4), c = i % (D / 4);
        int64_t row;
        int h;
        t.find(at_most(r, t.rows - 1), row, h);
        qs[c * RB + r] = *(const f32x4 *)((const float *)a.p.q + row * a.p.q_stride_tok + (int64_t)h * a.p.q_stride_head + c * 4);
    }
    __syncthreads();

    const KeySource<4> src(a, t, keys);
    const float c2 = a.p.softmax_scale * kLog2e;
    const int position = t.position(at_most(col, t.rows - 1));
    Acc<D> o;
#pragma unroll
    for (int x = 0; x < D / 16; ++x) o[x] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    for (int b = first + wave; b < end; b += W) {
        const int k0 = blocks.start(b), page = src.page_of(k0);
        if (page < 0) continue;
        const int64_t at = src.offset(page, k0);
        const int last = at_most(RB - 1, src.room(k0));
        f32x4 kf[S::J], x[4][S::NC];
        load_row<D>((const float *)(src.k + at + (int64_t)at_most(col, last) * src.row_bytes), quarter, kf);
        if (D == 64) load_columns<D>((const float *)(src.v + at), src.row_bytes, last, lane, x);
        f32x4 s = row_product<D>(kf, qs, lane);
        if (D != 64) {
            __builtin_amdgcn_sched_barrier(0);       // (V takes the registers of K)
            load_columns<D>((const float *)(src.v + at), src.row_bytes, last, lane, x);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = k0 + 4 * quarter + i;
            const bool between = (unsigned)(key - a.mask.sinks) < hidden_keys(a.mask, position);
            s[i] = key > position ? -INFINITY : s[i] * c2;
            if (between) s[i] = -INFINITY;
        }
        const float m_new = fmaxf(m, max_over_quarters(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))));
        const float ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m - ref);
        m = m_new;
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] - ref);
        l = l * alpha + ((s[0] + s[1]) + (s[2] + s[3]));
#pragma unroll
        for (int x = 0; x < D / 16; ++x) o[x] *= alpha;
        add_column_product<D>(x, s, o);
    }
    l = sum_over_quarters(l);
    if (quarter == 0) {
        m_s[wave][col] = m;
        l_s[wave][col] = l;
    }
    const int used = at_most(W, end - first);       // wavefronts that had a block
    if (wave < used) write_part<D>(o, parts + wave * S::PART, lane);
    __syncthreads();

    const PagedArgs &e = arguments();
    const int r = threadIdx.x / (D / 4), c = threadIdx.x % (D / 4);
    bool bad = false;
    if (r < t.rows) {
        float M = -INFINITY, L = 0.f;
        for (int w = 0; w < used; ++w) M = fmaxf(M, m_s[w][r]);
        const float ref = M == -INFINITY ? 0.f : M;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < used; ++w) {
            const float g = __builtin_amdgcn_exp2f(m_s[w][r] - ref);
            L += g * l_s[w][r];
            sum += g * *(const f32x4 *)(parts + w * S::PART + r * S::OS + c * 4);
        }
        bad = !finite(sum) || !(L < INFINITY);
        if (e.parts > 1) {
            const int64_t flat = t.flat(e, r);
            *(f32x4 *)(e.part_o + (part * all + flat) * D + c * 4) = sum;
            if (c == 0) e.part_ml[flat * e.parts + part] = make_float2(M, L);
        } else {
            *(f32x4 *)(t.out(e, r) + c * 16) = sum * (L == 0.f ? 0.f : 1.f / L);
            if (c == 0) t.put_lse(e, r, L == 0.f ? -INFINITY : M * kLn2 + logf(L));
        }
    }
    for_rows_of<D>(__ballot(bad), [&](int at) {
        const int x = (wave * 64 + at) / (D / 4);
        int64_t row;
        int h;
        t.find(x, row, h);
        const float *q = row_of<float>(e.p.q, (int)row, e.p.q_stride_tok, h, e.p.q_stride_head);
        const RowSums<float, D> sums = paged_row<float, D, 4, RB>(e, e.table(t.seq), t.position(x), t.kh, blocks, first, end, [&](int i) { return q[i]; });
        const bool none = sums.m == -INFINITY && sums.z == 0.f;
        if (e.parts > 1) {
            const int64_t flat = t.flat(e, x);
            for (int i = 0; i < D / 64; ++i) e.part_o[(part * all + flat) * D + lane + 64 * i] = sums.acc[i];
            if (lane == 0) e.part_ml[flat * e.parts + part] = make_float2(sums.m * kLog2e, sums.z);
        } else {
            for (int i = 0; i < D / 64; ++i) ((float *)t.out(e, x))[lane + 64 * i] = none ? 0.f : sums.acc[i] / sums.z;
            if (lane == 0) t.put_lse(e, x, none ? -INFINITY : sums.m + logf(sums.z));
        }
    });
}

int64_t groups_most(const cf_attn_paged_params &p) { return places_most(p.n_tokens, p.n_seqs, p.n_q_heads / p.n_kv_heads, RB) * p.n_kv_heads; }

}  // namespace

int64_t paged_f32_launch_size(const PagedArgs &a) { return groups_most(a.p) * a.parts * W * 64; }

// Parts of at least one block for each wavefront, so many that there is a workgroup for each of the chip's 512 places (for 256 / 512 / 1024
// workgroups: the case above 22.4 / 18.9 / 18.9 us, 64 tokens behind 4000 keys 132 / 102 / 109).
void cut_paged_f32(PagedArgs &a)
{
    const cf_attn_paged_params &p = a.p;
    const int64_t capacity = (int64_t)p.pages_per_seq * p.page_size;
    int64_t blocks = ((p.max_kv_len > 0 ? std::min<int64_t>(p.max_kv_len, capacity) : capacity) + RB - 1) / RB;
    if (p.window > 0) blocks = std::min(blocks, ((int64_t)p.window + RB) / RB + 2 + ((int64_t)a.mask.sinks + RB - 1) / RB);
    const int64_t groups = groups_most(p), parts = std::min<int64_t>({(512 + groups - 1) / groups, (blocks + W - 1) / W, kMostParts});
    a.parts = (int)std::max<int64_t>(1, parts);
    a.tiles_per_part = (int)((blocks + a.parts - 1) / a.parts);
}

hipError_t launch_paged_f32(const PagedArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)(groups_most(a.p) * a.parts));
    if (a.p.head_dim == 64) f32_paged_kernel<64><<<grid, W * 64, 0, s>>>(a);
    else f32_paged_kernel<128><<<grid, W * 64, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cf
