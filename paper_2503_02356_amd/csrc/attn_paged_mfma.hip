// bf16 attention of new tokens over a paged cache, head_dim 64 and 128.
//
// The rows of a sequence and a key/value head are its new tokens times the G query heads of the group, row r being token r / G, head r % G:
// they all multiply with the same keys and values.  A tile is 128 of them.  A workgroup (4 wavefronts, 16x16x32 MFMAs, everything
// transposed as in attn_mfma_fwd.hip: S^T = K Q^T, O^T += V^T P^T, the row on the lane axis) takes a tile and a part of its keys:
//   many rows  (more than 32)  a wavefront has 32 rows; key tiles of 64 are shared through LDS, double buffered.  Bound by the MFMAs and
//              the arithmetic between them, like the forward kernel of a chunk.
//   few rows   every wavefront has all of them and takes every fourth block of 32 keys, copied into its own part of LDS: it waits for
//              nobody.  Bound by the memory that holds the cache: 16 KB of keys and values a wavefront, 8 wavefronts a compute unit, are in
//              flight or in use.  The four results meet in LDS at the end.
// A long cache with few tiles is cut into parts, joined by a kernel behind this one (attn_paged.hip).
// Pages: 16 consecutive keys lie in one page (a page holds a multiple of 16), so that each copy instruction (512 / D rows of a tile) has one
// base, found with scalar instructions from a table entry that was loaded a tile ahead.  Keys that are hidden as a whole group (no such page,
// or behind the last key) are copied from a row of zeros, never from the pages, and masked.
// P enters the second product as bf16 (half a step, 2^-8 of the value, as o itself is rounded; its sum is taken before that).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mfma_common.h"
#include "paged.h"

namespace cf {
namespace {

constexpr int BM = 128, BN = 64;             // rows of a tile, keys of a key tile
constexpr int FEW = 32;                      // rows that the wavefronts share, keys of their blocks
using F = Mfma<16>;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLazy = 8.f;                 // log2 units a row maximum may exceed the running reference (attn_mfma_fwd.hip)

__device__ __align__(16) unsigned zeros[64];                 // a row of zeros

// A part of a tile, as its workgroup finds it.
struct TileRows {
    int seq, q0;                 // sequence, its first row of q
    int row0, rows;              // first row of the tile among the sequence's token-head rows, and how many it has
    int first_position;
};

// Tile `rank`, counted from the last one of the last sequence: sequence g has the ranks from cu[g] * G / 128 + g on.
__device__ __forceinline__ bool find_tile(const PagedArgs &a, int G, int rank, TileRows &t)
{
    const cf_attn_paged_params &p = a.p;
    const int32_t *cu = p.cu_seqlens_q;
    const int lane = threadIdx.x & 63;
    const int place = (int)((int64_t)p.n_tokens * G / BM) + p.n_seqs - 1 - rank;
    int lo = 0, hi = p.n_seqs;
    while (hi - lo > 64) {
        const int step = (hi - lo + 63) / 64, g = lo + lane * step;
        const unsigned long long before = __ballot(g < hi && cu[min(g, hi - 1)] * G / BM + g <= place);
        lo += (63 - __clzll((long long)before)) * step;      // (lane 0 always says yes)
        hi = min(hi, lo + step);
    }
    const int g = min(lo + lane, hi - 1);
    const int begin = cu[g], end = cu[g + 1], keys = p.kv_lens[g];
    const int last = 63 - __clzll((long long)__ballot(lo + lane < hi && begin * G / BM + g <= place));
    t.seq = uniform(lo + last);
    const int q0 = __builtin_amdgcn_readlane(begin, last), q1 = __builtin_amdgcn_readlane(end, last);
    const NewRows rows(q0, q1, __builtin_amdgcn_readlane(keys, last));
    t.q0 = q0;
    t.row0 = (place - q0 * G / BM - t.seq) * BM;
    t.rows = at_most(BM, rows.lq * G - t.row0);
    t.first_position = rows.first_position;
    return t.rows > 0;
}

// Copies ROWS keys of a head, from key `start` (a multiple of 16) on, into a swizzled LDS tile, by WAVES wavefronts: groups of 16 keys, each
// in one page.  pages[g]: the page of group g, -1: none.  last: the last key that may be read.
template <int ROWS, int D, int WAVES>
struct PagedDma {
    static constexpr int RPI = 512 / D, UNITS = D / 8, PARTS = ROWS / (RPI * WAVES), GROUPS = ROWS / 16;
    int wv, r;                   // this wavefront among those that copy; this lane's row of an instruction
    unsigned unit16[(RPI * WAVES) % 16 == 0 ? 1 : 16 / (RPI * WAVES)];
    unsigned row_bytes;
    static constexpr int KINDS = (RPI * WAVES) % 16 == 0 ? 1 : 16 / (RPI * WAVES);

    __device__ __forceinline__ void init(int64_t row_bytes_, int wave)
    {
        const int lane = threadIdx.x & 63;
        wv = wave;
        r = lane / UNITS;
        row_bytes = (unsigned)row_bytes_;
#pragma unroll
        for (int i = 0; i < KINDS; ++i) unit16[i] = ((lane % UNITS) ^ swz<D>(RPI * (WAVES * i + wv) + r)) * 16;
    }
    // base(page, row in group's page): address of a key's row
    template <typename Base>
    __device__ __forceinline__ void issue(int start, int last, const int (&pages)[GROUPS], char *tile, Base base) const
    {
#pragma unroll
        for (int c = 0; c < PARTS; ++c) {
            const int first = RPI * (WAVES * c + wv);        // of the instruction's rows in the tile (wave-uniform)
            int page;
            if constexpr (RPI * WAVES <= 16) {
                page = pages[RPI * WAVES * c / 16];
            } else {                                          // (64-wide heads, four wavefronts: two groups to a step)
                page = wv < 2 ? pages[RPI * WAVES * c / 16] : pages[RPI * WAVES * c / 16 + 1];
            }
            const int key = start + first, room = last - key;            // rows of the instruction up to the last key: room + 1
            const bool some = page >= 0 && room >= 0;
            const char *src = some ? base(page, key) : (const char *)zeros;
            unsigned off = (unsigned)min(r, room) * row_bytes;
            off = some ? off : 0;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(TileDma<64, D>::descriptor(uniform(src)), (CF_LDS void *)(tile + (c * WAVES + wv) * 1024), 16,
                                                     (int)(off + unit16[c % KINDS]), 0, 0, 0);
        }
    }
};

// What both bodies need of a call.
template <int D>
struct Setup {
    const PagedArgs &a;
    const TileRows &t;
    PageTable table;
    int G, kh;
    int64_t key_row_bytes, page_bytes;
    const char *k, *v;
    float c2;
    unsigned flip;               // sign of the scale, on two bf16
    bool zero;                   // scale 0: every score is 0
    __device__ __forceinline__ Setup(const PagedArgs &a_, const TileRows &t_, int G_, int kh_)
        : a(a_), t(t_), table(a_.table(t_.seq)), G(G_), kh(kh_), key_row_bytes(a_.p.kv_stride_tok * 2), page_bytes(a_.p.page_stride * 2),
          k((const char *)a_.p.k_pages + (int64_t)kh_ * a_.p.kv_stride_head * 2), v((const char *)a_.p.v_pages + (int64_t)kh_ * a_.p.kv_stride_head * 2)
    {
        zero = a.p.softmax_scale == 0.f;
        flip = a.p.softmax_scale < 0.f ? 0x80008000u : 0u;
        c2 = zero ? 1.f : fabsf(a.p.softmax_scale) * kLog2e;
    }
    // token-head row x of the tile: its token of q, head, position
    __device__ __forceinline__ int token(int x) const { return (t.row0 + x) / G; }
    __device__ __forceinline__ int position(int x) const { return at_least(-1, t.first_position + token(x)); }
    __device__ __forceinline__ int64_t flat(int x) const
    {
        const int i = token(x);
        return (int64_t)(t.q0 + i) * a.p.n_q_heads + kh * G + (t.row0 + x - i * G);
    }
    __device__ __forceinline__ bf16x8 query(int x, int d) const
    {
        const int i = token(x), h = kh * G + (t.row0 + x - i * G);
        i32x4 w = *(const i32x4 *)((const char *)a.p.q + ((int64_t)(t.q0 + i) * a.p.q_stride_tok + (int64_t)h * a.p.q_stride_head + d) * 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = zero ? 0 : w[e] ^ (int)flip;
        return __builtin_bit_cast(bf16x8, w);
    }
    __device__ __forceinline__ char *out(int x) const
    {
        const int i = token(x), h = kh * G + (t.row0 + x - i * G);
        return (char *)a.p.o + ((int64_t)(t.q0 + i) * a.p.o_stride_tok + (int64_t)h * a.p.o_stride_head) * 2;
    }
    __device__ __forceinline__ float *lse(int x) const
    {
        const int i = token(x), h = kh * G + (t.row0 + x - i * G);
        return a.p.lse + (int64_t)h * a.p.n_tokens + t.q0 + i;
    }
    __device__ __forceinline__ const char *key_row(const char *base, int page, int key) const
    {
        return base + (int64_t)page * page_bytes + (int64_t)table.row_in_page(key) * key_row_bytes;
    }
    // The pages of GROUPS groups of 16 keys from `start` on.
    template <int GROUPS>
    __device__ __forceinline__ void find_pages(int start, int last, int (&pages)[GROUPS]) const
    {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int page = table.row[min(start + 16 * g, last) >> table.shift];
            pages[g] = page >= 0 && page < table.n_pages && start + 16 * g <= last ? page : -1;
        }
    }
    // One row over the part's keys, pair by pair (a row whose result is not finite).
    template <typename Tiles>
    __device__ __forceinline__ RowSums<unsigned short, D> again(int x, const Tiles &tiles, int first, int end) const
    {
        const int i = token(x), h = kh * G + (t.row0 + x - i * G);
        const unsigned short *q = row_of<unsigned short>(a.p.q, t.q0 + i, a.p.q_stride_tok, h, a.p.q_stride_head);
        return paged_row<unsigned short, D, 4>(a, table, position(x), kh, tiles, first, end, [&](int e) { return ld(q + e); });
    }
    // Its result: into the call's tensors, or as a part.
    __device__ __forceinline__ void put_again(int x, const RowSums<unsigned short, D> &r, int part) const
    {
        const int lane = threadIdx.x & 63;
        const bool none = r.m == -INFINITY && r.z == 0.f;
        if (a.parts > 1) {
            float *o = a.part_o + ((int64_t)part * a.p.n_tokens * a.p.n_q_heads + flat(x)) * D;
            for (int e = 0; e < D / 64; ++e) o[lane + 64 * e] = r.acc[e];
            if (lane == 0) a.part_ml[flat(x) * a.parts + part] = make_float2(r.m * kLog2e, r.z);
        } else {
            unsigned short *o = (unsigned short *)out(x);
            for (int e = 0; e < D / 64; ++e) st(o + lane + 64 * e, none ? 0.f : r.acc[e] / r.z);
            if (lane == 0 && a.p.lse) *lse(x) = none ? -INFINITY : r.m + logf(r.z);
        }
    }
};

// One block of KB x 16 keys, for QB x 16 rows: scores of a K tile, masks, the running softmax, P.
template <int D, int KB, int QB>
struct Rows {
    static constexpr int KS = D / F::K, DB = D / 16, NS = KB * F::R;
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
    // lowest, highest: positions of the wavefront's rows.  groups: hidden groups of 16 keys, a bit each.
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
            const int sink = mask.sinks - start - group * 4;
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                const int far = pos[qb] - mask.window - start - group * 4;
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    if (F::place(i) <= far && F::place(i) >= sink) s[i / F::R][qb][i % F::R] = -INFINITY;
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
    __device__ __forceinline__ void values(const char *v_tile, const LaneOffsets<D, 16> &lo, const f32x4 (&s)[KB][QB])
    {
#pragma unroll
        for (int t = 0; t < KB * 16 / F::K; ++t) {
            bf16x8 pb[QB];
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = s[(8 * t + e) / F::R][qb][(8 * t + e) % F::R];
                pb[qb] = pack8(f);
            }
            const char *va = v_tile + t * (F::K * 2 * D);
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const bf16x8 x = lds_read_tr_pair(va + lo.tr_lo[db], va + lo.tr_hi(db));
#pragma unroll
                for (int y = 0; y < QB; ++y) {
                    const int qb = db & 1 ? QB - 1 - y : y;
                    o[db][qb] = F::mul(x, pb[qb], o[db][qb]);
                }
            }
        }
    }
};

// Many rows: 32 to a wavefront, key tiles shared.
template <int D>
__device__ __forceinline__ void many_rows(const Setup<D> &c, const KeyTiles<BN, WindowMask> &tiles, int first, int end, int last, int part, char *stage_a,
                                          char *stage_b)
{
    constexpr int TILE = BN * 2 * D;
    const PagedArgs &a = c.a;
    const int wave = wave_id(), col = F::column(), group = F::group();
    const int x0 = 32 * wave, rows = at_most(32, c.t.rows - x0);           // this wavefront's rows of the tile (rows <= 0: none)
    Rows<D, BN / 16, 2> r;
    r.clear();
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const int x = min(x0 + 16 * qb + col, c.t.rows - 1);
        r.pos[qb] = c.position(x);
#pragma unroll
        for (int ks = 0; ks < D / F::K; ++ks) r.q[qb][ks] = c.query(x, ks * F::K + group * 8);
    }
    const int lowest = c.position(at_most(x0, c.t.rows - 1)), highest = c.position(at_most(x0 + 31, c.t.rows - 1));
    const LaneOffsets<D, 16> lo = lane_offsets<D, 16>();
    PagedDma<BN, D, 4> dma;
    dma.init(c.key_row_bytes, wave);
    int pages[4];
    unsigned hidden = 0;
    auto issue = [&](int start, char *stage) {
        dma.issue(start, last, pages, stage, [&](int page, int key) { return c.key_row(c.k, page, key); });
        dma.issue(start, last, pages, stage + TILE, [&](int page, int key) { return c.key_row(c.v, page, key); });
        hidden = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) hidden |= (unsigned)(pages[g] < 0) << g;
    };
    c.find_pages(tiles.start(first), last, pages);
    issue(tiles.start(first), stage_a);
    if (first + 1 < end) c.find_pages(tiles.start(first + 1), last, pages);
    wait_lds_dma();
    __syncthreads();
    auto do_tile = [&](int t, const char *stage, char *next) {
        const int start = tiles.start(t);
        const unsigned hid = hidden;
        if (t + 1 < end) issue(tiles.start(t + 1), next);
        if (t + 2 < end) c.find_pages(tiles.start(t + 2), last, pages);
        if (rows > 0 && start <= highest && (start + BN > lowest + 1 - a.mask.window || start < a.mask.sinks)) {
            f32x4 s[BN / 16][2];
            r.scores(stage, lo, a.mask, start, lowest, highest, hid, c.c2, s);
            r.values(stage + TILE, lo, s);
        }
        wait_lds_dma();
        __syncthreads();
    };
    for (int t = first; t < end; t += 2) {
        do_tile(t, stage_a, stage_b);
        if (t + 1 < end) do_tile(t + 1, stage_b, stage_a);
    }
    if (rows <= 0) return;
    float l[2], scale[2];
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        l[qb] = sum_over_groups<16>(r.l[qb]);
        scale[qb] = l[qb] == 0.f ? 0.f : 1.f / l[qb];
    }
    if (a.parts > 1) {
        const int64_t all = (int64_t)a.p.n_tokens * a.p.n_q_heads;
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            const int x = 16 * qb + col;
            if (x >= rows) continue;
            const int64_t flat = c.flat(x0 + x);
            float *o = a.part_o + (part * all + flat) * D + 4 * group;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) *(f32x4 *)(o + 16 * db) = r.o[db][qb];
            if (group == 0) a.part_ml[flat * a.parts + part] = make_float2(r.m[qb], l[qb]);
        }
    } else {
        char *scratch = (wave < 2 ? stage_a : stage_b) + (wave & 1) * RowScratch<D>::bytes;
        store_rows_bf16<D, 16>(r.o, scale, scratch, rows, [&](int x) { return c.out(x0 + x); });
#pragma unroll
        for (int qb = 0; qb < 2; ++qb)
            if (group == 0 && 16 * qb + col < rows && a.p.lse)
                *c.lse(x0 + 16 * qb + col) = l[qb] == 0.f ? -INFINITY : __builtin_fmaf(r.m[qb], kLn2, __logf(l[qb]));
    }
    for_rows_not_finite<D, 16>(r.o, scale, rows, [&](int x) { c.put_again(x0 + x, c.again(x0 + x, tiles, first, end), part); });
}

// Few rows: all of them in every wavefront, which has blocks of 32 keys of its own.
template <int D, int QB>
__device__ __forceinline__ void few_rows(const Setup<D> &c, const KeyTiles<BN, WindowMask> &tiles, int first, int end, int last, int part, char *k_stage,
                                         char *v_stage)
{
    constexpr int TILE = FEW * 2 * D, COPIES = TILE / 1024;       // copy instructions of a block's keys
    const PagedArgs &a = c.a;
    const int wave = wave_id(), lane = threadIdx.x & 63, col = F::column(), group = F::group();
    char *k_tile = k_stage + wave * TILE, *v_tile = v_stage + wave * TILE;
    Rows<D, FEW / 16, QB> r;
    r.clear();
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int x = min(16 * qb + col, c.t.rows - 1);
        r.pos[qb] = c.position(x);
#pragma unroll
        for (int ks = 0; ks < D / F::K; ++ks) r.q[qb][ks] = c.query(x, ks * F::K + group * 8);
    }
    const int lowest = c.position(0), highest = c.position(c.t.rows - 1);
    const LaneOffsets<D, 16> lo = lane_offsets<D, 16>();
    PagedDma<FEW, D, 1> dma;
    dma.init(c.key_row_bytes, 0);
    // block u of the part: half u % 2 of its key tile u / 2
    auto start_of = [&](int u) { return tiles.start(first + u / 2) + FEW * (u & 1); };
    const int blocks = 2 * (end - first);
    int k_pages[2], v_pages[2], next_pages[2];
    auto issue_k = [&](int u) { dma.issue(start_of(u), last, k_pages, k_tile, [&](int page, int key) { return c.key_row(c.k, page, key); }); };
    auto issue_v = [&](int u) { dma.issue(start_of(u), last, v_pages, v_tile, [&](int page, int key) { return c.key_row(c.v, page, key); }); };
    // vmcnt(COPIES): all but the copies issued last have landed
    auto wait_older = [] {
        __builtin_amdgcn_s_waitcnt(0x0F70 | COPIES);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    static_assert(COPIES < 16, "vmcnt's low bits");
    // lgkmcnt(0): what was read of a stage has been read, before copies into it are issued
    auto reads_done = [] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_s_waitcnt(0xC07F);
    };
    int u = wave;
    if (u < blocks) {
        c.find_pages(start_of(u), last, k_pages);
        v_pages[0] = k_pages[0], v_pages[1] = k_pages[1];
        issue_k(u);
        issue_v(u);
    }
    for (; u < blocks; u += 4) {
        const int start = start_of(u), next = u + 4;
        const bool more = next < blocks;
        unsigned hidden = (unsigned)(v_pages[0] < 0) | (unsigned)(v_pages[1] < 0) << 1;
        if (more) c.find_pages(start_of(next), last, next_pages);
        f32x4 s[FEW / 16][QB];
        wait_older();                                // K is there
        r.scores(k_tile, lo, a.mask, start, lowest, highest, hidden, c.c2, s);
        if (more) {
            reads_done();
            k_pages[0] = next_pages[0], k_pages[1] = next_pages[1];
            issue_k(next);
            wait_older();                            // V is there
        } else {
            wait_lds_dma();
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        r.values(v_tile, lo, s);
        if (more) {
            reads_done();
            v_pages[0] = k_pages[0], v_pages[1] = k_pages[1];
            issue_v(next);
        }
    }
    // The wavefronts meet: maximum and sum of each row, then its result, in the order of the wavefronts.
    __shared__ float m_s[4][16 * QB], l_s[4][16 * QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const float l = sum_over_groups<16>(r.l[qb]);
        if (group == 0) m_s[wave][16 * qb + col] = r.m[qb], l_s[wave][16 * qb + col] = l;
    }
    // (a row of the wavefront's result: D floats, piece x of 4 at x ^ (row & 15); it takes the room of its keys and values)
    constexpr int HALF = D * 4 * 16;                 // bytes of 16 rows
    static_assert(HALF <= TILE, "16 rows to a stage");
    __syncthreads();
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int db = 0; db < D / 16; ++db)
            *(f32x4 *)((qb ? v_tile : k_tile) + col * (D * 4) + (((4 * db + group) ^ col) << 4)) = r.o[db][qb];
    __syncthreads();
    constexpr int PIECES = D / 4, STEP = 256 / PIECES;        // lanes of a row, rows of a step
    const int piece = threadIdx.x % PIECES;
    const int64_t all = (int64_t)a.p.n_tokens * a.p.n_q_heads;
    for (int x0 = 0; x0 < c.t.rows; x0 += STEP) {
        const int x = x0 + threadIdx.x / PIECES;
        const bool mine = x < c.t.rows;
        bool bad = false;
        if (mine) {
            float M = m_s[0][x];
#pragma unroll
            for (int w = 1; w < 4; ++w) M = fmaxf(M, m_s[w][x]);
            const float ref = M == -INFINITY ? 0.f : M;
            float L = 0.f;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = __builtin_amdgcn_exp2f(m_s[w][x] - ref);
                L += f * l_s[w][x];
                sum += f * *(const f32x4 *)((x < 16 ? k_stage : v_stage) + w * TILE + (x & 15) * (D * 4) + ((piece ^ (x & 15)) << 4));
            }
            const float total = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            bad = !(fabsf(total) < INFINITY) || !(L < INFINITY);
            if (a.parts > 1) {
                const int64_t flat = c.flat(x);
                *(f32x4 *)(a.part_o + (part * all + flat) * D + 4 * piece) = sum;
                if (piece == 0) a.part_ml[flat * a.parts + part] = make_float2(M, L);
            } else {
                const float inv = L == 0.f ? 0.f : 1.f / L;
                bf16x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = (__bf16)(sum[e] * inv);
                *(bf16x4 *)(c.out(x) + piece * 8) = w;
                if (piece == 0 && a.p.lse) *c.lse(x) = L == 0.f ? -INFINITY : __builtin_fmaf(M, kLn2, __logf(L));
            }
        }
        // (a wavefront holds whole rows)
        for (unsigned long long left = __ballot(bad); left != 0;) {
            const int at = (__ffsll((long long)left) - 1) / PIECES;
            left &= ~(((PIECES == 64 ? 0ull : 1ull << PIECES) - 1) << (at * PIECES));
            const int row = x0 + wave * (64 / PIECES) + at;
            c.put_again(row, c.again(row, tiles, first, end), part);
        }
    }
}

template <int D>
__global__ __launch_bounds__(256, 2) void mfma_paged_kernel(PagedArgs a)
{
    // Separate arrays: the compiler must see that copies into one do not touch what is read from the other.
    __shared__ __attribute__((aligned(16))) char stage_a[2 * BN * 2 * D];
    __shared__ __attribute__((aligned(16))) char stage_b[2 * BN * 2 * D];
    const int G = a.p.n_q_heads / a.p.n_kv_heads;
    int id = blockIdx.x;
    const int kh = id % a.p.n_kv_heads;              // (fastest: an XCD keeps reading the same heads; attn_mfma_fwd.hip)
    id /= a.p.n_kv_heads;
    const int part = id % a.parts;
    TileRows t;
    if (!find_tile(a, G, id / a.parts, t)) return;
    const Setup<D> c(a, t, G, kh);
    const int lowest = c.position(0), highest = c.position(t.rows - 1);
    const int keys = at_most(highest + 1, c.table.capacity());
    const KeyTiles<BN, WindowMask> tiles(a.mask, lowest, keys);
    const int n = at_least(0, tiles.n), first = at_most(n, a.parts > 1 ? part * a.tiles_per_part : 0);
    const int end = a.parts > 1 && part + 1 < a.parts ? at_most(n, first + a.tiles_per_part) : n;
    if (first >= end) {                              // no keys: what is left of the rows
        for (int x = threadIdx.x; x < t.rows && a.parts > 1; x += 256) a.part_ml[c.flat(x) * a.parts + part] = make_float2(-INFINITY, 0.f);
        if (a.parts > 1) return;
        for (int x = threadIdx.x / (D / 8); x < t.rows; x += 256 / (D / 8)) {
            *(uint4 *)(c.out(x) + threadIdx.x % (D / 8) * 16) = uint4{0, 0, 0, 0};
            if (threadIdx.x % (D / 8) == 0 && a.p.lse) *c.lse(x) = -INFINITY;
        }
        return;
    }
    if (t.rows > FEW) many_rows<D>(c, tiles, first, end, keys - 1, part, stage_a, stage_b);
    else if (t.rows > 16) few_rows<D, 2>(c, tiles, first, end, keys - 1, part, stage_a, stage_b);
    else few_rows<D, 1>(c, tiles, first, end, keys - 1, part, stage_a, stage_b);
}

int64_t tiles_most(const cf_attn_paged_params &p) { return (int64_t)p.n_tokens * (p.n_q_heads / p.n_kv_heads) / BM + p.n_seqs; }

}  // namespace

// Parts: so many that the chip's 512 workgroup slots each get several, of two key tiles at least.
void cut_paged_mfma(PagedArgs &a)
{
    const cf_attn_paged_params &p = a.p;
    const int64_t capacity = (int64_t)p.pages_per_seq * p.page_size, G = p.n_q_heads / p.n_kv_heads;
    int64_t keys = p.max_kv_len > 0 ? std::min<int64_t>(p.max_kv_len, capacity) : capacity;
    int64_t tiles = (keys + BN - 1) / BN;
    if (p.window > 0) tiles = std::min(tiles, ((int64_t)p.window + BM / G) / BN + 2 + ((int64_t)a.mask.sinks + BN - 1) / BN);
    const int64_t groups = tiles_most(p) * p.n_kv_heads, slots = 512;
    const int64_t parts = std::min<int64_t>({(8 * slots + groups - 1) / groups, (tiles + 1) / 2, kMostParts});
    a.parts = groups >= 4 * slots ? 1 : (int)std::max<int64_t>(1, parts);
    a.tiles_per_part = (int)((tiles + a.parts - 1) / a.parts);
}

hipError_t launch_paged_mfma(const PagedArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)(tiles_most(a.p) * a.p.n_kv_heads * a.parts));
    if (a.p.head_dim == 64) mfma_paged_kernel<64><<<grid, 256, 0, s>>>(a);
    else mfma_paged_kernel<128><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cf
