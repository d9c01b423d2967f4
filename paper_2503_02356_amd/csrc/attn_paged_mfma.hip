// bf16 attention of new tokens over a paged cache, head_dim 64 and 128.
//
// The rows of a sequence and a key/value head are its new tokens times the G query heads of the group, row r being token r / G, head r % G:
// they all multiply with the same keys and values.  A tile is 128 of them.  A workgroup (4 wavefronts, 16x16x32 MFMAs, everything
// transposed as in attn_mfma_fwd.hip: S^T = K Q^T, O^T += V^T P^T, the row on the lane axis) takes a tile and a part of its keys:
//   many rows  (more than 32)  a wavefront has 32 rows; key tiles of 64 are shared through LDS, double buffered.  Bound by the MFMAs and
//              the arithmetic between them, like the forward kernel of a chunk (8192 rows behind 24576 keys, 28/4 heads, D = 128: 2.96 ms,
//              1137 TFLOP/s; that kernel on contiguous keys 2.85).
//   few rows   every wavefront has all of them and takes every fourth block of 32 keys, copied into its own part of LDS: it waits for
//              nobody.  Bound by the memory that holds the cache: 16 KB of keys and values a wavefront, 8 wavefronts a compute unit, are in
//              flight or in use.  The four results meet in LDS at the end.  (64 tokens behind up to 16384 keys, 32/8 heads, D = 128, pages of 64:
//              2.43 GB in 441 us, 5.5 TB/s; 256 with a window of 1024, 16/4, D = 64, pages of 32: 58 us, 4.7 TB/s.)
// A long cache with few tiles is cut into parts, joined by a kernel behind this one (attn_paged.hip).
// Pages: 16 consecutive keys lie in one page (a page holds a multiple of 16), so that each copy instruction (512 / D rows of a tile) has one
// base, found with scalar instructions from a table entry that was loaded a tile ahead.  Keys that are hidden as a whole group (no such page,
// or behind the last key) are copied from a row of zeros, never from the pages, and masked.
// P's sum is taken in fp32.  Into the second product P goes as bf16 with, where rows are few, the bf16 rounding of what that rounding leaves (2^-16 of
// the value is left over): the wavefronts wait for memory and have the time (64 tokens behind up to 16384 keys 440.6 us without, 441.2 with; o's error
// against 64 bits 2.2e-3 without, 1.6e-3 with, which is o's own rounding).  Where rows are many it is as in cf_attn_fwd, so that evaluating over pages is
// what training computed: at head_dim 64 P keeps its bits (two operands leave 1.66e-3 in o, cf_attn_fwd's three 1.6e-3, one 2.3e-3; 8192 rows behind
// 24576 keys, 16/4 heads 1061 us with one, 1495 with two; cf_attn_fwd 1845), at head_dim 128 it is one operand (half a step, 2^-8 of the value, as o itself
// is rounded; 8192 rows behind 24576 keys 2883 us, with two 4044; o's error 2.3e-3 and 1.7e-3).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "paged_mfma.h"

namespace cf {
namespace {

constexpr int BM = 128, BN = 64;             // rows of a tile, keys of a key tile
constexpr int FEW = 32;                      // rows that the wavefronts share, keys of their blocks
// Tiles of FEW rows of a windowed chunk that goes this way: one round of workgroups; of half as many rows where that still is one round.  Forward,
// 28/4 heads, window 256, us, its rows to the wavefronts / its keys, tiles of 32 / of 16: 1 row behind 500 keys 11.5 / 8.0 / 7.9, 33 behind 500
// 13.5 / 11.3 / 8.1, 250 behind 5000 14.3 / 11.7 / 10.3, 500 behind 8000 14.4 / 13.4 / 16.7 (two rounds); 32/8 heads, window 4000: 100 behind 2000 41.5 /
// 27.0 / 19.6, 400 behind 2000 with tiles of 32 35.7, of 16 47.1.
constexpr int64_t kWindowFewTiles = 512;
// Copies a group of GROUP consecutive keys of one page into its place in a swizzled LDS tile, WAVES wavefronts together (an instruction of
// one of them: RPI rows).
template <int D, int GROUP, int WAVES>
struct GroupDma {
    static constexpr int RPI = 512 / D, UNITS = D / 8, COPIES = GROUP / (RPI * WAVES);
    static constexpr int KINDS = (RPI * WAVES) % 16 == 0 ? 1 : 16 / (RPI * WAVES);
    static_assert(COPIES >= 1, "a group is at least an instruction of each");
    int wv, r;                   // of the wavefronts that copy together; this lane's row of its first instruction
    unsigned row_bytes, unit16[KINDS], lane_off[KINDS];
    __device__ __forceinline__ void init(unsigned row_bytes_, int wave)
    {
        const int lane = threadIdx.x & 63;
        wv = wave;
        r = RPI * wave + lane / UNITS;
        row_bytes = row_bytes_;
#pragma unroll
        for (int i = 0; i < KINDS; ++i) {
            unit16[i] = ((lane % UNITS) ^ swz<D>(RPI * WAVES * i + r)) * 16;
            lane_off[i] = (unsigned)r * row_bytes + unit16[i];
        }
    }
    __device__ __forceinline__ void copy(__amdgpu_buffer_rsrc_t rsrc, char *lds, int c, unsigned off, unsigned scalar_off) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (CF_LDS void *)(lds + (c * WAVES + wv) * 1024), 16, (int)off, (int)scalar_off, 0, 0);
    }
    // room: rows of the group that may be read, less one; rows behind them read the last of these
    __device__ __forceinline__ void issue(const char *src, int room, char *lds) const
    {
        const __amdgpu_buffer_rsrc_t rsrc = TileDma<64, D>::descriptor(src);
        if (room >= GROUP - 1) {
#pragma unroll
            for (int c = 0; c < COPIES; ++c)
                copy(rsrc, lds, c, lane_off[c % KINDS], RPI * WAVES * c * row_bytes);
        } else {
#pragma unroll
            for (int c = 0; c < COPIES; ++c)
                copy(rsrc, lds, c, (unsigned)min(r + RPI * WAVES * c, room) * row_bytes + unit16[c % KINDS], 0);
        }
    }
};

// One row over the key tiles [first, end), pair by pair, into the call's tensors or as a part (a row whose result is not finite).
template <int D, bool CHUNK = false>
__device__ __forceinline__ void row_again(const PagedArgs &a, const TileRows &t, int x, const KeyTiles<BN, WindowMask> &tiles, int first, int end, int part)
{
    const int lane = threadIdx.x & 63;
    int64_t row;
    int h;
    t.find(x, row, h);
    const unsigned short *q = row_of<unsigned short>(a.p.q, (int)row, a.p.q_stride_tok, h, a.p.q_stride_head);
    const RowSums<unsigned short, D> r = paged_row<unsigned short, D, 4, BN>(
        a, CHUNK ? PageTable{(const int32_t *)zeros, 1, 30, 1} : a.table(t.seq), t.position(x), t.kh, tiles, first, end, [&](int e) { return ld(q + e); }, t.key0);
    const bool none = r.m == -INFINITY && r.z == 0.f;
    if (a.parts > 1) {
        const int64_t flat = t.flat(a, x);
        float *o = a.part_o + ((int64_t)part * a.p.n_tokens * a.p.n_q_heads + flat) * D;
        for (int e = 0; e < D / 64; ++e) o[lane + 64 * e] = r.acc[e];
        if (lane == 0) a.part_ml[flat * a.parts + part] = make_float2(r.m * kLog2e, r.z);
    } else {
        unsigned short *o = (unsigned short *)t.out(a, x);
        for (int e = 0; e < D / 64; ++e) st(o + lane + 64 * e, none ? 0.f : r.acc[e] / r.z);
        if (lane == 0) t.put_lse(a, x, none ? -INFINITY : r.m + logf(r.z));
    }
}

// Many rows: 32 to a wavefront, key tiles shared.
// WHOLE: a page holds 64 keys or more, so that a key tile has one base, else one for each 16 keys.  A tile that is not full, or that has a
// group of no page, is copied group by group.
template <int D, bool WHOLE>
__device__ __forceinline__ void many_rows(const PagedArgs &a, const TileRows &t, const KeyTiles<BN, WindowMask> &tiles, int first, int end, int keys,
                                          int part, char *stage_a, char *stage_b)
{
    constexpr int TILE = BN * 2 * D, GROUP = 16 * 2 * D, WAVES = D == 128 ? 4 : 2;      // (wavefronts that a group's rows take)
    const int wave = wave_id(), col = F::column(), group = F::group();
    const int x0 = 32 * wave, rows = at_most(32, t.rows - x0);           // this wavefront's rows of the tile (rows <= 0: none)
    const KeySource<2> src(a, t, keys);
    TileDma<BN, D> tile_dma;
    tile_dma.init(src.row_bytes);
    GroupDma<D, 16, WAVES> group_dma;
    group_dma.init(src.row_bytes, wave % WAVES);
    int pages[WHOLE ? 1 : 4];
    unsigned hidden = 0;
    auto find_pages = [&](int start, int (&p)[WHOLE ? 1 : 4]) {
#pragma unroll
        for (int g = 0; g < (WHOLE ? 1 : 4); ++g) p[g] = src.entry(start + 16 * g);
    };
    auto issue = [&](int start, char *stage) {
        bool plain = start + BN - 1 <= src.last;
#pragma unroll
        for (int g = 0; g < (WHOLE ? 1 : 4); ++g) plain = plain && src.is_page(pages[g]);
        hidden = 0;
        if (plain) {
            if constexpr (WHOLE) {
                const int64_t at = src.offset(pages[0], start);
                tile_dma.issue(src.k + at, BN - 1, stage);
                tile_dma.issue(src.v + at, BN - 1, stage + TILE);
            } else {
#pragma unroll
                for (int c = 0; c < WAVES; ++c) {
                    const int g = D == 128 ? c : 2 * c + (wave >> 1), page = D == 128 ? pages[c] : wave < 2 ? pages[2 * c] : pages[2 * c + 1];
                    const int64_t at = src.offset(page, start + 16 * g);
                    group_dma.issue(src.k + at, 15, stage + g * GROUP);
                    group_dma.issue(src.v + at, 15, stage + TILE + g * GROUP);
                }
            }
        } else {
#pragma unroll 1
            for (int g = 0; g < 4; ++g) {
                const int key = start + 16 * g, page = src.page_of(key);
                const int64_t at = page < 0 ? 0 : src.offset(page, key);
                const int room = page < 0 ? 0 : src.room(key);
                hidden |= (unsigned)(page < 0) << g;
                if (D == 64 && (wave >> 1) != (g & 1)) continue;
                group_dma.issue(page < 0 ? (const char *)zeros : src.k + at, room, stage + g * GROUP);
                group_dma.issue(page < 0 ? (const char *)zeros : src.v + at, room, stage + TILE + g * GROUP);
            }
        }
    };
    find_pages(tiles.start(first), pages);
    issue(tiles.start(first), stage_a);
    if (first + 1 < end) find_pages(tiles.start(first + 1), pages);

    Rows<D, BN / 16, 2, D == 64> r;
    r.clear();
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const int x = min(x0 + 16 * qb + col, t.rows - 1);
        r.pos[qb] = t.position(x);
#pragma unroll
        for (int ks = 0; ks < D / F::K; ++ks) r.q[qb][ks] = query(a, t, x, ks * F::K + group * 8);
    }
    const int lowest = t.position(at_most(x0, t.rows - 1)), highest = t.position(at_most(x0 + 31, t.rows - 1));
    const float c2 = score_factor(a);
    const WindowMask mask = a.mask;
    const LaneOffsets<D, 16> lo = lane_offsets<D, 16>();
    wait_lds_dma();
    __syncthreads();
    auto do_tile = [&](int n, const char *stage, char *next) {
        const int start = tiles.start(n);
        const unsigned hid = hidden;
        // (The table's entries are asked for before the copies are issued and waited for behind that: with scalar loads in flight no LDS read
        // can be waited for but all of them.)
        int coming[WHOLE ? 1 : 4] = {};
        if (n + 2 < end) find_pages(tiles.start(n + 2), coming);
        if (n + 1 < end) issue(tiles.start(n + 1), next);
        scalar_loads_done();
#pragma unroll
        for (int g = 0; g < (WHOLE ? 1 : 4); ++g) pages[g] = coming[g];
        if (rows > 0 && start <= highest && (start + BN > lowest + 1 - mask.window || start < mask.sinks)) {
            f32x4 s[BN / 16][2];
            r.scores(stage, lo, mask, start, lowest, highest, hid, c2, s);
            r.values(stage + TILE, lo, s);
        }
        wait_lds_dma();
        __syncthreads();
    };
    for (int n = first; n < end; n += 2) {
        do_tile(n, stage_a, stage_b);
        if (n + 1 < end) do_tile(n + 1, stage_b, stage_a);
    }
    if (rows <= 0) return;
    const PagedArgs &e = arguments();
    float l[2], scale[2];
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        l[qb] = sum_over_groups<16>(r.l[qb]);
        scale[qb] = l[qb] == 0.f ? 0.f : 1.f / l[qb];
    }
    if (e.parts > 1) {
        const int64_t all = (int64_t)e.p.n_tokens * e.p.n_q_heads;
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            const int x = 16 * qb + col;
            if (x >= rows) continue;
            const int64_t flat = t.flat(e, x0 + x);
            float *o = e.part_o + (part * all + flat) * D + 4 * group;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) *(f32x4 *)(o + 16 * db) = r.o[db][qb];
            if (group == 0) e.part_ml[flat * e.parts + part] = make_float2(r.m[qb], l[qb]);
        }
    } else {
        char *scratch = (wave < 2 ? stage_a : stage_b) + (wave & 1) * RowScratch<D>::bytes;
        store_rows_bf16<D, 16>(r.o, scale, scratch, rows, [&](int x) { return t.out(e, x0 + x); });
#pragma unroll
        for (int qb = 0; qb < 2; ++qb)
            if (group == 0 && 16 * qb + col < rows)
                t.put_lse(e, x0 + 16 * qb + col, l[qb] == 0.f ? -INFINITY : __builtin_fmaf(r.m[qb], kLn2, __logf(l[qb])));
    }
    for_rows_not_finite<D, 16>(r.o, scale, rows, [&](int x) { row_again<D>(e, t, x0 + x, tiles, first, end, part); });
}

// Few rows: all of them in every wavefront, which has blocks of 32 keys of its own.
template <int D, int QB, bool WHOLE, bool CHUNK>
__device__ __forceinline__ void few_rows(const PagedArgs &a, const TileRows &t, const KeyTiles<BN, WindowMask> &tiles, int first, int end, int keys,
                                         int part, char *k_stage, char *v_stage)
{
    constexpr int TILE = FEW * 2 * D, COPIES = TILE / 1024;       // copy instructions of a block's keys
    const int wave = wave_id(), col = F::column(), group = F::group();
    char *k_tile = k_stage + wave * TILE, *v_tile = v_stage + wave * TILE;
    const KeySource<2, CHUNK> src(a, t, keys);
    GroupDma<D, 32, 1> dma;
    dma.init(src.row_bytes, 0);
    GroupDma<D, 16, 1> half_dma;
    half_dma.init(src.row_bytes, 0);
    // block u of the part: half u % 2 of its key tile u / 2
    auto start_of = [&](int u) { return tiles.start(first + u / 2) + FEW * (u & 1); };
    const int blocks = 2 * (end - first);
    int pages[2], next_pages[2];                     // of the two halves
    auto find_pages = [&](int start, int (&p)[2]) {
        p[0] = src.entry(start);
        p[1] = WHOLE ? p[0] : src.entry(start + 16);
    };
    // (the same number of copies whatever the pages are: they are counted)
    auto issue = [&](const char *base, int start, const int (&p)[2], char *tile) {
        if constexpr (WHOLE) {
            const bool none = src.none(p[0], start);
            dma.issue(uniform(none ? (const char *)zeros : base + src.offset(p[0], start)), none ? 0 : src.room(start), tile);
        } else {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const bool none = src.none(p[g], start + 16 * g);
                half_dma.issue(uniform(none ? (const char *)zeros : base + src.offset(p[g], start + 16 * g)), none ? 0 : src.room(start + 16 * g),
                               tile + g * (16 * 2 * D));
            }
        }
    };
    // vmcnt(COPIES): all but the copies issued last have landed
    auto wait_older = [] {
        __builtin_amdgcn_s_waitcnt(0x0F70 | COPIES);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    static_assert(COPIES < 16, "vmcnt's low bits");
    // lgkmcnt(0): what was read of a stage has been read, before copies into it are issued
    auto reads_done = [] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        scalar_loads_done();
    };
    int u = wave;
    if (u < blocks) {
        find_pages(start_of(u), pages);
        issue(src.k, start_of(u), pages, k_tile);
        issue(src.v, start_of(u), pages, v_tile);
    }
    Rows<D, FEW / 16, QB, true> r;
    r.clear();
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int x = min(16 * qb + col, t.rows - 1);
        r.pos[qb] = t.position(x);
#pragma unroll
        for (int ks = 0; ks < D / F::K; ++ks) r.q[qb][ks] = query(a, t, x, ks * F::K + group * 8);
    }
    const int lowest = t.position(0), highest = t.position(t.rows - 1);
    const float c2 = score_factor(a);
    const WindowMask mask = a.mask;
    const LaneOffsets<D, 16> lo = lane_offsets<D, 16>();
    for (; u < blocks; u += 4) {
        const int start = start_of(u), next = u + 4;
        const bool more = next < blocks;
        // (keys behind the last one are those of later rows, or behind the table's last column, where groups end)
        const unsigned hidden = (unsigned)src.none(pages[0], start) | (unsigned)src.none(pages[1], start + 16) << 1;
        if (more) find_pages(start_of(next), next_pages);
        f32x4 s[FEW / 16][QB];
        wait_older();                                // K is there
        scalar_loads_done();
        r.scores(k_tile, lo, mask, start, lowest, highest, hidden, c2, s);
        if (more) {
            reads_done();
            issue(src.k, start_of(next), next_pages, k_tile);
            wait_older();                            // V is there
        } else {
            wait_lds_dma();
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        r.values(v_tile, lo, s);
        if (more) {
            reads_done();
            issue(src.v, start_of(next), next_pages, v_tile);
            pages[0] = next_pages[0], pages[1] = next_pages[1];
        }
    }
    const PagedArgs &e = arguments();
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
    const int64_t all = (int64_t)e.p.n_tokens * e.p.n_q_heads;
    for (int x0 = 0; x0 < t.rows; x0 += STEP) {
        const int x = x0 + threadIdx.x / PIECES;
        const bool mine = x < t.rows;
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
            if (e.parts > 1) {
                const int64_t flat = t.flat(e, x);
                *(f32x4 *)(e.part_o + (part * all + flat) * D + 4 * piece) = sum;
                if (piece == 0) e.part_ml[flat * e.parts + part] = make_float2(M, L);
            } else {
                const float inv = L == 0.f ? 0.f : 1.f / L;
                bf16x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = (__bf16)(sum[i] * inv);
                *(bf16x4 *)(t.out(e, x) + piece * 8) = w;
                if (piece == 0) t.put_lse(e, x, L == 0.f ? -INFINITY : __builtin_fmaf(M, kLn2, __logf(L)));
            }
        }
        // (a wavefront holds whole rows)
        for (unsigned long long left = __ballot(bad); left != 0;) {
            const int at = (__ffsll((long long)left) - 1) / PIECES;
            left &= ~(((PIECES == 64 ? 0ull : 1ull << PIECES) - 1) << (at * PIECES));
            const int row = x0 + wave * (64 / PIECES) + at;
            row_again<D, CHUNK>(e, t, row, tiles, first, end, part);
        }
    }
}

// MODE: FEW rows to a tile, all by few_rows; BM rows, all by many_rows; BOTH: BM rows, by what a tile holds; CHUNK: as FEW, keys in one piece;
// CHUNK_HALF: the same with half the rows.
enum Mode { kFew, kMany, kBoth, kChunk, kChunkHalf };
template <int D, Mode MODE, bool WHOLE>
__global__ __launch_bounds__(256, 2) void mfma_paged_kernel(PagedArgs a)
{
    // Separate arrays: the compiler must see that copies into one do not touch what is read from the other.
    __shared__ __attribute__((aligned(16))) char stage_a[2 * BN * 2 * D];
    __shared__ __attribute__((aligned(16))) char stage_b[2 * BN * 2 * D];
    TileRows t;
    t.G = a.p.n_q_heads / a.p.n_kv_heads;
    int id = blockIdx.x;
    t.kh = id % a.p.n_kv_heads;                      // (fastest: an XCD keeps reading the same heads; attn_mfma_fwd.hip)
    id /= a.p.n_kv_heads;
    const int part = id % a.parts;
    constexpr bool CHUNK = MODE == kChunk || MODE == kChunkHalf;
    if (!find_tile<MODE == kChunkHalf ? FEW / 2 : MODE == kFew || MODE == kChunk ? FEW : BM, CHUNK>(a, id / a.parts, t)) return;
    const int lowest = t.position(0), highest = t.position(t.rows - 1);
    const int keys = CHUNK ? highest + 1 : keys_within(highest, a.p.pages_per_seq, a.shift);
    const KeyTiles<BN, WindowMask> tiles(a.mask, lowest, keys);
    // (BOTH: tiles of many rows are cut a third as often, for a part of them leaves four times as much to be joined)
    const int thirds = MODE == kBoth && t.rows > FEW ? 3 : 1, per_part = a.tiles_per_part * thirds, last_part = (a.parts - 1) / thirds;
    const int n = at_least(0, tiles.n), first = at_most(n, a.parts == 1 ? 0 : part > last_part ? n : part * per_part);
    const int end = a.parts > 1 && part < last_part ? at_most(n, first + per_part) : n;
    if (first >= end) {                              // no keys: what is left of the rows
        const PagedArgs &e = arguments();
        for (int x = threadIdx.x; x < t.rows && e.parts > 1; x += 256) e.part_ml[t.flat(e, x) * e.parts + part] = make_float2(-INFINITY, 0.f);
        if (e.parts > 1) return;
        for (int x = threadIdx.x / (D / 8); x < t.rows; x += 256 / (D / 8)) {
            *(uint4 *)(t.out(e, x) + threadIdx.x % (D / 8) * 16) = uint4{0, 0, 0, 0};
            if (threadIdx.x % (D / 8) == 0) t.put_lse(e, x, -INFINITY);
        }
        return;
    }
    if (MODE == kMany || (MODE == kBoth && t.rows > FEW)) {
        many_rows<D, WHOLE>(a, t, tiles, first, end, keys, part, stage_a, stage_b);
    } else if constexpr (MODE != kMany) {
        if (MODE != kChunkHalf && t.rows > 16) few_rows<D, 2, WHOLE, CHUNK>(a, t, tiles, first, end, keys, part, stage_a, stage_b);
        else few_rows<D, 1, WHOLE, CHUNK>(a, t, tiles, first, end, keys, part, stage_a, stage_b);
    }
}

// Tiles of single tokens and short runs only, of chunks only, or of both?  By the mean number of token-head rows of a sequence; every kernel
// takes any of them.  From how many on a call goes as chunks only, 256 / 512 / 1024 rows, us, 28/4 heads, D = 128: 40 tokens behind up to 4000 keys
// beside a chunk of 4096 301 / 301 / 917, 5 behind up to 8000 beside 700 132 / 132 / 177, 10 behind up to 30000 beside 1000 613 / 613 / 629; 32/8, 16
// beside four of 500 137 / 146 / 146, 30 beside two of 2048 162 / 520 / 520; 16/4, D = 64, 10 behind up to 9000 beside 2000 157 / 157 / 132.  (A call's
// mean says little of its sequences: with a few long chunks beside tokens, a call for each kind may be faster than one for both.)
Mode mode_of(const cf_attn_paged_params &p)
{
    const int64_t rows = (int64_t)p.n_tokens * (p.n_q_heads / p.n_kv_heads);
    return rows <= (int64_t)FEW * p.n_seqs ? kFew : p.n_seqs == 1 || rows >= 512 * (int64_t)p.n_seqs ? kMany : kBoth;
}
int64_t tiles_most(const cf_attn_paged_params &p)
{
    return places_most(p.n_tokens, p.n_seqs, p.n_q_heads / p.n_kv_heads, mode_of(p) == kFew ? FEW : BM);
}

}  // namespace

int64_t paged_mfma_launch_size(const PagedArgs &a) { return tiles_most(a.p) * a.p.n_kv_heads * a.parts * 256; }

// Parts: so many that the chip's 512 workgroup slots each get several, of four key tiles at least (two blocks of 32 keys to a wavefront; 32/8
// heads, us, parts of at least 2 / 4 / 6 tiles: one token behind 2000 keys 10.2 / 10.3 / 11.0, 8192 13.9 / 13.6 / 13.7, 4 behind up to 8192
// 24.7 / 21.9 / 18.9).
// Rounds of slots, us, D = 128 but where it says 64:
//   tokens, 3 / 4 / 5 / 6 / 8        32/8 heads: 8 behind up to 8000 keys 47.7 / 48.4 / 48.9 / 49.1 / 49.0, 32 up to 16000 214 / 217 / 209 / 210 / 210, 64 up to
//                                    16384 448 / 484 / 440 / 447 / 457, 128 up to 2000 146 / 146 / 141 / 141 / 156; 16/4, 64, 256 up to 4000 146 / 146 / 117 / 118 / 134
//   beside chunks, 4 / 6 / 8 / 12    32/8: 40 up to 9000 beside a chunk of 500 185 / 189 / 195 / 207, 100 up to 3000 beside three of 300 235 / 187 / 291 / 217;
//                                    28/4: 20 up to 20000 beside 1000 290 / 325 / 325 / 393; 64/8: 30 up to 9000 beside 500 527 / 300 / 359 / 317; 16/4, 64: 60 up
//                                    to 6000 beside two of 400 84 / 97 / 79 / 102.  None is best everywhere.
// Tiles of many rows beside tokens are cut into as many parts / half / a third / a sixth of them: of the same five calls 218 / 197 / 195 / 184,
// 247 / 270 / 291 / 301, 355 / 329 / 325 / 319, 340 / 313 / 359 / 518, 86 / 81 / 79 / 136; with few tokens, 28/4, 8 up to 4000 beside 200, 28.6 / 32.5 / 37.6 / 59.4.
void cut_paged_mfma(PagedArgs &a)
{
    const cf_attn_paged_params &p = a.p;
    const int64_t capacity = (int64_t)p.pages_per_seq * p.page_size, G = p.n_q_heads / p.n_kv_heads;
    int64_t keys = p.max_kv_len > 0 ? std::min<int64_t>(p.max_kv_len, capacity) : capacity;
    int64_t tiles = (keys + BN - 1) / BN;
    if (p.window > 0) tiles = std::min(tiles, ((int64_t)p.window + BM / G) / BN + 2 + ((int64_t)a.mask.sinks + BN - 1) / BN);
    const int64_t groups = tiles_most(p) * p.n_kv_heads, slots = 512;
    // Workgroup slots' rounds, and from how many on a call is left whole.  Parts of many rows leave and read again 128 KB of results each.
    const Mode mode = mode_of(p);
    const int64_t rounds = mode == kMany ? 1 : mode == kFew ? 5 : 8, enough = mode == kMany ? 1 : 4;
    const int64_t parts = std::min<int64_t>({(rounds * slots + groups - 1) / groups, (tiles + 3) / 4, kMostParts});
    a.parts = groups >= enough * slots ? 1 : (int)std::max<int64_t>(1, parts);
    a.tiles_per_part = (int)((tiles + a.parts - 1) / a.parts);
}

template <int D, bool WHOLE>
static hipError_t launch(const PagedArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)(tiles_most(a.p) * a.p.n_kv_heads * a.parts));
    switch (mode_of(a.p)) {
        case kFew: mfma_paged_kernel<D, kFew, WHOLE><<<grid, 256, 0, s>>>(a); break;
        case kMany: mfma_paged_kernel<D, kMany, WHOLE><<<grid, 256, 0, s>>>(a); break;
        default: mfma_paged_kernel<D, kBoth, WHOLE><<<grid, 256, 0, s>>>(a);
    }
    return hipGetLastError();
}
// A windowed chunk of few rows: its wavefronts share the keys instead of the rows.
bool window_few(const cf_attn_fwd_params &p)
{
    return ((int64_t)p.n_tokens * (p.n_q_heads / p.n_kv_heads) / FEW + p.n_segments) * p.n_kv_heads <= kWindowFewTiles && (int64_t)p.n_tokens * p.n_q_heads < 0x7fffffffLL &&
           p.n_kv_tokens < (1 << 30);
}
hipError_t launch_window_few(const cf_attn_fwd_params &p, const WindowMask &mask, hipStream_t s)
{
    PagedArgs a{};
    a.p.dtype = p.dtype, a.p.n_q_heads = p.n_q_heads, a.p.n_kv_heads = p.n_kv_heads, a.p.head_dim = p.head_dim, a.p.softmax_scale = p.softmax_scale;
    a.p.n_tokens = p.n_tokens, a.p.n_seqs = p.n_segments, a.p.cu_seqlens_q = p.cu_seqlens_q, a.p.kv_lens = p.cu_seqlens_k;
    a.p.q = p.q, a.p.q_stride_tok = p.q_stride_tok, a.p.q_stride_head = p.q_stride_head;
    a.p.k_pages = p.k, a.p.v_pages = p.v, a.p.kv_stride_tok = p.kv_stride_tok, a.p.kv_stride_head = p.kv_stride_head;
    a.p.o = p.o, a.p.o_stride_tok = p.o_stride_tok, a.p.o_stride_head = p.o_stride_head, a.p.lse = p.lse;
    a.mask = mask, a.parts = 1, a.tiles_per_part = 1 << 28, a.shift = 30;
    auto grid = [&](int rows) { return dim3((unsigned)(((int64_t)p.n_tokens * (p.n_q_heads / p.n_kv_heads) / rows + p.n_segments) * p.n_kv_heads)); };
    if (((int64_t)p.n_tokens * (p.n_q_heads / p.n_kv_heads) / (FEW / 2) + p.n_segments) * p.n_kv_heads <= kWindowFewTiles) {
        if (p.head_dim == 64) mfma_paged_kernel<64, kChunkHalf, true><<<grid(FEW / 2), 256, 0, s>>>(a);
        else mfma_paged_kernel<128, kChunkHalf, true><<<grid(FEW / 2), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    if (p.head_dim == 64) mfma_paged_kernel<64, kChunk, true><<<grid(FEW), 256, 0, s>>>(a);
    else mfma_paged_kernel<128, kChunk, true><<<grid(FEW), 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_paged_mfma(const PagedArgs &a, hipStream_t s)
{
    const bool whole = a.p.page_size >= BN;
    if (a.p.head_dim == 64) return whole ? launch<64, true>(a, s) : launch<64, false>(a, s);
    return whole ? launch<128, true>(a, s) : launch<128, false>(a, s);
}

}  // namespace cf
