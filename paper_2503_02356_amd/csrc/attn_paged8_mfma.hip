// Attention of new tokens over a paged cache of 8 bits, head_dim 64 and 128: rows, tiles, parts, pages and the running softmax as in
// attn_paged_mfma.hip.
//
// A number times its power of two is a bf16 number exactly, so keys and values enter the bf16 matrix products (16x16x32) as they are:
// v_cvt_scalef32_pk_bf16_fp8 makes two operand elements of two bytes and their block's scale, a scalar, in one instruction.
//   many rows  (more than 32)  a key tile of 64 is converted once for the four wavefronts: each loads a quarter of its bytes into registers, a
//              tile ahead, and writes bf16 into the stage that attn_paged_mfma.hip's copies fill; from there on it is that kernel.
//   few rows   every wavefront has all of them and takes every fourth tile of 64 keys, copied as bytes into its own part of LDS (16 KB of keys
//              and values are in flight or in use, as there), and converts its operands itself.
// fp32: queries and P enter as three bf16 operands each, which make up all 24 bits of them; tiles of 16 rows, all of them few.
// (Products of bytes would take half the instructions, but queries would have to be bytes too, and the sums of the scaled 16x16x128 one are off by up to 6e-5 of
// the sum of their sizes: too much for scores, whose error is lse's.)
// P's sum is taken in fp32.  Into the second product P goes, in bf16, as over a cache of bf16 (attn_paged_mfma.hip):
//   few rows              two operands, the second one the rounding of what the first one's leaves (2^-16 of the value is left over).  64 tokens behind up to 16384 keys,
//                         32/8 x 128, 260.2 us and an error of o against 64 bits of 1.63e-3, which is o's own rounding; with one operand 259.7 and 1.75e-3
//   many rows, D = 64     two.  2048 rows behind 20000 keys, 16/4, 341 us and 1.58e-3; one 242 and 1.72e-3
//   many rows, D = 128    one: half a step, 2^-8 of the value, as o itself is rounded.  8192 rows behind 24576 keys, 28/4, 3.25 ms and 1.92e-3; two 4.37 and
//                         1.61e-3; 512 behind 8000 92 us and 1.82e-3; two 116 and 1.65e-3
//
// Many rows: bound by the matrix instructions and the vector ones between them (a wavefront's key tile takes 257 vector instructions, 224 of them the bf16
// kernel's, and 64 products).  8192 rows behind 24576 keys, 28/4 heads x 128: 3.25 ms, 1038 TFLOP/s (the bf16 kernel over a cache of twice the bytes 2.88 ms; a large
// matrix product 1234).  Steps there, ms: LDS writes spread over the banks 4.14 -> 3.50; lane addresses instead of descriptors, which with the tile's scalars were
// more than the scalar registers, 3.50 -> 3.23; the conversion in front of the scores 3.23, between scores and values 3.56, behind the values 3.32;
// raised priority around the products 3.37, around the conversion 3.24; eight wavefronts of 256 rows 3.38.
// Few rows: bound by memory.  64 tokens behind up to 16384 keys, 32/8 x 128: 260 us with its join for 1.22 GB (4.7 TB/s; 64 equally long sequences 5.3, a large copy's rate
// 5.1).  Keys straight into registers 309 (a row's 64 bytes an instruction: twice the requests); 16-row tiles of five wavefronts 1 % slower.  D = 64: 64 tokens
// behind 16000 keys, 16/4, 108 us (4.9 TB/s; 161 with the heads of a cache line on different XCDs, which fetches each line twice).  One token behind 4097 keys, 28/4: 7.1 us and 4 for the join.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "paged8.h"
#include "paged_mfma.h"

namespace cf {
namespace {

constexpr int BM = 128, BN = 64;             // rows of a tile, keys of a key tile
constexpr int FEW = 32;                      // rows that the wavefronts share
constexpr int FEWER = 16;                    // in fp32, and at D = 64 where sequences have no more (see mode_of)

// Key tiles as bytes in LDS: rows of D bytes, no padding, 16-byte unit u of row r at u ^ swz8(r).  Two rows (D = 128; four at 64) cover the 64 banks.
//   keys     ds_read_b128, lane's row = lane % 16, unit 4 s + lane / 16; served in groups of lanes 0-3, 12-15, 20-23, 24-27 and 4-11, 16-19,
//            28-31: unit u of rows 0-3, 12-15 beside unit u + 1 of rows 4-11
//   values   the transposing read of bytes (tr8 below), 32 lanes a clock: one unit of rows 0-7 beside the same of rows 16-23
// D = 128: h = row / 2 % 8 with bit 2 turned where row % 32 >= 16: h, or h ^ 1 for rows 4-11, are 8 different units of even and of odd
// rows, and 0-3 beside 8-11 turned are too.  D = 64: f = 0, 2, 3, 1 of row / 4 % 4, bit 0 turned likewise.
template <int D>
__device__ __forceinline__ int swz8(int row)
{
    if (D == 128) return (row >> 1 & 7) ^ (row >> 4 & 1) << 2;
    return ((((row >> 2) ^ (row >> 3)) & 1) << 1 | (row >> 3 & 1)) ^ (row >> 4 & 1);
}

// The numbers of four words, times the power of two `scale`, as bf16.
__device__ __forceinline__ bf16x8 numbers(int w0, int w1, int bits0, int bits1)
{
    const float scale0 = __builtin_bit_cast(float, bits0), scale1 = __builtin_bit_cast(float, bits1);
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w0, scale0, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w0, scale0, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w1, scale1, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w1, scale1, true);
    return __builtin_shufflevector(__builtin_shufflevector(a, b, 0, 1, 2, 3), __builtin_shufflevector(c, d, 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
}

// Where a workgroup's keys and their scales stand.
struct KeySource8 : KeySource<1> {
    const CF_CONSTANT int *k_scales, *v_scales;          // of this head (nothing writes them meanwhile: scalar loads)
    int64_t scale_page;
    __device__ __forceinline__ KeySource8(const Paged8Args &c, const TileRows &t, int keys)
        : KeySource<1>(c.a, t, keys), k_scales((const CF_CONSTANT int *)c.k_scales + (int64_t)t.kh * c.scale_head),
          v_scales((const CF_CONSTANT int *)c.v_scales + (int64_t)t.kh * c.scale_head), scale_page(c.scale_page)
    {
    }
    __device__ __forceinline__ int64_t scale_at(int page, int key) const { return page * scale_page + (key & ((1 << shift) - 1)) / kBlock8; }
    // The scales of N blocks from `key` on, of one page (of none, anything: see factors).  As integers, which stay in scalar registers.
    template <int N>
    __device__ __forceinline__ void scales(int entry, int key, int *k, int *v) const
    {
        const int64_t at = none(entry, key) ? 0 : scale_at(entry, key);
#pragma unroll
        for (int i = 0; i < N; ++i) k[i] = k_scales[at + i], v[i] = v_scales[at + i];
    }
};
// The factor of a block whose scale is `bits`: 1 where the block is hidden (what stands there, nobody may have written).
__device__ __forceinline__ int factor(int bits, unsigned hidden, int g) { return hidden >> g & 1 ? 0x3f800000 : bits; }

// Copies rows of a key tile, 16 or all 64 from its row `row0` on, into their place in LDS.  An instruction takes RPI rows, its swizzle is one of two.
template <int D>
struct Dma8 {
    static constexpr int RPI = 1024 / D, UNITS = D / 16;
    unsigned row_bytes, unit16[2], lane_off[2];
    int r;
    __device__ __forceinline__ static constexpr int kind(int c) { return D == 128 ? (c ^ c >> 1) & 1 : c & 1; }
    __device__ __forceinline__ void init(unsigned row_bytes_)
    {
        const int lane = threadIdx.x & 63;
        row_bytes = row_bytes_, r = lane / UNITS;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            unit16[i] = ((lane % UNITS) ^ swz8<D>(RPI * i + r)) * 16;
            lane_off[i] = (unsigned)r * row_bytes + unit16[i];
        }
    }
    // src: the group's first row
    template <int GROUP>
    __device__ __forceinline__ void issue(const char *src, char *tile, int row0) const
    {
        const __amdgpu_buffer_rsrc_t rsrc = TileDma<64, 128>::descriptor(src);
#pragma unroll
        for (int c = 0; c < GROUP / RPI; ++c) {
            const int at = row0 / RPI + c;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (CF_LDS void *)(tile + at * 1024), 16, (int)lane_off[kind(at)], (int)(RPI * c * row_bytes), 0, 0);
        }
    }
    // room: its rows that may be read, less one; rows behind them read the last of these
    template <int GROUP>
    __device__ __forceinline__ void issue_ragged(__amdgpu_buffer_rsrc_t rsrc, int room, char *tile, int row0) const
    {
#pragma unroll
        for (int c = 0; c < GROUP / RPI; ++c) {
            const int at = row0 / RPI + c;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (CF_LDS void *)(tile + at * 1024), 16,
                                                     (int)((unsigned)min(r + RPI * c, room) * row_bytes + unit16[kind(at)]), 0, 0, 0);
        }
    }
};

// One row over the key tiles [first, end), pair by pair, into the call's tensors or as a part (a row whose result is not finite).
template <typename T, int D>
__device__ __forceinline__ void row_again8(const Paged8Args &c, const TileRows &t, int x, const KeyTiles<BN, WindowMask> &tiles, int first, int end, int part)
{
    const PagedArgs &a = c.a;
    const int lane = threadIdx.x & 63;
    int64_t row;
    int h;
    t.find(x, row, h);
    const T *q = row_of<T>(a.p.q, (int)row, a.p.q_stride_tok, h, a.p.q_stride_head);
    const RowSums<float, D> r = paged8_row<D, 1, BN>(c, a.table(t.seq), t.position(x), t.kh, tiles, first, end, [&](int e) { return ld(q + e); });
    const bool none = r.m == -INFINITY && r.z == 0.f;
    if (a.parts > 1) {
        const int64_t flat = t.flat(a, x);
        float *o = a.part_o + ((int64_t)part * a.p.n_tokens * a.p.n_q_heads + flat) * D;
        for (int e = 0; e < D / 64; ++e) o[lane + 64 * e] = r.acc[e];
        if (lane == 0) a.part_ml[flat * a.parts + part] = make_float2(r.m * kLog2e, r.z);
    } else {
        T *o = (T *)t.out(a, x);
        for (int e = 0; e < D / 64; ++e) st(o + lane + 64 * e, none ? 0.f : r.acc[e] / r.z);
        if (lane == 0) t.put_lse(a, x, none ? -INFINITY : r.m + logf(r.z));
    }
}

// Eight elements of a query as operands: one of bf16, three of fp32.
__device__ __forceinline__ void query_operands(const PagedArgs &a, const TileRows &t, int x, int d, bf16x8 (&w)[1]) { w[0] = query(a, t, x, d); }
__device__ __forceinline__ void query_operands(const PagedArgs &a, const TileRows &t, int x, int d, bf16x8 (&w)[3])
{
    int64_t row;
    int h;
    t.find(x, row, h);
    const float4 *q = (const float4 *)((const float *)a.p.q + row * a.p.q_stride_tok + (int64_t)h * a.p.q_stride_head + d);
    const float4 lo = q[0], hi = q[1];
    float f[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = a.p.softmax_scale < 0.f ? -f[e] : a.p.softmax_scale == 0.f ? 0.f : f[e];
    split_exact(f, w);
}

// QB x 16 rows over key tiles of bytes.  QP, PP: operands that a query and P are made of (P: 2 leaves 2^-16 of it, 3 nothing).
template <int D, int QB, int QP, int PP>
struct Rows8 {
    static constexpr int KS = D / F::K, DB = D / 16;
    bf16x8 q[QP][QB][KS];
    f32x4 o[DB][QB];
    float m[QB], l[QB];          // as in Rows
    int pos[QB];
    int row_unit, tr8;           // this lane's offsets in a tile: of its key row's unit, and of its part of a transposing read

    __device__ __forceinline__ void clear()
    {
        const int lane = threadIdx.x & 63, group = lane / 16, e = lane % 16 / 2, row = (e < 4 ? 0 : 12) + 4 * group + e;
        row_unit = lane % 16 * D + ((group ^ swz8<D>(lane % 16)) << 4);
        tr8 = row * D + (swz8<D>(row) << 4) + 8 * (lane & 1);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            m[qb] = -INFINITY, l[qb] = 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db][qb] = F::zero();
        }
    }
    // The element of a query that contraction step ks, element 0 of a lane's eight, takes: a lane reads 16 numbers of a key at once, which are two
    // steps' operands, so step ks has elements 64 (ks / 2) + 8 (ks % 2) + 16 group ..
    __device__ __forceinline__ static int element(int ks) { return 64 * (ks / 2) + 8 * (ks % 2) + 16 * F::group(); }

    __device__ __forceinline__ void scores(const char *k_tile, const int (&scale)[4], const WindowMask &mask, int start, int lowest, int highest,
                                           unsigned groups, float c2, f32x4 (&s)[4][QB])
    {
        i32x4 w[4][KS / 2];
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int x = 0; x < KS / 2; ++x)         // (rows 16 further turn the unit's bit 2, or 0, and so does x)
                w[kb][x] = *(const i32x4 *)(k_tile + kb * (16 * D) + (row_unit ^ ((D == 128 ? (kb ^ x) & 1 : 0) << 6) ^ ((D == 64 ? kb & 1 : 0) << 4)));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) s[kb][qb] = F::zero();
#pragma unroll
            for (int x = 0; x < KS / 2; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const bf16x8 k = numbers(w[kb][x][2 * y], w[kb][x][2 * y + 1], scale[kb], scale[kb]);
#pragma unroll
                    for (int n = 0; n < QP; ++n)
#pragma unroll
                        for (int qb = 0; qb < QB; ++qb) s[kb][qb] = F::mul(k, q[QP - 1 - n][qb][2 * x + y], s[kb][qb]);      // (smallest first)
                }
        }
        settle<D, 4, QB>(s, m, l, o, pos, mask, start, lowest, highest, groups, c2);
    }
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    __device__ __forceinline__ void values(const char *v_tile, const int (&scale)[4], const f32x4 (&s)[4][QB])
    {
        // (all reads together: left to itself the compiler waits for each where it is used)
        i32x2 w[2][DB];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int db = 0; db < DB; ++db) w[t][db] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((CF_LDS i32x2 *)(v_tile + t * (32 * D) + (tr8 ^ (db << 4))));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            bf16x8 p[QB][3];
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = s[2 * t + e / 4][qb][e % 4];
                if (PP == 3) {
                    split_exact(f, p[qb]);
                } else {
                    p[qb][0] = pack8(f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] -= (float)p[qb][0][e];
                    p[qb][1] = pack8(f);
                }
            }
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const bf16x8 v = numbers(w[t][db][0], w[t][db][1], scale[2 * t], scale[2 * t + 1]);
#pragma unroll
                for (int n = 0; n < PP; ++n)
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) o[db][qb] = F::mul(v, p[qb][PP - 1 - n], o[db][qb]);
            }
        }
    }
};

// Few rows: all of them in every wavefront, which has key tiles of its own.
// GROUPS: of a key tile, each in one page: 1 where a page holds 64 keys or more, 2 of 32, 4 of 16.  (256 tokens with a window of 1024 in pages of 32, 16/4 heads x 64,
// with their append: 40.3 us with 4, 39.6 with 2.)
template <typename T, int D, int QB, int GROUPS>
__device__ __forceinline__ void few_rows8(const Paged8Args &c, const TileRows &t, const KeyTiles<BN, WindowMask> &tiles, int first, int end, int keys, int part,
                                          char *k_stage, char *v_stage)
{
    constexpr int TILE = BN * D, COPIES = TILE / 1024, KEYS = BN / GROUPS;
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int QP = F32 ? 3 : 1, PP = F32 ? 3 : 2;
    const PagedArgs &a = c.a;
    const int wave = wave_id(), col = F::column(), group = F::group();
    char *k_tile = k_stage + wave * TILE, *v_tile = v_stage + wave * TILE;
    const KeySource8 src(c, t, keys);
    Dma8<D> dma;
    dma.init(src.row_bytes);
    auto find_pages = [&](int start, int (&p)[GROUPS]) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) p[g] = src.entry(start + KEYS * g);
    };
    auto find_scales = [&](int start, const int (&p)[GROUPS], int (&k)[4], int (&v)[4]) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) src.scales<KEYS / kBlock8>(p[g], start + KEYS * g, k + KEYS / kBlock8 * g, v + KEYS / kBlock8 * g);
    };
    // Where a tile's groups stand, and whether all of them are there as a whole.
    int64_t at[GROUPS];
    bool full;
    auto find_groups = [&](int start, const int (&p)[GROUPS]) {
        full = start + BN - 1 <= src.last;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            full = full && src.is_page(p[g]);
            at[g] = src.offset(p[g], start + KEYS * g);
        }
    };
    // (the same number of copies whatever the pages are: they are counted)
    auto issue = [&](const char *base, int start, const int (&p)[GROUPS], char *tile) {
        if (full) {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) dma.template issue<KEYS>(base + at[g], tile, KEYS * g);
        } else {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const int key = start + KEYS * g;
                const bool none = src.none(p[g], key);
                dma.template issue_ragged<KEYS>(TileDma<64, 128>::descriptor(uniform(none ? (const char *)zeros : base + at[g])), none ? 0 : src.room(key), tile,
                                                KEYS * g);
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
    int pages[GROUPS] = {}, next_pages[GROUPS] = {};
    int k_scale[4] = {}, v_scale[4] = {};
    int u = first + wave;
    if (u < end) {
        find_pages(tiles.start(u), pages);
        if (u + 4 < end) find_pages(tiles.start(u + 4), next_pages);
        find_groups(tiles.start(u), pages);
        issue(src.k, tiles.start(u), pages, k_tile);
        issue(src.v, tiles.start(u), pages, v_tile);
        find_scales(tiles.start(u), pages, k_scale, v_scale);
    }
    Rows8<D, QB, QP, PP> r;
    r.clear();
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int x = min(16 * qb + col, t.rows - 1);
        r.pos[qb] = t.position(x);
#pragma unroll
        for (int ks = 0; ks < D / F::K; ++ks) {
            bf16x8 w[QP];
            query_operands(a, t, x, r.element(ks), w);
#pragma unroll
            for (int n = 0; n < QP; ++n) r.q[n][qb][ks] = w[n];
        }
    }
    const int lowest = t.position(0), highest = t.position(t.rows - 1);
    const float c2 = score_factor(a);
    const WindowMask mask = a.mask;
    for (; u < end; u += 4) {
        const int start = tiles.start(u);
        const bool more = u + 4 < end;
        // (keys behind the last one are those of later rows, or behind the table's last column, where groups end)
        unsigned hidden = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) hidden |= (unsigned)src.none(pages[g * GROUPS / 4], start + 16 * g) << g;
        int after[GROUPS] = {};
        int k_next[4] = {}, v_next[4] = {};
        if (more) find_scales(tiles.start(u + 4), next_pages, k_next, v_next);
        if (u + 8 < end) find_pages(tiles.start(u + 8), after);
        f32x4 s[4][QB];
        wait_older();                                // K is there
        scalar_loads_done();
#pragma unroll
        for (int g = 0; g < 4; ++g) k_scale[g] = factor(k_scale[g], hidden, g), v_scale[g] = factor(v_scale[g], hidden, g);
        r.scores(k_tile, k_scale, mask, start, lowest, highest, hidden, c2, s);
        if (more) {
            find_groups(tiles.start(u + 4), next_pages);
            reads_done();
            issue(src.k, tiles.start(u + 4), next_pages, k_tile);
            wait_older();                            // V is there
        } else {
            wait_lds_dma();
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        r.values(v_tile, v_scale, s);
        if (more) {
            reads_done();
            issue(src.v, tiles.start(u + 4), next_pages, v_tile);
        }
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) pages[g] = next_pages[g], next_pages[g] = after[g];
#pragma unroll
        for (int g = 0; g < 4; ++g) k_scale[g] = k_next[g], v_scale[g] = v_next[g];
    }
    const Paged8Args &e8 = (const Paged8Args &)arguments();
    const PagedArgs &e = e8.a;
    // The wavefronts meet: maximum and sum of each row, then its result, in the order of the wavefronts.
    __shared__ float m_s[4][16 * QB], l_s[4][16 * QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const float l = sum_over_groups<16>(r.l[qb]);
        if (group == 0) m_s[wave][16 * qb + col] = r.m[qb], l_s[wave][16 * qb + col] = l;
    }
    // (a row of the wavefront's result: D floats, piece x of 4 at x ^ (row & 15); it takes the room of its keys and values)
    static_assert(D * 4 * 16 <= TILE, "16 rows to a stage");
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
                if constexpr (F32) {
                    *(f32x4 *)(t.out(e, x) + piece * 16) = sum * inv;
                } else {
                    bf16x4 w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = (__bf16)(sum[i] * inv);
                    *(bf16x4 *)(t.out(e, x) + piece * 8) = w;
                }
                if (piece == 0) t.put_lse(e, x, L == 0.f ? -INFINITY : __builtin_fmaf(M, kLn2, logf(L)));
            }
        }
        // (a wavefront holds whole rows)
        for (unsigned long long left = __ballot(bad); left != 0;) {
            const int at = (__ffsll((long long)left) - 1) / PIECES;
            left &= ~(((1ull << PIECES) - 1) << (at * PIECES));
            row_again8<T, D>(e8, t, x0 + wave * (64 / PIECES) + at, tiles, first, end, part);
        }
    }
}

// Many rows: 32 to a wavefront, key tiles shared.
template <int D, bool WHOLE>
__device__ __forceinline__ void many_rows8(const Paged8Args &c, const TileRows &t, const KeyTiles<BN, WindowMask> &tiles, int first, int end, int keys,
                                           int part, char *stage_a, char *stage_b)
{
    // A lane converts a unit of 16 bytes of K and of V of LOADS rows: a wavefront has 16 rows, one block of keys, of 4 units each.  What it
    // writes into a bf16 tile is served 8 lanes at a time, over 32 banks: lanes 8 x .. + 7 are 4 units of rows x and x + 8, whose swizzles differ in bit 0, so
    // that the one's even units stand beside the other's odd ones.
    constexpr int TILE = BN * 2 * D, LOADS = D / 64, GROUPS = WHOLE ? 1 : 4;
    const PagedArgs &a = c.a;
    const int wave = wave_id(), col = F::column(), group = F::group(), lane = threadIdx.x & 63;
    const int x0 = 32 * wave, rows = at_most(32, t.rows - x0);           // this wavefront's rows of the tile (rows <= 0: none)
    const KeySource8 src(c, t, keys);
    const int my_row = 8 * (lane >> 2 & 1) + (lane >> 3), my_unit = (lane & 3) + (D == 128 ? 4 * (wave & 1) : 0);      // row of the block
    const unsigned my_off = (unsigned)my_row * src.row_bytes + 16 * my_unit;
    auto block = [&](int i) { return D == 128 ? (wave >> 1) + 2 * i : wave; };
    int to[2];                                                           // (swz() has period 16 rows)
#pragma unroll
    for (int y = 0; y < 2; ++y) to[y] = tile_off<D>(my_row, 2 * my_unit + y) + (D == 128 ? wave >> 1 : wave) * (16 * 2 * D);
    i32x4 pages = {0, 0, 0, 0}, next_pages = pages;
    int k_scale[LOADS], v_scale[LOADS];              // (in vector registers: there are too few scalar ones, and their loads would have to be waited for early)
    i32x4 k_raw[LOADS], v_raw[LOADS];
    unsigned coming_hidden = 0;                      // blocks of the tile in the registers that are hidden as a whole
    // (addresses of the lane, in vector registers)
    const CF_GLOBAL char *k_lane = (const CF_GLOBAL char *)src.k + my_off, *v_lane = (const CF_GLOBAL char *)src.v + my_off;
    const CF_GLOBAL int *k_scale_lane = (const CF_GLOBAL int *)src.k_scales, *v_scale_lane = (const CF_GLOBAL int *)src.v_scales;
    asm volatile("" : "+v"(k_lane), "+v"(v_lane), "+v"(k_scale_lane), "+v"(v_scale_lane));
    auto my_page = [&](const i32x4 &p, int i) {
        return WHOLE ? p[0] : D == 128 ? (wave < 2 ? p[2 * i] : p[2 * i + 1]) : wave < 2 ? (wave == 0 ? p[0] : p[1]) : wave == 2 ? p[2] : p[3];
    };
    auto find_pages = [&](int start, i32x4 &p) {
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) p[g] = src.entry(start + 16 * g);
    };
    auto load = [&](int start) {
        bool plain = start + BN - 1 <= src.last;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) plain = plain && src.is_page(pages[g]);
        coming_hidden = 0;
        if (!plain) {
#pragma unroll
            for (int g = 0; g < 4; ++g) coming_hidden |= (unsigned)src.none(pages[WHOLE ? 0 : g], start + 16 * g) << g;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int key = start + 16 * block(i);
            const int page = my_page(pages, i);
            if (plain) {
                const int64_t at = src.offset(page, key), scale = src.scale_at(page, key);
                k_raw[i] = *(const CF_GLOBAL i32x4 *)(k_lane + at), v_raw[i] = *(const CF_GLOBAL i32x4 *)(v_lane + at);
                k_scale[i] = k_scale_lane[scale], v_scale[i] = v_scale_lane[scale];
            } else {
                const bool none = src.none(page, key);
                const int64_t at = none ? 0 : src.offset(page, key), scale = none ? 0 : src.scale_at(page, key);
                const int64_t back = (int64_t)(my_row - min(my_row, none ? 0 : src.room(key))) * src.row_bytes;
                const CF_GLOBAL char *k = k_lane + at - back, *v = v_lane + at - back;
                k_raw[i] = *(const CF_GLOBAL i32x4 *)(none ? (const CF_GLOBAL char *)zeros : k), v_raw[i] = *(const CF_GLOBAL i32x4 *)(none ? (const CF_GLOBAL char *)zeros : v);
                k_scale[i] = k_scale_lane[scale], v_scale[i] = v_scale_lane[scale];
            }
        }
    };
    auto convert = [&](char *stage) {
        if (coming_hidden != 0) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                k_scale[i] = factor(k_scale[i], coming_hidden, block(i)), v_scale[i] = factor(v_scale[i], coming_hidden, block(i));
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                *(bf16x8 *)(stage + 32 * i * 2 * D + to[y]) = numbers(k_raw[i][2 * y], k_raw[i][2 * y + 1], k_scale[i], k_scale[i]);
                *(bf16x8 *)(stage + TILE + 32 * i * 2 * D + to[y]) = numbers(v_raw[i][2 * y], v_raw[i][2 * y + 1], v_scale[i], v_scale[i]);
            }
    };
    find_pages(tiles.start(first), pages);
    load(tiles.start(first));
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
    convert(stage_a);
    unsigned hidden = coming_hidden;
    if (first + 1 < end) {
        find_pages(tiles.start(first + 1), pages);
        load(tiles.start(first + 1));
    }
    if (first + 2 < end) find_pages(tiles.start(first + 2), next_pages);
    __syncthreads();
    auto do_tile = [&](int n, const char *stage, char *next) {
        const int start = tiles.start(n);
        const unsigned hid = hidden;
        // (the table's entries are asked for before the conversion and waited for behind it: with scalar loads in flight no LDS read can be waited
        // for but all of them)
        pages = next_pages;
        if (n + 3 < end) find_pages(tiles.start(n + 3), next_pages);
        if (n + 1 < end) {
            convert(next);
            hidden = coming_hidden;
        }
        if (n + 2 < end) load(tiles.start(n + 2));
        scalar_loads_done();
        if (rows > 0 && start <= highest && (start + BN > lowest + 1 - mask.window || start < mask.sinks)) {
            f32x4 s[BN / 16][2];
            r.scores(stage, lo, mask, start, lowest, highest, hid, c2, s);
            r.values(stage + TILE, lo, s);
        }
        __syncthreads();
    };
    for (int n = first; n < end; n += 2) {
        do_tile(n, stage_a, stage_b);
        if (n + 1 < end) do_tile(n + 1, stage_b, stage_a);
    }
    if (rows <= 0) return;
    const Paged8Args &e8 = (const Paged8Args &)arguments();
    const PagedArgs &e = e8.a;
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
                t.put_lse(e, x0 + 16 * qb + col, l[qb] == 0.f ? -INFINITY : __builtin_fmaf(r.m[qb], kLn2, logf(l[qb])));
    }
    for_rows_not_finite<D, 16>(r.o, scale, rows, [&](int x) { row_again8<unsigned short, D>(e8, t, x0 + x, tiles, first, end, part); });
}

// MODE: kFewer, kFew: tiles of FEWER and FEW rows, kMany: of BM rows, kBoth: of BM rows, by what a tile holds.
enum Mode { kFewer, kFew, kMany, kBoth };
template <typename T, int D, Mode MODE, int GROUPS>
__global__ __launch_bounds__(256, D == 64 && MODE == kFewer ? 4 : 2) void mfma_paged8_kernel(Paged8Args c)
{
    // Separate arrays: the compiler must see that what is written to one does not touch what is read from the other.
    constexpr int ROWS = MODE == kFewer ? FEWER : MODE == kFew ? FEW : BM, STAGE = MODE == kFewer || MODE == kFew ? 4 * BN * D : 2 * BN * 2 * D;
    __shared__ __attribute__((aligned(16))) char stage_a[STAGE];
    __shared__ __attribute__((aligned(16))) char stage_b[STAGE];
    const PagedArgs &a = c.a;
    TileRows t;
    t.G = a.p.n_q_heads / a.p.n_kv_heads;
    int id = blockIdx.x;
    if (D == 64 && MODE != kMany && a.p.n_kv_heads % 2 == 0) {
        // Two heads' 64 bytes are a cache line: both workgroups on one XCD (workgroups take turns on 8), one soon after the other.
        const HeadPair pair(id, gridDim.x);
        t.kh = pair.pair % (a.p.n_kv_heads / 2) * 2 + pair.second;
        id = pair.pair / (a.p.n_kv_heads / 2);
    } else {
        t.kh = id % a.p.n_kv_heads;                  // (fastest: an XCD keeps reading the same heads; attn_mfma_fwd.hip)
        id /= a.p.n_kv_heads;
    }
    const int part = id % a.parts;
    if (!find_tile<ROWS>(a, id / a.parts, t)) return;
    const int lowest = t.position(0), highest = t.position(t.rows - 1);
    const int keys = keys_within(highest, a.p.pages_per_seq, a.shift);
    const KeyTiles<BN, WindowMask> tiles(a.mask, lowest, keys);
    const int n = at_least(0, tiles.n), first = at_most(n, a.parts == 1 ? 0 : part * a.tiles_per_part);
    const int end = part < a.parts - 1 ? at_most(n, first + a.tiles_per_part) : n;
    if (first >= end) {                              // no keys: what is left of the rows
        const PagedArgs &e = arguments();
        for (int x = threadIdx.x; x < t.rows && e.parts > 1; x += 256) e.part_ml[t.flat(e, x) * e.parts + part] = make_float2(-INFINITY, 0.f);
        if (e.parts > 1) return;
        constexpr int UNITS = D * (int)sizeof(T) / 16;
        for (int x = threadIdx.x / UNITS; x < t.rows; x += 256 / UNITS) {
            *(uint4 *)(t.out(e, x) + threadIdx.x % UNITS * 16) = uint4{0, 0, 0, 0};
            if (threadIdx.x % UNITS == 0) t.put_lse(e, x, -INFINITY);
        }
        return;
    }
    if constexpr (MODE == kFewer) {
        few_rows8<T, D, 1, GROUPS>(c, t, tiles, first, end, keys, part, stage_a, stage_b);
    } else if (MODE == kMany || (MODE == kBoth && t.rows > FEW)) {
        many_rows8<D, GROUPS == 1>(c, t, tiles, first, end, keys, part, stage_a, stage_b);
    } else if constexpr (MODE != kMany) {
        if (t.rows > 16) few_rows8<T, D, 2, GROUPS>(c, t, tiles, first, end, keys, part, stage_a, stage_b);
        else few_rows8<T, D, 1, GROUPS>(c, t, tiles, first, end, keys, part, stage_a, stage_b);
    }
}

constexpr int64_t kSlots = 512;              // workgroups that run at once, two to a compute unit (of FEWER rows at D = 64 four; see cut_paged8_mfma)
// Key tiles that a tile of rows sees at most, as far as the host knows.
int64_t key_tiles(const cf_attn_paged_params &p)
{
    const int64_t capacity = (int64_t)p.pages_per_seq * p.page_size, keys = p.max_kv_len > 0 ? std::min<int64_t>(p.max_kv_len, capacity) : capacity;
    const int64_t tiles = (keys + BN - 1) / BN, sinks = std::min<int64_t>(p.n_sinks, capacity);
    return p.window > 0 ? std::min(tiles, ((int64_t)p.window + BM / (p.n_q_heads / p.n_kv_heads)) / BN + 2 + (sinks + BN - 1) / BN) : tiles;
}
// As in attn_paged_mfma.hip; and at D = 64, where with 16 rows a tile four workgroups have room on a compute unit, not three, such tiles in calls whose lengths are
// latencies more than bytes (us, FEW / FEWER rows, 16/4 heads: 32 tokens behind up to 4000 keys 19.5 / 15.9, 256 behind up to 500 17.1 / 14.4, 256 with a window of 1024 37.3 /
// 34.4; 64/8: 128 behind up to 2000 63.4 / 54.4; but 64 behind 16000 229 / 245, 16/4 109 / 115, 256 behind 4000 102 / 105; at D = 128, two either way, 32/8: 32 behind up
// to 4000 48.6 / 48.7, 128 behind up to 2000 84.3 / 91.7).
Mode mode_of(const cf_attn_paged_params &p)
{
    const int64_t rows = (int64_t)p.n_tokens * (p.n_q_heads / p.n_kv_heads);
    if (p.dtype == CF_FP32) return kFewer;
    if (p.head_dim == 64 && rows <= (int64_t)FEWER * p.n_seqs && key_tiles(p) <= 80 * kSlots / ((int64_t)p.n_seqs * p.n_kv_heads)) return kFewer;
    return rows <= (int64_t)FEW * p.n_seqs ? kFew : p.n_seqs == 1 || rows >= 512 * (int64_t)p.n_seqs ? kMany : kBoth;
}
int rows_of(Mode mode) { return mode == kFewer ? FEWER : mode == kFew ? FEW : BM; }
int64_t tiles_most(const cf_attn_paged_params &p)
{
    return places_most(p.n_tokens, p.n_seqs, p.n_q_heads / p.n_kv_heads, rows_of(mode_of(p)));
}

template <typename T, int D, int GROUPS>
hipError_t launch(const Paged8Args &c, hipStream_t s)
{
    const dim3 grid((unsigned)(tiles_most(c.a.p) * c.a.p.n_kv_heads * c.a.parts));
    if constexpr (sizeof(T) == 4) {
        mfma_paged8_kernel<T, D, kFewer, GROUPS><<<grid, 256, 0, s>>>(c);
    } else {
        const Mode mode = mode_of(c.a.p);
        if constexpr (D == 64) {
            if (mode == kFewer) {
                mfma_paged8_kernel<T, D, kFewer, GROUPS><<<grid, 256, 0, s>>>(c);
                return hipGetLastError();
            }
        }
        switch (mode) {
            case kFew: mfma_paged8_kernel<T, D, kFew, GROUPS><<<grid, 256, 0, s>>>(c); break;
            case kMany: mfma_paged8_kernel<T, D, kMany, GROUPS == 1 ? 1 : 4><<<grid, 256, 0, s>>>(c); break;
            default: mfma_paged8_kernel<T, D, kBoth, GROUPS><<<grid, 256, 0, s>>>(c);
        }
    }
    return hipGetLastError();
}
template <typename T, int D>
hipError_t launch(const Paged8Args &c, hipStream_t s)
{
    return c.a.p.page_size >= BN ? launch<T, D, 1>(c, s) : c.a.p.page_size == 32 ? launch<T, D, 2>(c, s) : launch<T, D, 4>(c, s);
}

}  // namespace

int64_t paged8_mfma_launch_size(const PagedArgs &a) { return tiles_most(a.p) * a.p.n_kv_heads * a.parts * 256; }

// Parts.  A part costs what it finds before its first keys and leaves behind its last ones, some 3 key tiles' time, and a join, 3 us and more: tiles of few rows are whole
// up to 8 key tiles, two to a wavefront (us, whole / cut: one token behind 300 keys, 28/4 heads, 7.8 / 9.3, fp32, 6/2, 9.0 / 10.1; 1000 keys 11.4 / 9.3).  Parts have 4
// tiles at least, one to a wavefront, or 8 where that makes more parts than there are workgroup slots (4 / 8 at least: one token behind 4097 keys 10.1 / 11.7, 4 behind 2000 9.5 /
// 11.2, 16 behind 2000 14.0 / 15.2, 30 with a window of 512 12.4 / 14.2; 4 behind 8000 14.8 / 14.3; 8 behind up to 8000, 32/8, 34.3 / 30.5); in fp32, whose tiles take
// longer, and beside chunks always 4; chunks 2 (four wavefronts have a tile together: 100 rows behind 1000, 28/4, 4 / 2 tiles at least 18.9 / 18.0, 16/4, D = 64, 14.1 / 12.4).
// Where all tiles see about as many keys (windows) the rounds of the slots decide: of 1 .. 64 parts those whose rounds, of a part's tiles and those 3 each, are shortest.
// (Two workgroups a compute unit are counted there also in tiles of FEWER rows at D = 64, of which four have room: what the others take of the memory's rate and a join cost more than
// the room gives, but for the longest windows.  us, for 512 / 1024 slots: 128 tokens of 16/4 with a window of 512 12.4 / 17.5, of 1024 17.9 / 21.4, of 2048 38.4 / 38.0, of 4096 70.5 / 62.7; 64
// of 64/8, 1024 to 4096, 16.5 / 22.7, 33.6 / 42.6, 60.6 / 73.9; 256 of 14/2 17.5 / 22.8, 37.2 / 40.6, 67.4 / 65.8; 32 of 32/8 15.4 / 15.6, 21.0 / 20.7, 45.7 / 38.0.)
// Chunks, and all calls in fp32: the same with what a step, a key tile (of few rows four), takes a workgroup alone on its compute unit and beside others, 1.5 and 2.5 us at D =
// 128 (1.5, 2.3 and 3 at 64; fp32 2.4 and 3.2, 1.7 to 2.5), and a join 3 us, of many rows 4, and its bytes' time (us, parts 1 / 2 / 3 / 4 / 8: 512 rows behind 8000 keys, 28/4,
// 207 / 120 / 114 / 92 / 100, behind none 19 / 24 / 23 / 23 / 23, 1000 behind 1000 55 / 59 / 58 / 63 / 76, 2048 behind 20000 702 / 752 / 723 / 683 / 715, 16/4, D = 64, 512 /
// 385 / 341 / 348 / 339; fp32, 6/2 x 128: 300 behind 5000 59 / 37 / 34 / 30 / 37, 2000 behind none 37 / 55 / 52 / 72 / 102, 64 tokens behind up to 5000 59 / 47 / 37 / 35 / 40,
// 200 behind up to 600 19 / 27 / 23 / 33 / 34).
// Single tokens whose lengths nobody knows here: enough parts for 5 rounds (us, rounds 3 / 4 / 5 / 6 / 8: 64 tokens behind up to 16384 keys, 32/8, 266 / 301 / 262 / 268 / 280;
// 32 up to 16000 139 / 141 / 132 / 134 / 135; 128 up to 2000 85 / 85 / 73 / 73 / 101), in tiles of FEWER rows, of which more run at once, for 8 (5 / 8 / 10 / 12 / 16: 32 up
// to 16000, 16/4, 46 / 42 / 42 / 42 / 42; 128 up to 2000, 64/8, 62 / 54 / 67 / 67 / 67; 256 up to 4000, 14/2, 52 / 46 / 45 / 57 / 57).  (Longer parts first and short ones last,
// in the order of the parts, gains nothing: the memory's rate, 5.3 TB/s where all sequences are equally long, is all but reached.)
// Tokens beside chunks, all cut alike: 5 rounds (us, rounds 3 / 5 / 8: 40 up to 9000 keys beside a chunk of 500, 32/8, 201 / 130 / 138; 100 up to 3000 beside three of 300
// 151 / 142 / 181; 20 up to 20000 beside 1000, 28/4, 409 / 395 / 424; 30 up to 9000 beside 500, 64/8, 127 / 138 / 193; with chunks cut a third as often, as in
// attn_paged_mfma.hip, at 8 rounds 126, 234, 457, 260).
void cut_paged8_mfma(PagedArgs &a)
{
    const cf_attn_paged_params &p = a.p;
    const int64_t tiles = key_tiles(p), G = p.n_q_heads / p.n_kv_heads, slots = kSlots;
    const Mode mode = mode_of(p);
    const bool few = mode == kFewer || mode == kFew;
    const int64_t rows = rows_of(mode), groups = std::max<int64_t>(p.n_seqs, (p.n_tokens * G + rows - 1) / rows) * p.n_kv_heads;      // (tiles that there are at least)
    const int64_t least = few && p.dtype == CF_BF16 && (tiles + 3) / 4 > slots / groups ? 8 : mode == kMany ? 2 : 4;
    const int64_t most = few && tiles <= 8 ? 1 : std::min<int64_t>((tiles + least - 1) / least, kMostParts);
    auto rounds_of = [&](int64_t parts) { return (groups * parts + slots - 1) / slots; };
    int64_t parts = 1;
    if (groups < (mode == kMany ? 1 : 4) * slots) {
        auto shortest = [&](auto time) {
            for (int64_t n = 2; n <= most; ++n)
                if (time(n) < time(parts)) parts = n;
        };
        if (mode == kMany || p.dtype == CF_FP32) {
            // Hundredths of a microsecond; t[k]: a step's, of one of k workgroups on a compute unit.
            constexpr int many64[] = {150, 150, 225, 300}, many128[] = {150, 150, 250}, fp32_64[] = {170, 170, 190, 220, 250}, fp32_128[] = {240, 240, 320};
            const bool wide = p.head_dim == 128, chunk = mode == kMany;
            const int *t = chunk ? (wide ? many128 : many64) : wide ? fp32_128 : fp32_64;
            const int64_t together = 256 * (wide ? 2 : chunk ? 3 : 4), at_once = chunk ? 1 : 4, around = chunk ? 3 : 2;
            shortest([&](int64_t n) {
                const int64_t steps = ((tiles + n - 1) / n + at_once - 1) / at_once + around, full = groups * n / together, rest = groups * n % together, k = rest / 256;
                const int64_t last = rest == 0 ? 0 : chunk ? t[(rest + 255) / 256] : t[k] + (t[k + 1] - t[k]) * (rest % 256) / 256;
                return steps * (full * t[together / 256] + last) + (n == 1 ? 0 : (chunk ? 400 : 300) + n * p.n_tokens * p.n_q_heads * p.head_dim * 8 / 50000);
            });
        } else if (few && p.window > 0) {
            shortest([&](int64_t n) { return rounds_of(n) * ((tiles + n - 1) / n + 3) + (n > 1 ? 3 : 0); });
        } else {
            const int64_t places = tiles_most(p) * p.n_kv_heads;
            parts = std::min(((mode == kFewer && p.dtype == CF_BF16 ? 8 : 5) * slots + places - 1) / places, most);
        }
    }
    a.parts = (int)std::max<int64_t>(1, parts);
    a.tiles_per_part = (int)((tiles + a.parts - 1) / a.parts);
}

hipError_t launch_paged8_mfma(const Paged8Args &c, hipStream_t s)
{
    if (c.a.p.dtype == CF_FP32) return c.a.p.head_dim == 64 ? launch<float, 64>(c, s) : launch<float, 128>(c, s);
    return c.a.p.head_dim == 64 ? launch<unsigned short, 64>(c, s) : launch<unsigned short, 128>(c, s);
}

}  // namespace cf
