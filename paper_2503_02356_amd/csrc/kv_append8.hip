// Writing new tokens' keys and values into a paged cache of 8 bits.
//
// A wavefront has a block of 16 keys of one head, of K or of V: the new rows that fall into it (a lane a unit of 16 elements of one or two
// of them, rotation.h), their largest element, the block's scale, the older rows again where that grows, the new rows' numbers.  No other wavefront
// writes the block, so a scale is found, compared and written without atomics, the same in every run.  blockIdx.y: workgroups of rows and groups of
// heads of the queries (a lane a unit of a row), one behind the other in as many rows of the grid as they fill, then K and V of each head.
//
// Bound by memory where a call is large, 2 bytes read and 1 written of each element (and the queries both ways), and by its launch and three trips to memory, one behind
// the other (lists, rows and table, the scale that there is), where it is small.  Measured, us: 8192 tokens of 28 + 4 heads x 128, 28.4 with their queries (5.0 TB/s; what it reads is partly in the
// caches); one token of each of 256 sequences 5.6.  Queries in fewer workgroups than alone (rotate.hip), 128, since the blocks fill the chip with theirs (128 / 256 /
// 512: 4000 rows of 28 + 4 heads 14.2 / 13.8 / 15.6, of 16 + 4 x 64 7.9 / 8.9 / 10.0, 256 tokens of 64 + 8 7.9 / 9.4 / 10.1).
// All places of a head one behind the other.  All heads of a place beside each other, which touches a page once, gains 2 - 8 % in prompts whose inputs are in the caches and
// loses elsewhere (us, places / heads beside each other, heads x 128, three sets of inputs in turn: 1200 tokens of as many sequences, 28 + 4 13.7 / 16.7, 2048 of 28 + 4 20.6 / 25.4, 16000 rows of 28 + 4
// 59.6 / 60.9, of 8 + 8 40.2 / 44.9, 4000 of 64 + 8 33.7 / 34.4, 16000 keys and values of 8 heads alone 20.3 / 20.1; one set, in the caches, 16000 of 28 + 4 47.2 / 44.1).
#include <hip/hip_runtime.h>

#include "kv_append.h"
#include "paged_checks.h"
#include "pages8.h"

namespace cf {
namespace {

struct Append8Args {
    TurnArgs turn;                       // t[0]: queries
    const void *k, *v;
    int64_t kv_tok, kv_head;
    char *k_pages, *v_pages;
    int64_t page_tok, page_head;         // bytes
    float *k_scales, *v_scales;
    int64_t scale_page, scale_head;
    int row_blocks, query_rows;          // workgroups of rows of queries; of the grid's y, those that they fill
};

// Four elements times `factor`, as numbers.
__device__ __forceinline__ unsigned encode4(const float *x, float factor)
{
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * factor, x[1] * factor, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * factor, x[3] * factor, low, true);
}
// Four numbers times a power of two, rounded again.
__device__ __forceinline__ unsigned again4(unsigned w, float factor)
{
    const float x[4] = {__builtin_amdgcn_cvt_f32_fp8((int)w, 0), __builtin_amdgcn_cvt_f32_fp8((int)w, 1), __builtin_amdgcn_cvt_f32_fp8((int)w, 2),
                        __builtin_amdgcn_cvt_f32_fp8((int)w, 3)};
    return encode4(x, factor);
}

template <typename T, int D, bool INTERLEAVED>
__device__ __forceinline__ void add_to_block(const Append8Args &a, const BlockPlaces &places, int end, int place, bool values, int h)
{
    constexpr int UNITS = D / 16, PASSES = UNITS / 4, STEP = 64 / UNITS;     // units of a row; times that a lane has a row; rows of each time
    const int lane = threadIdx.x & 63, n = a.turn.n_seqs;
    const int32_t *cu = a.turn.cu;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, g = lo + lane * step;
        const unsigned long long before = __ballot(g < hi && places.first(cu[min(g, hi - 1)], g) <= place);
        lo += (63 - __clzll((long long)before)) * step;      // (lane 0 always says yes)
        hi = min(hi, lo + step);
    }
    const int seq = __builtin_amdgcn_readfirstlane(lo), begin = cu[seq];
    const NewRows rows(begin, cu[seq + 1], a.turn.lens[seq]);
    const NewBlocks blocks(rows);
    const int x = place - places.first(begin, seq);
    if (x >= blocks.n) return;
    const int key0 = (blocks.first + x) * kBlock8;
    const int u = lane % UNITS;
    const bool turned = !values && a.turn.inv_freq != nullptr;
    const Unit unit(u, D, turned ? a.turn.rot : 0, INTERLEAVED);
    // The new rows' loads first: they do not wait for the table.
    Eight<T> w0[PASSES], w1[PASSES];
    bool fresh[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int key = key0 + STEP * i + lane / UNITS;
        const int row = rows.q0 + (key - rows.first_position);
        fresh[i] = key >= blocks.begin && key < blocks.end && row < end;
        if (fresh[i]) {
            const T *from = (const T *)(values ? a.v : a.k) + (int64_t)row * a.kv_tok + (int64_t)h * a.kv_head;
            w0[i].load(from + unit.at[0]), w1[i].load(from + unit.at[1]);
        } else {
            w0[i] = w1[i] = {};
        }
    }
    const PageTable table{a.turn.table + (int64_t)seq * a.turn.table_stride, a.turn.pages, a.turn.shift, a.turn.n_pages};
    const int page = table.page_of(key0), in_page = table.row_in_page(key0);
    float *scale = (values ? a.v_scales : a.k_scales) + (int64_t)max(page, 0) * a.scale_page + (int64_t)h * a.scale_head + in_page / kBlock8;
    char *to = (values ? a.v_pages : a.k_pages) + (int64_t)page * a.turn.page_stride + (int64_t)in_page * a.page_tok + (int64_t)h * a.page_head;
    const bool older = blocks.begin > key0;                  // (the new rows are the block's from there on)
    const float scale_before = older ? *scale : 0.f;

    float e0[PASSES][8], e1[PASSES][8];
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        w0[i].get(e0[i]), w1[i].get(e1[i]);
        if (turned && unit.any() && fresh[i]) {
            Turn turn;
            turn.set(a.turn.inv_freq, unit, key0 + STEP * i + lane / UNITS, false);
            turn.apply<INTERLEAVED>(unit, e0[i], e1[i]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p = fabsf(e0[i][e]), q = fabsf(e1[i][e]);
            most = fmaxf(most, fmaxf(p < INFINITY ? p : 0.f, q < INFINITY ? q : 0.f));
        }
    }
    if (page < 0) return;
    most = wave_max(most);
    const int wanted = exponent_for(most), had = exponent_of(scale_before), exponent = older ? max(wanted, had) : wanted;
    if (older && exponent > had) {
        const float factor = power8(max(had - exponent, -40));       // (from 2^-20 on every number becomes 0)
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int r = STEP * i + lane / UNITS;
            if (key0 + r >= blocks.begin) continue;
            uint4 *at = (uint4 *)(to + (int64_t)r * a.page_tok + 16 * u);
            const uint4 w = *at;
            *at = uint4{again4(w.x, factor), again4(w.y, factor), again4(w.z, factor), again4(w.w, factor)};
        }
    }
    const float factor = inverse8(exponent);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        if (!fresh[i]) continue;
        char *at = to + (int64_t)(STEP * i + lane / UNITS) * a.page_tok;
        *(uint2 *)(at + unit.at[0]) = uint2{encode4(e0[i], factor), encode4(e0[i] + 4, factor)};
        *(uint2 *)(at + unit.at[1]) = uint2{encode4(e1[i], factor), encode4(e1[i] + 4, factor)};
    }
    if (lane == 0 && !(older && exponent == had)) *scale = power8(exponent);
}

template <typename T, int D, bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(256) void append8_kernel(Append8Args a)
{
    const int end = min(a.turn.n_tokens, a.turn.cu[a.turn.n_seqs]);
    if ((int)blockIdx.y < a.query_rows) {
        const unsigned id = blockIdx.y * gridDim.x + blockIdx.x, group = id / (unsigned)a.row_blocks;
        if ((int)group < a.turn.t[0].groups) turn_rows<INTERLEAVED, STREAM>(a.turn, end, (int)group, (int)(id - group * (unsigned)a.row_blocks));
        return;
    }
    const int which = blockIdx.y - a.query_rows, place = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const BlockPlaces places(a.turn.n_tokens, a.turn.n_seqs);
    if (place < (int)places.all(end, a.turn.n_seqs)) add_to_block<T, D, INTERLEAVED>(a, places, end, place, which & 1, which >> 1);
}

template <typename T, int D, bool STREAM>
void launch(const Append8Args &a, dim3 grid, hipStream_t s)
{
    if (a.turn.interleaved) append8_kernel<T, D, true, STREAM><<<grid, 256, 0, s>>>(a);
    else append8_kernel<T, D, false, STREAM><<<grid, 256, 0, s>>>(a);
}
template <typename T, int D>
void launch(const Append8Args &a, dim3 grid, hipStream_t s)
{
    a.turn.stream ? launch<T, D, true>(a, grid, s) : launch<T, D, false>(a, grid, s);
}

}  // namespace
}  // namespace cf

extern "C" int cf_kv_append8(const cf_kv_append8_params *p8, const cf_append_rotation *r, void *hip_stream)
{
    const char *who = "cf_kv_append8";
    if (!p8) return cf::fail(CF_EINVAL, "%s: params is NULL", who);
    const cf_kv_append_params *p = &p8->a;
    if (int rc = cf::check_append(p, who, true)) return rc;
    if (int rc = cf::check_scales(who, p8->k_scales, p8->v_scales, p8->scale_stride_page, p8->scale_stride_head, p->page_size)) return rc;
    if (r)
        if (int rc = cf::check_append_rotation(who, r, p->dtype, p->head_dim)) return rc;
    if (int rc = cf::check_rows(who, p->n_tokens, p->head_dim)) return rc;
    const int64_t blocks = (cf::BlockPlaces(p->n_tokens, p->n_seqs).all(p->n_tokens, p->n_seqs) + 3) / 4;
    if (blocks * 256 > 0xffffffffLL) return cf::fail(CF_EINVAL, "%s: %d sequences are more than one launch holds", who, p->n_seqs);
    cf::Append8Args a;
    a.turn = cf::turn_args(r ? &r->rotation : nullptr, p->head_dim, p->n_tokens, p->n_seqs, p->cu_seqlens_q, p->kv_lens);
    cf::queries_of(a.turn, r, p->dtype);
    cf::pages_of(a.turn, p);
    a.turn.group(128);
    a.k = p->k, a.v = p->v, a.kv_tok = p->kv_stride_tok, a.kv_head = p->kv_stride_head;
    a.k_pages = (char *)p->k_pages, a.v_pages = (char *)p->v_pages, a.page_tok = p->page_stride_tok, a.page_head = p->page_stride_head;
    a.k_scales = p8->k_scales, a.v_scales = p8->v_scales, a.scale_page = p8->scale_stride_page, a.scale_head = p8->scale_stride_head;
    const int rows = 256 / (p->head_dim / 16);
    a.row_blocks = (int)(((int64_t)p->n_tokens + rows - 1) / rows);
    a.query_rows = (int)(((int64_t)a.turn.t[0].groups * a.row_blocks + blocks - 1) / blocks);
    const int64_t y = (int64_t)a.query_rows + 2 * p->n_kv_heads;
    if (y > 65535 || y * blocks > 0x7fffffffLL) return cf::fail(CF_EINVAL, "%s: %lld rows of workgroups are more than one launch holds", who, (long long)y);
    const dim3 grid((unsigned)blocks, (unsigned)y);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (p->dtype == CF_FP32) p->head_dim == 64 ? cf::launch<float, 64>(a, grid, s) : cf::launch<float, 128>(a, grid, s);
    else p->head_dim == 64 ? cf::launch<unsigned short, 64>(a, grid, s) : cf::launch<unsigned short, 128>(a, grid, s);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CF_OK : cf::fail(CF_EHIP, "%s: %s", who, hipGetErrorString(e));
}
