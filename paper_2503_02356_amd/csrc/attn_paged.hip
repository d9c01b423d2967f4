// Attention of new tokens over a paged cache, and writing into the cache.
//
// Scalar kernels: one wavefront per (query row, head), pair by pair, fp32 arithmetic.  They serve the cross-check flag and what the matrix
// kernels do not cover.  Tiles of 64 keys are gone through in order, a lane to a key; a hidden key is never read.  Bound by a lane's loads of its key,
// 16 or 32 of them behind each other (64 tokens behind up to 4000 keys, 8/2 heads, D = 128: 1.43 ms in bf16, 1.93 in fp32).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "common.h"
#include "paged.h"

namespace cf {
namespace {

constexpr int kWaves = 4;        // wavefronts per workgroup of the scalar kernels

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void paged_rows_kernel(PagedArgs a)
{
    const cf_attn_paged_params &p = a.p;
    __shared__ float sq[kWaves][D];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = blockIdx.y;
    const int64_t row = (int64_t)blockIdx.x * kWaves + wave;
    if (row >= min(p.n_tokens, p.cu_seqlens_q[p.n_seqs])) return;      // whole wavefront leaves together; no barrier below
    const int seq = find_segment(p.cu_seqlens_q, p.n_seqs, (int)row);
    const NewRows rows = a.rows(seq);
    const PageTable table = a.table(seq);
    const int position = rows.position((int)row - rows.q0);
    const T *q = row_of<T>(p.q, (int)row, p.q_stride_tok, h, p.q_stride_head);
    for (int t = 0; t < D / 64; ++t) sq[wave][lane + 64 * t] = ld(q + lane + 64 * t);
    __builtin_amdgcn_wave_barrier();
    const KeyTiles<64, WindowMask> tiles(a.mask, position, at_most(position + 1, table.capacity()));
    const RowSums<T, D> r = paged_row<T, D, 0, 64>(a, table, position, h / (p.n_q_heads / p.n_kv_heads), tiles, 0, tiles.n, [&](int x) { return sq[wave][x]; });
    T *o = (T *)p.o + row * p.o_stride_tok + (int64_t)h * p.o_stride_head;
    const bool none = r.m == -INFINITY && r.z == 0.f;
    for (int t = 0; t < D / 64; ++t) st(o + lane + 64 * t, none ? 0.f : r.acc[t] / r.z);
    if (lane == 0 && p.lse) p.lse[(int64_t)h * p.n_tokens + row] = none ? -INFINITY : r.m + logf(r.z);
}

// O and LSE of the rows from their parts: WAVES wavefronts to a row, a lane to a part's maximum and sum, then to some elements of every
// WAVES-th part's result.  The order of the sums is fixed, so are the bits.  Bound by latency where there are few rows, else by the parts'
// bytes.  More than 16 parts: four wavefronts, 16 parts in flight each, the first ones before the weights are known (one token behind 8192
// keys, 32/8 heads, 64 parts: the whole call 13.9 us, with one wavefront and 8 in flight 17.4).  Fewer: one, 8 in flight, and only parts that
// had keys are read (256 tokens of 16 heads, 5 parts: 68 us, 75 with four wavefronts).
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(kWaves * 64) void paged_join_kernel(PagedArgs a)
{
    const cf_attn_paged_params &p = a.p;
    constexpr int E = D / 64, AT_ONCE = WAVES == 1 ? 8 : 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = wave % WAVES;
    const int64_t all = (int64_t)p.n_tokens * p.n_q_heads, r = (int64_t)blockIdx.x * (kWaves / WAVES) + wave / WAVES;
    const bool inside = r < all;                     // (part_o and part_ml hold all rows, also those of a padded batch that nobody wrote)
    const float *o_parts = a.part_o + (inside ? r : 0) * D + lane * E;
    float v[AT_ONCE][E], acc[E] = {};
    auto fetch = [&](int x, int part) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[x][e] = o_parts[(int64_t)part * all * D + e];
    };
    // held: of a part that had keys.  (One without holds anything.  A weight of 0 takes an infinity or a NaN along, as it does in one piece.)
    auto add = [&](int x, float w, bool held) {
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += held ? w * v[x][e] : 0.f;
    };
    auto fetch_every = [&](int x0) {
#pragma unroll
        for (int x = 0; x < AT_ONCE; ++x) fetch(x, min(x0 + WAVES * x, a.parts - 1));
    };
    if (WAVES > 1) fetch_every(sub);
    float2 ml = {-INFINITY, 0.f};
    if (inside && lane < a.parts) ml = a.part_ml[r * a.parts + lane];
    const int64_t rows = (int64_t)min(p.n_tokens, p.cu_seqlens_q[p.n_seqs]) * p.n_q_heads;
    // A part without keys is (-infinity, 0); (-infinity, NaN) is one whose scores are NaN (a maximum takes none), and so is its row.
    const unsigned long long with_keys = __ballot(!(ml.x == -INFINITY && ml.y == 0.f));
    const float M = wave_max(ml.x), ref = M == -INFINITY ? 0.f : M;
    const float w = __builtin_amdgcn_exp2f(ml.x - ref);
    const float L = wave_sum(w * ml.y);
    if constexpr (WAVES == 1) {
        for (unsigned long long left = with_keys; left != 0;) {
            int at[AT_ONCE], n = 0;
#pragma unroll
            for (int x = 0; x < AT_ONCE; ++x) {      // (the last one again where there are no more)
                at[x] = left != 0 ? __ffsll((long long)left) - 1 : at[x > 0 ? x - 1 : 0];
                n += left != 0;
                left &= left - 1;
                fetch(x, at[x]);
            }
#pragma unroll
            for (int x = 0; x < AT_ONCE; ++x) {
                const float wx = __shfl(w, at[x]);
                add(x, wx, x < n);
            }
        }
    } else {
        for (int x0 = sub;;) {
#pragma unroll
            for (int x = 0; x < AT_ONCE; ++x) {
                const int at = x0 + WAVES * x;
                const float wx = __shfl(w, at & 63);
                add(x, wx, at < a.parts && (with_keys >> (at & 63) & 1));
            }
            x0 += WAVES * AT_ONCE;
            if (x0 >= a.parts) break;
            fetch_every(x0);
        }
        __shared__ float sums[kWaves][E][64];
#pragma unroll
        for (int e = 0; e < E; ++e) sums[wave][e][lane] = acc[e];
        __syncthreads();
        if (sub != 0) return;
#pragma unroll
        for (int e = 0; e < E; ++e)
            for (int x = 1; x < WAVES; ++x) acc[e] += sums[wave + x][e][lane];
    }
    if (r >= rows) return;
    const int64_t row = r / p.n_q_heads, h = r - row * p.n_q_heads;
    T *o = (T *)p.o + row * p.o_stride_tok + h * p.o_stride_head;
    const bool none = M == -INFINITY && L == 0.f;
    const float inv = none ? 0.f : 1.f / L;
#pragma unroll
    for (int e = 0; e < E; ++e) st(o + lane * E + e, acc[e] * inv);
    if (lane == 0 && p.lse) p.lse[h * p.n_tokens + row] = none ? -INFINITY : __builtin_fmaf(M, 0.69314718055994530942f, logf(L));
}

// 16 bytes a thread: a token's key (blockIdx.y 0) or value row, all heads.  Bound by memory, few tokens by the launch and three loads that depend on
// each other (8192 tokens, 4 heads of 128, bf16: 10.5 us, 3.2 TB/s read and written; one token 2.4 us).
__global__ __launch_bounds__(256) void kv_append_kernel(cf_kv_append_params p, int shift, int units)
{
    const int bytes = p.dtype == CF_BF16 ? 2 : 4, per_row = units * p.n_kv_heads;      // units: 16-byte pieces of a head's row
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = id / per_row;
    const int rest = (int)(id - row * per_row), h = rest / units, unit = rest - h * units;
    // The sequence of the wavefront's first row, 64 bounds at a time, by all lanes, those behind the last row too (one that has left has no bound to
    // compare).  The others' are that or one of the next, or lie behind a run of empty ones: looked for at twice the distance each time.
    const int lane = threadIdx.x & 63, end = min(p.n_tokens, p.cu_seqlens_q[p.n_seqs]), first = __builtin_amdgcn_readfirstlane((int)row);
    if (first >= end) return;
    int lo = 0, hi = p.n_seqs;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, g = lo + lane * step;
        const unsigned long long before = __ballot(g < hi && p.cu_seqlens_q[min(g, hi - 1)] <= first);
        lo += (63 - __clzll((long long)before)) * step;      // (lane 0 always says yes)
        hi = min(hi, lo + step);
    }
    if (row >= end) return;
    int far = 1;
    while (far < p.n_seqs - lo && p.cu_seqlens_q[lo + far] <= row) far *= 2;
    const int near = lo + far / 2, seq = near + find_segment(p.cu_seqlens_q + near, min(far, p.n_seqs - lo) - far / 2, (int)row);
    const NewRows rows(p.cu_seqlens_q[seq], p.cu_seqlens_q[seq + 1], p.kv_lens[seq]);
    const PageTable table{p.block_table + (int64_t)seq * p.table_stride, p.pages_per_seq, shift, p.n_pages};
    const int position = rows.position((int)row - rows.q0), page = table.page_of(position);
    if (page < 0) return;
    const char *from = (const char *)(blockIdx.y ? p.v : p.k) + (row * p.kv_stride_tok + (int64_t)h * p.kv_stride_head) * bytes;
    char *to = (char *)(blockIdx.y ? p.v_pages : p.k_pages) +
               ((int64_t)page * p.page_stride + (int64_t)table.row_in_page(position) * p.page_stride_tok + (int64_t)h * p.page_stride_head) * bytes;
    ((uint4 *)to)[unit] = ((const uint4 *)from)[unit];
}

template <typename T, int D>
hipError_t run_rows(const PagedArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)(((int64_t)a.p.n_tokens + kWaves - 1) / kWaves), (unsigned)a.p.n_q_heads);
    paged_rows_kernel<T, D><<<grid, kWaves * 64, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t run_join(const PagedArgs &a, hipStream_t s)
{
    const int64_t rows = (int64_t)a.p.n_tokens * a.p.n_q_heads;
    if (a.parts > 16 && rows <= 0x7fffffffLL / (kWaves * 64)) paged_join_kernel<T, D, 4><<<dim3((unsigned)rows), kWaves * 64, 0, s>>>(a);
    else paged_join_kernel<T, D, 1><<<dim3((unsigned)((rows + kWaves - 1) / kWaves)), kWaves * 64, 0, s>>>(a);
    return hipGetLastError();
}

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) % n) == 0; }

int check_common(const char *who, int dtype, int D, int n_tokens, int n_seqs, const int32_t *cu, const int32_t *lens, const int32_t *table,
                 int64_t table_stride, int pages, int page_size, int n_pages)
{
    if (dtype != CF_BF16 && dtype != CF_FP32) return fail(CF_EUNSUPPORTED, "%s: dtype %d not supported", who, dtype);
    if (D != 64 && D != 128) return fail(CF_EUNSUPPORTED, "%s: head_dim %d not supported (64 or 128)", who, D);
    if (n_tokens < 1 || n_seqs < 1 || n_seqs > (1 << 30))        // (the kernels' searches add two places or double one)
        return fail(CF_EINVAL, "%s: need n_tokens >= 1 and 1 <= n_seqs <= 2^30 (got %d, %d)", who, n_tokens, n_seqs);
    if (page_size < 16 || page_size > 65536 || (page_size & (page_size - 1)))
        return fail(CF_EINVAL, "%s: page_size %d must be a power of two from 16 to 65536", who, page_size);
    if (n_pages < 1 || pages < 1 || (int64_t)pages * page_size > (1 << 30) || table_stride < pages)
        return fail(CF_EINVAL, "%s: need n_pages >= 1, 1 <= pages_per_seq <= table_stride, pages_per_seq * page_size <= 2^30 (got %d, %d, %lld)", who,
                    n_pages, pages, (long long)table_stride);
    if (!cu || !lens || !table) return fail(CF_EINVAL, "%s: NULL device pointer", who);
    if (!aligned(cu, 4) || !aligned(lens, 4) || !aligned(table, 4)) return fail(CF_EINVAL, "%s: misaligned descriptor", who);
    return CF_OK;
}

int check_strides(const char *who, int dtype, int D, std::initializer_list<int64_t> strides)
{
    const int64_t vec = dtype == CF_BF16 ? 8 : 4;
    for (int64_t s : strides)
        if (s < D || s % vec != 0)
            return fail(CF_EINVAL, "%s: stride %lld must be >= head_dim and a multiple of %lld elements", who, (long long)s, (long long)vec);
    return CF_OK;
}

int check_paged(const cf_attn_paged_params *p, const char *who, bool sizes_only, PagedArgs *a)
{
    if (!p) return fail(CF_EINVAL, "%s: params is NULL", who);
    if (p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads != 0 || p->n_q_heads > 65535)
        return fail(CF_EINVAL, "%s: n_q_heads %d must be a positive multiple of n_kv_heads %d, at most 65535", who, p->n_q_heads, p->n_kv_heads);
    static const int32_t dummy[1] = {0};
    const int32_t *cu = sizes_only ? dummy : p->cu_seqlens_q, *lens = sizes_only ? dummy : p->kv_lens, *table = sizes_only ? dummy : p->block_table;
    if (int rc = check_common(who, p->dtype, p->head_dim, p->n_tokens, p->n_seqs, cu, lens, table, p->table_stride, p->pages_per_seq, p->page_size,
                              p->n_pages))
        return rc;
    if ((int64_t)p->n_tokens * p->n_q_heads > 0x7fffffffLL)
        return fail(CF_EINVAL, "%s: n_tokens * n_q_heads = %lld must be below 2^31", who, (long long)p->n_tokens * p->n_q_heads);
    if (p->flags & ~CF_FLAG_SCALAR_KERNELS) return fail(CF_EINVAL, "%s: unknown flags 0x%x", who, p->flags);
    if (p->max_kv_len < 0 || p->window < 0 || p->n_sinks < 0 || (p->window == 0 && p->n_sinks != 0))
        return fail(CF_EINVAL, "%s: need max_kv_len, window, n_sinks >= 0 and no sinks without a window (got %d, %d, %d)", who, p->max_kv_len, p->window,
                    p->n_sinks);
    a->p = *p;
    const int capacity = p->pages_per_seq * p->page_size;
    a->mask = p->window == 0 ? WindowMask{0x7fffffff, 0} : WindowMask{p->window, std::min(p->n_sinks, capacity)};
    a->shift = __builtin_ctz((unsigned)p->page_size);
    if (sizes_only) return CF_OK;
    if (!p->q || !p->k_pages || !p->v_pages || !p->o) return fail(CF_EINVAL, "%s: NULL device pointer", who);
    if (!(p->softmax_scale - p->softmax_scale == 0.f)) return fail(CF_EINVAL, "%s: softmax_scale is not finite", who);
    if (int rc = check_strides(who, p->dtype, p->head_dim, {p->q_stride_tok, p->q_stride_head, p->page_stride, p->kv_stride_tok, p->kv_stride_head,
                                                            p->o_stride_tok, p->o_stride_head}))
        return rc;
    if (!aligned(p->q, 16) || !aligned(p->k_pages, 16) || !aligned(p->v_pages, 16) || !aligned(p->o, 16) || !aligned(p->lse, 4))
        return fail(CF_EINVAL, "%s: q, pages and o must be 16-byte aligned", who);
    return CF_OK;
}

// The matrix kernels' offsets inside a group of 16 keys have 32 bits, and a HIP launch holds fewer than 2^32 work-items.  (Wider rows and
// larger calls: a wavefront to a row.)
enum Path { kRows, kMfma, kF32 };
Path path_of(const PagedArgs &a)
{
    if ((a.p.flags & CF_FLAG_SCALAR_KERNELS) || a.p.kv_stride_tok >= (1 << 25)) return kRows;
    if (a.p.dtype == CF_BF16) return paged_mfma_launch_size(a) <= 0xffffffffLL ? kMfma : kRows;
    return paged_f32_launch_size(a) <= 0xffffffffLL ? kF32 : kRows;
}
// Chooses the parts; bytes of workspace.
int64_t cut(PagedArgs &a)
{
    a.parts = 1, a.tiles_per_part = 1 << 28, a.part_o = nullptr, a.part_ml = nullptr;
    if (a.p.dtype == CF_BF16) cut_paged_mfma(a);
    else cut_paged_f32(a);
    if (path_of(a) == kRows) a.parts = 1;
    if (a.parts == 1) return 0;
    const int64_t rows = (int64_t)a.p.n_tokens * a.p.n_q_heads;
    return a.parts * rows * (a.p.head_dim * 4 + 8);
}

}  // namespace

hipError_t launch_paged_join(const PagedArgs &a, hipStream_t s)
{
    if (a.p.dtype == CF_FP32) return a.p.head_dim == 64 ? run_join<float, 64>(a, s) : run_join<float, 128>(a, s);
    return a.p.head_dim == 64 ? run_join<unsigned short, 64>(a, s) : run_join<unsigned short, 128>(a, s);
}

}  // namespace cf

extern "C" int64_t cf_attn_paged_workspace_bytes(const cf_attn_paged_params *p)
{
    cf::PagedArgs a;
    if (int rc = cf::check_paged(p, "cf_attn_paged_workspace_bytes", true, &a)) return rc;
    return cf::cut(a);
}

extern "C" int cf_attn_paged_fwd(const cf_attn_paged_params *p, void *hip_stream)
{
    const char *who = "cf_attn_paged_fwd";
    cf::PagedArgs a;
    if (int rc = cf::check_paged(p, who, false, &a)) return rc;
    const int64_t need = cf::cut(a);
    if (need > 0) {
        if (!p->workspace || !cf::aligned(p->workspace, 256)) return cf::fail(CF_EINVAL, "%s: workspace must be non-NULL and 256-byte aligned", who);
        if (p->workspace_bytes < need)
            return cf::fail(CF_EINVAL, "%s: workspace has %lld bytes, %lld needed", who, (long long)p->workspace_bytes, (long long)need);
        a.part_o = static_cast<float *>(p->workspace);
        a.part_ml = reinterpret_cast<float2 *>(a.part_o + (int64_t)a.parts * p->n_tokens * p->n_q_heads * p->head_dim);
    }
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const cf::Path path = cf::path_of(a);
    hipError_t e;
    if (path == cf::kMfma) e = cf::launch_paged_mfma(a, s);
    else if (path == cf::kF32) e = cf::launch_paged_f32(a, s);
    else if (p->dtype == CF_FP32) e = p->head_dim == 64 ? cf::run_rows<float, 64>(a, s) : cf::run_rows<float, 128>(a, s);
    else e = p->head_dim == 64 ? cf::run_rows<unsigned short, 64>(a, s) : cf::run_rows<unsigned short, 128>(a, s);
    if (e == hipSuccess && a.parts > 1) e = cf::launch_paged_join(a, s);
    return e == hipSuccess ? CF_OK : cf::fail(CF_EHIP, "%s: %s", who, hipGetErrorString(e));
}

extern "C" int cf_kv_append(const cf_kv_append_params *p, void *hip_stream)
{
    const char *who = "cf_kv_append";
    if (!p) return cf::fail(CF_EINVAL, "%s: params is NULL", who);
    if (p->n_kv_heads < 1 || p->n_kv_heads > 65535) return cf::fail(CF_EINVAL, "%s: n_kv_heads %d must be from 1 to 65535", who, p->n_kv_heads);
    if (int rc = cf::check_common(who, p->dtype, p->head_dim, p->n_tokens, p->n_seqs, p->cu_seqlens_q, p->kv_lens, p->block_table, p->table_stride,
                                  p->pages_per_seq, p->page_size, p->n_pages))
        return rc;
    if (!p->k || !p->v || !p->k_pages || !p->v_pages) return cf::fail(CF_EINVAL, "%s: NULL device pointer", who);
    if (int rc = cf::check_strides(who, p->dtype, p->head_dim, {p->kv_stride_tok, p->kv_stride_head, p->page_stride, p->page_stride_tok, p->page_stride_head}))
        return rc;
    if (!cf::aligned(p->k, 16) || !cf::aligned(p->v, 16) || !cf::aligned(p->k_pages, 16) || !cf::aligned(p->v_pages, 16))
        return cf::fail(CF_EINVAL, "%s: k, v and pages must be 16-byte aligned", who);
    const int units = p->head_dim * (p->dtype == CF_BF16 ? 2 : 4) / 16;
    const int64_t blocks = ((int64_t)p->n_tokens * p->n_kv_heads * units + 255) / 256;
    if (blocks * 256 > 0xffffffffLL) return cf::fail(CF_EINVAL, "%s: %d tokens of %d heads are more than one launch holds", who, p->n_tokens, p->n_kv_heads);
    cf::kv_append_kernel<<<dim3((unsigned)blocks, 2), 256, 0, static_cast<hipStream_t>(hip_stream)>>>(*p, __builtin_ctz((unsigned)p->page_size), units);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CF_OK : cf::fail(CF_EHIP, "%s: %s", who, hipGetErrorString(e));
}
