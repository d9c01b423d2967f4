// Rotation of a training chunk's queries and keys and of their gradients, and the append to a paged cache that rotates on the way.
//
// One launch for all tensors of a call.  Measured, us: 64 + 8 heads x 128 of 32768 rows in bf16, there and back, 526, which is
// 92 % of the rate of a large copy (5.1 TB/s); 28 + 4 heads of 8192 packed rows there and back 58 (93 %); one token into pages 4.7, 5.5 with its launch.
#include <hip/hip_runtime.h>

#include "kv_append.h"
#include "paged_checks.h"
#include "rotation.h"

namespace cf {
namespace {

// A lane a unit of a row (rotation.h) of the heads of a group; a group of heads to each blockIdx.y.  The first heads' loads are on their way while the
// row's page is looked up and its sines are taken.
template <bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(256) void turn_rows_kernel(TurnArgs a)
{
    turn_rows<INTERLEAVED, STREAM>(a, min(a.n_tokens, a.cu[a.n_seqs]), blockIdx.y, blockIdx.x);
}

}  // namespace

hipError_t launch_turn_rows(const TurnArgs &a, hipStream_t s)
{
    const int rows = 256 >> a.units_shift;
    const dim3 grid((unsigned)(((int64_t)a.n_tokens + rows - 1) / rows), (unsigned)a.all_groups());
    if (a.interleaved) a.stream ? turn_rows_kernel<true, true><<<grid, 256, 0, s>>>(a) : turn_rows_kernel<true, false><<<grid, 256, 0, s>>>(a);
    else a.stream ? turn_rows_kernel<false, true><<<grid, 256, 0, s>>>(a) : turn_rows_kernel<false, false><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

int check_rotation(const char *who, const cf_rotation &r, int D)
{
    if (!r.inv_freq || !aligned(r.inv_freq, 4)) return fail(CF_EINVAL, "%s: inv_freq must be a device pointer to floats", who);
    if (r.rot_dim < 16 || r.rot_dim > D || r.rot_dim % 16 != 0)
        return fail(CF_EINVAL, "%s: rot_dim %d must be a multiple of 16 from 16 to head_dim %d", who, r.rot_dim, D);
    return CF_OK;
}

int check_turned(const char *who, const char *name, int D, int dtype_in, int dtype_out, int n_heads, const void *x, int64_t x_tok, int64_t x_head,
                 const void *y, int64_t y_tok, int64_t y_head)
{
    if ((dtype_in != CF_BF16 && dtype_in != CF_FP32) || (dtype_out != CF_BF16 && dtype_out != CF_FP32) || (dtype_in == CF_BF16 && dtype_out != CF_BF16))
        return fail(CF_EUNSUPPORTED, "%s: %s from dtype %d to %d not supported", who, name, dtype_in, dtype_out);
    if (n_heads < 1 || n_heads > 65535) return fail(CF_EINVAL, "%s: %s: %d heads, need 1 to 65535", who, name, n_heads);
    if (!x || !y || !aligned(x, 16) || !aligned(y, 16)) return fail(CF_EINVAL, "%s: %s and its result must be non-NULL and 16-byte aligned", who, name);
    if (int rc = check_strides(who, dtype_in, D, {x_tok, x_head})) return rc;
    if (int rc = check_strides(who, dtype_out, D, {y_tok, y_head})) return rc;
    if (x == y && (dtype_in != dtype_out || x_tok != y_tok || x_head != y_head))
        return fail(CF_EINVAL, "%s: %s in place needs the same dtype and strides", who, name);
    return CF_OK;
}

int check_append_rotation(const char *who, const cf_append_rotation *r, int dtype, int D)
{
    if (int rc = check_rotation(who, r->rotation, D)) return rc;
    if (!r->q && !r->q_out) return CF_OK;
    return check_turned(who, "q", D, dtype, dtype, r->n_q_heads, r->q, r->q_stride_tok, r->q_stride_head, r->q_out, r->q_out_stride_tok,
                        r->q_out_stride_head);
}

int check_append(const cf_kv_append_params *p, const char *who, bool eight_bits)
{
    if (p->n_kv_heads < 1 || p->n_kv_heads > 65535) return fail(CF_EINVAL, "%s: n_kv_heads %d must be from 1 to 65535", who, p->n_kv_heads);
    if (int rc = check_common(who, p->dtype, p->head_dim, p->n_tokens, p->n_seqs, p->cu_seqlens_q, p->kv_lens, p->block_table, p->table_stride,
                              p->pages_per_seq, p->page_size, p->n_pages))
        return rc;
    if (!p->k || !p->v || !p->k_pages || !p->v_pages) return fail(CF_EINVAL, "%s: NULL device pointer", who);
    if (int rc = check_strides(who, p->dtype, p->head_dim, {p->kv_stride_tok, p->kv_stride_head})) return rc;
    if (int rc = check_page_strides(who, p->dtype, p->head_dim, eight_bits, {p->page_stride, p->page_stride_tok, p->page_stride_head})) return rc;
    if (!aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->k_pages, 16) || !aligned(p->v_pages, 16))
        return fail(CF_EINVAL, "%s: k, v and pages must be 16-byte aligned", who);
    return CF_OK;
}

// The rows of workgroups of 256 lanes, a lane to a unit: as many as a launch holds?
int check_rows(const char *who, int n_tokens, int D)
{
    if (((int64_t)n_tokens * (D / 16) + 255) / 256 * 256 > 0xffffffffLL) return fail(CF_EINVAL, "%s: %d tokens are more than one launch holds", who, n_tokens);
    return CF_OK;
}

TurnArgs turn_args(const cf_rotation *r, int D, int n_tokens, int n_seqs, const int32_t *cu, const int32_t *lens)
{
    TurnArgs a{};
    if (r) a.inv_freq = r->inv_freq, a.rot = r->rot_dim, a.interleaved = r->interleaved != 0;
    a.units_shift = D == 64 ? 2 : 3;
    a.n_tokens = n_tokens, a.n_seqs = n_seqs, a.cu = cu, a.lens = lens;
    return a;
}
void queries_of(TurnArgs &a, const cf_append_rotation *r, int dtype)
{
    if (r && r->q)
        a.t[0] = TurnTensor{r->q, r->q_out, r->q_stride_tok, r->q_stride_head, r->q_out_stride_tok, r->q_out_stride_head, r->n_q_heads,
                            dtype == CF_FP32, dtype == CF_FP32, 1, 0, 0};
}
void pages_of(TurnArgs &a, const cf_kv_append_params *p)
{
    a.table = p->block_table, a.table_stride = p->table_stride, a.pages = p->pages_per_seq, a.n_pages = p->n_pages, a.page_stride = p->page_stride;
    a.shift = __builtin_ctz((unsigned)p->page_size);
}

// Heads of a group: the more, the fewer sines (one set a unit and group); the fewer, the more workgroups.  So many that `workgroups` are left, 16 at most, one
// in small calls (a trip to memory each, all at once).  us, 256 / 512 / 1024 / 2048 workgroups, 28 + 4 heads x 128 in bf16: 2000 rows there and back
// 16.9 / 15.6 / 21.9 / 21.9, 4000 rows 26.9 / 25.3 / 27.8 / 38.1, 2000 rows into pages 8.9 / 8.2 / 9.1 / 11.6; less than 1 % apart from 8192 rows there and back on.
// Stores go past the caches from 1024 blocks of rows and heads on (in the caches / past them: 2000 rows there and back 18.7 / 15.6, 4000 34.1 / 25.3, 8192 rows
// into pages 33.8 / 23.9; 250 rows 9.8 / 9.8: small results stay where the next call finds them).
void TurnArgs::group(int workgroups)
{
    int heads = 0;
    for (TurnTensor &x : t) heads += x.n_heads;
    const int64_t blocks = ((int64_t)n_tokens + (256 >> units_shift) - 1) / (256 >> units_shift);
    per_group = (int)std::min<int64_t>(16, std::max<int64_t>(1, blocks * heads / workgroups));
    for (TurnTensor &x : t) x.group(per_group);
    stream = blocks * heads >= 1024;
}

}  // namespace cf

extern "C" int cf_rotate(const cf_rotate_params *p, void *hip_stream)
{
    const char *who = "cf_rotate";
    if (!p) return cf::fail(CF_EINVAL, "%s: params is NULL", who);
    const int D = p->head_dim;
    if (D != 64 && D != 128) return cf::fail(CF_EUNSUPPORTED, "%s: head_dim %d not supported (64 or 128)", who, D);
    if (p->n_tokens < 1 || p->n_segments < 1 || p->n_segments > (1 << 30))
        return cf::fail(CF_EINVAL, "%s: need n_tokens >= 1 and 1 <= n_segments <= 2^30 (got %d, %d)", who, p->n_tokens, p->n_segments);
    if (p->inverse != 0 && p->inverse != 1) return cf::fail(CF_EINVAL, "%s: inverse must be 0 or 1 (got %d)", who, p->inverse);
    if (!p->cu_seqlens_q || !p->cu_seqlens_k || !cf::aligned(p->cu_seqlens_q, 4) || !cf::aligned(p->cu_seqlens_k, 4))
        return cf::fail(CF_EINVAL, "%s: NULL or misaligned list of segments", who);
    if (int rc = cf::check_rotation(who, p->rotation, D)) return rc;
    if (p->q.n_heads == 0 && p->k.n_heads == 0) return cf::fail(CF_EINVAL, "%s: neither q nor k", who);
    cf::TurnArgs a = cf::turn_args(&p->rotation, D, p->n_tokens, p->n_segments, p->cu_seqlens_q, p->cu_seqlens_k);
    a.chunk = 1, a.inverse = p->inverse;
    const cf_rotate_tensor *tensors[] = {&p->q, &p->k};
    for (int i = 0; i < 2; ++i) {
        const cf_rotate_tensor &t = *tensors[i];
        if (t.n_heads == 0) continue;
        if (int rc = cf::check_turned(who, i ? "k" : "q", D, t.dtype_in, t.dtype_out, t.n_heads, t.x, t.x_stride_tok, t.x_stride_head, t.y, t.y_stride_tok,
                                      t.y_stride_head))
            return rc;
        a.t[i] = cf::TurnTensor{t.x, t.y, t.x_stride_tok, t.x_stride_head, t.y_stride_tok, t.y_stride_head, t.n_heads, t.dtype_in == CF_FP32,
                                t.dtype_out == CF_FP32, 1, 0, 0};
    }
    if (int rc = cf::check_rows(who, p->n_tokens, D)) return rc;
    a.group(512);
    if (a.all_groups() > 65535) return cf::fail(CF_EINVAL, "%s: %d groups of heads are more than one launch holds", who, a.all_groups());
    const hipError_t e = cf::launch_turn_rows(a, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? CF_OK : cf::fail(CF_EHIP, "%s: %s", who, hipGetErrorString(e));
}

extern "C" int cf_kv_append_rotated(const cf_kv_append_params *p, const cf_append_rotation *r, void *hip_stream)
{
    const char *who = "cf_kv_append_rotated";
    if (!p || !r) return cf::fail(CF_EINVAL, "%s: params or rotation is NULL", who);
    if (int rc = cf::check_append(p, who, false)) return rc;
    if (int rc = cf::check_append_rotation(who, r, p->dtype, p->head_dim)) return rc;
    if (int rc = cf::check_rows(who, p->n_tokens, p->head_dim)) return rc;
    cf::TurnArgs a = cf::turn_args(&r->rotation, p->head_dim, p->n_tokens, p->n_seqs, p->cu_seqlens_q, p->kv_lens);
    cf::queries_of(a, r, p->dtype);
    cf::pages_of(a, p);
    const int fp32 = p->dtype == CF_FP32;
    a.t[1] = cf::TurnTensor{p->k, p->k_pages, p->kv_stride_tok, p->kv_stride_head, p->page_stride_tok, p->page_stride_head, p->n_kv_heads, fp32, fp32, 1, 1, 0};
    a.t[2] = cf::TurnTensor{p->v, p->v_pages, p->kv_stride_tok, p->kv_stride_head, p->page_stride_tok, p->page_stride_head, p->n_kv_heads, fp32, fp32, 0, 1, 0};
    a.group(512);
    if (a.all_groups() > 65535) return cf::fail(CF_EINVAL, "%s: %d groups of heads are more than one launch holds", who, a.all_groups());
    const hipError_t e = cf::launch_turn_rows(a, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? CF_OK : cf::fail(CF_EHIP, "%s: %s", who, hipGetErrorString(e));
}
