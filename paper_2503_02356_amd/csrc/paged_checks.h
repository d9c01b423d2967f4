// Argument checks that the calls on paged caches share.
#pragma once
#include <algorithm>
#include <initializer_list>

#include "common.h"
#include "paged.h"

namespace cf {
namespace {

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

int check_multiples(const char *who, int D, int64_t vec, std::initializer_list<int64_t> strides)
{
    for (int64_t s : strides)
        if (s < D || s % vec != 0)
            return fail(CF_EINVAL, "%s: stride %lld must be >= head_dim and a multiple of %lld elements", who, (long long)s, (long long)vec);
    return CF_OK;
}
int check_strides(const char *who, int dtype, int D, std::initializer_list<int64_t> strides)
{
    return check_multiples(who, D, dtype == CF_BF16 ? 8 : 4, strides);
}
int check_page_strides(const char *who, int dtype, int D, bool eight_bits, std::initializer_list<int64_t> strides)
{
    return eight_bits ? check_multiples(who, D, 16, strides) : check_strides(who, dtype, D, strides);
}

// eight_bits: pages of bytes (strides of 16 of them), not of p's dtype.
int check_paged(const cf_attn_paged_params *p, const char *who, bool sizes_only, PagedArgs *a, bool eight_bits = false)
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
    if (int rc = check_strides(who, p->dtype, p->head_dim, {p->q_stride_tok, p->q_stride_head, p->o_stride_tok, p->o_stride_head})) return rc;
    if (int rc = check_page_strides(who, p->dtype, p->head_dim, eight_bits, {p->page_stride, p->kv_stride_tok, p->kv_stride_head})) return rc;
    if (!aligned(p->q, 16) || !aligned(p->k_pages, 16) || !aligned(p->v_pages, 16) || !aligned(p->o, 16) || !aligned(p->lse, 4))
        return fail(CF_EINVAL, "%s: q, pages and o must be 16-byte aligned", who);
    return CF_OK;
}

// Lays the parts' results out in the call's workspace, of which `need` bytes are needed.
int take_workspace(const char *who, int64_t need, PagedArgs *a)
{
    const cf_attn_paged_params &p = a->p;
    if (need == 0) return CF_OK;
    if (!p.workspace || !aligned(p.workspace, 256)) return fail(CF_EINVAL, "%s: workspace must be non-NULL and 256-byte aligned", who);
    if (p.workspace_bytes < need)
        return fail(CF_EINVAL, "%s: workspace has %lld bytes, %lld needed", who, (long long)p.workspace_bytes, (long long)need);
    a->part_o = static_cast<float *>(p.workspace);
    a->part_ml = reinterpret_cast<float2 *>(a->part_o + (int64_t)a->parts * p.n_tokens * p.n_q_heads * p.head_dim);
    return CF_OK;
}

// Scales of a cache of 8 bits.
int check_scales(const char *who, const void *k, const void *v, int64_t stride_page, int64_t stride_head, int page_size)
{
    if (!k || !v || !aligned(k, 4) || !aligned(v, 4)) return fail(CF_EINVAL, "%s: scales must be device pointers to floats", who);
    if (stride_page < page_size / CF_KV8_BLOCK || stride_head < page_size / CF_KV8_BLOCK)
        return fail(CF_EINVAL, "%s: strides of the scales (%lld, %lld) must be at least page_size / %d", who, (long long)stride_page, (long long)stride_head,
                    CF_KV8_BLOCK);
    return CF_OK;
}

}  // namespace
}  // namespace cf
