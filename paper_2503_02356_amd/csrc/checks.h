// Argument checks and rules that the entry points share: what a call must hold, which kernels it runs on, what scratch it needs.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace {

constexpr int kKnownFlags = CF_FLAG_SCALAR_KERNELS | CF_FLAG_DKV_SINGLE_WRITER;

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_fwd(const cf_attn_fwd_params *p, const char *who, bool sizes_only)
{
    if (!p) return cf::fail(CF_EINVAL, "%s: params is NULL", who);
    if (p->dtype != CF_BF16 && p->dtype != CF_FP32)
        return cf::fail(CF_EUNSUPPORTED, "%s: dtype %d not supported", who, p->dtype);
    if (p->head_dim != 64 && p->head_dim != 128)
        return cf::fail(CF_EUNSUPPORTED, "%s: head_dim %d not supported (64 or 128)", who, p->head_dim);
    if (p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads != 0)
        return cf::fail(CF_EINVAL, "%s: n_q_heads %d must be a positive multiple of n_kv_heads %d", who,
                        p->n_q_heads, p->n_kv_heads);
    if (p->n_q_heads > 65535) return cf::fail(CF_EINVAL, "%s: n_q_heads %d > 65535", who, p->n_q_heads);
    if (p->n_tokens < 1 || p->n_segments < 1 || p->n_kv_tokens < p->n_tokens)
        return cf::fail(CF_EINVAL, "%s: need n_tokens >= 1, n_segments >= 1, n_kv_tokens >= n_tokens (got %d, %d, %d)",
                        who, p->n_tokens, p->n_segments, p->n_kv_tokens);
    if (p->n_segments > p->n_tokens)
        return cf::fail(CF_EINVAL, "%s: n_segments %d > n_tokens %d (empty segments are not allowed)", who,
                        p->n_segments, p->n_tokens);
    if (sizes_only) return CF_OK;
    if (p->flags & ~kKnownFlags) return cf::fail(CF_EINVAL, "%s: unknown flags 0x%x", who, p->flags);
    if (!p->cu_seqlens_q || !p->cu_seqlens_k || !p->q || !p->k || !p->v || !p->o || !p->lse)
        return cf::fail(CF_EINVAL, "%s: NULL device pointer", who);
    if (!(p->softmax_scale == p->softmax_scale))
        return cf::fail(CF_EINVAL, "%s: softmax_scale is NaN", who);
    const int64_t vec = p->dtype == CF_BF16 ? 8 : 4;  // elements per 16-byte access
    const int64_t D = p->head_dim;
    const int64_t strides[] = {p->q_stride_tok, p->q_stride_head, p->kv_stride_tok, p->kv_stride_head,
                               p->o_stride_tok, p->o_stride_head};
    for (int64_t s : strides)
        if (s < D || s % vec != 0)
            return cf::fail(CF_EINVAL, "%s: stride %lld must be >= head_dim and a multiple of %lld elements", who,
                            (long long)s, (long long)vec);
    if (!aligned(p->q, 16) || !aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->o, 16) ||
        !aligned(p->lse, 4) || !aligned(p->cu_seqlens_q, 4) || !aligned(p->cu_seqlens_k, 4))
        return cf::fail(CF_EINVAL, "%s: q, k, v, o must be 16-byte aligned", who);
    // the optional tile table: between ceil(T / 128) and T / 128 + n_segments records of 32 bytes
    if ((p->q_tiles == nullptr) != (p->n_q_tiles == 0) || p->n_q_tiles < 0 || !aligned(p->q_tiles, 16))
        return cf::fail(CF_EINVAL, "%s: q_tiles / n_q_tiles = %d do not go together (NULL with 0, 16-byte aligned)", who,
                        p->n_q_tiles);
    if (p->q_tiles && (p->n_q_tiles < (p->n_tokens + 127) / 128 || p->n_q_tiles > p->n_tokens / 128 + p->n_segments))
        return cf::fail(CF_EINVAL, "%s: n_q_tiles = %d cannot be the tile count of %d tokens in %d segments", who,
                        p->n_q_tiles, p->n_tokens, p->n_segments);
    return CF_OK;
}

// Shapes the MFMA kernels cover (decides the workspace size, so it may only look at sizes, dtype, flags).
bool mfma_shape(const cf_attn_fwd_params &p)
{
    return p.dtype == CF_BF16 && !(p.flags & CF_FLAG_SCALAR_KERNELS);
}
// The matrix kernels address the rows of a block with 32-bit byte offsets: 63 rows x 2 bytes (bf16) and 31 rows x 4 bytes
// (fp32) of this many elements stay below 2^32.  Wider strides go to the scalar kernels.
constexpr int64_t kMostStride = 1 << 25;
bool narrow(const cf_attn_fwd_params &p) { return p.q_stride_tok < kMostStride && p.kv_stride_tok < kMostStride; }
// Their launches give every segment workgroups of its own: hundreds of thousands of segments can be more than one launch
// holds, and go to the scalar kernels (a row per wavefront).  (bf16 at head_dim 128 never had that way out.)
bool launchable_mfma(const cf_attn_fwd_params &p, bool backward)
{
    return p.head_dim == 128 || cf::mfma_launch_size(p, backward) <= cf::kMostWorkItems;
}
bool launchable_f32(const cf_attn_fwd_params &p, bool backward) { return cf::f32_launch_size(p, backward) <= cf::kMostWorkItems; }

// The MFMA kernels take the row maximum before scaling, which needs a positive scale.
bool use_mfma(const cf_attn_fwd_params &p) { return mfma_shape(p) && p.softmax_scale > 0.f && narrow(p) && launchable_mfma(p, false); }
bool use_mfma(const cf_attn_bwd_params &b) { return use_mfma(b.f) && b.do_stride_tok < kMostStride && launchable_mfma(b.f, true); }

// The fp32 matrix kernels: every fp32 shape, any scale.
bool use_f32(const cf_attn_fwd_params &p) { return p.dtype == CF_FP32 && !(p.flags & CF_FLAG_SCALAR_KERNELS) && narrow(p) && launchable_f32(p, false); }
bool use_f32(const cf_attn_bwd_params &b) { return use_f32(b.f) && b.do_stride_tok < kMostStride && launchable_f32(b.f, true); }

int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

int64_t delta_bytes(const cf_attn_fwd_params &p) { return round_up((int64_t)p.n_q_heads * p.n_tokens * 4, 256); }
// counters (256 bytes) + 16-byte items; head_dim 64 has no work list
bool has_worklist(const cf_attn_fwd_params &p) { return mfma_shape(p) && p.head_dim == 128; }
int64_t worklist_bytes(const cf_attn_fwd_params &p) { return has_worklist(p) ? 256 + cf::dkv_worklist_capacity(p) * 16 : 0; }
// The least scratch a backward runs in: with room for the coarse list only, its work is cut less finely.
int64_t least_scratch(const cf_attn_fwd_params &p) { return delta_bytes(p) + (has_worklist(p) ? 256 + cf::dkv_worklist_least(p) * 16 : 0); }

int hip_fail(const char *who, hipError_t e)
{
    return cf::fail(CF_EHIP, "%s: %s", who, hipGetErrorString(e));
}

// Argument checks of one backward call apart from its scratch memory.
int check_bwd_tensors(const cf_attn_bwd_params *b, const char *who)
{
    if (!b) return cf::fail(CF_EINVAL, "%s: params is NULL", who);
    if (int rc = check_fwd(&b->f, who, false)) return rc;
    const cf_attn_fwd_params &p = b->f;
    if (!b->d_o || !b->d_q || !b->d_k || !b->d_v)
        return cf::fail(CF_EINVAL, "%s: NULL device pointer", who);
    const int64_t vec = p.dtype == CF_BF16 ? 8 : 4, D = p.head_dim;
    const int64_t strides[] = {b->do_stride_tok, b->do_stride_head, b->dq_stride_tok, b->dq_stride_head};
    for (int64_t s : strides)
        if (s < D || s % vec != 0)
            return cf::fail(CF_EINVAL, "%s: stride %lld must be >= head_dim and a multiple of %lld elements", who,
                            (long long)s, (long long)vec);
    if (b->dkv_stride_tok < D || b->dkv_stride_head < D || b->dkv_stride_tok % 4 || b->dkv_stride_head % 4)
        return cf::fail(CF_EINVAL, "%s: d_k/d_v strides must be >= head_dim and multiples of 4 elements", who);
    if (!aligned(b->d_o, 16) || !aligned(b->d_q, 16) || !aligned(b->d_k, 16) || !aligned(b->d_v, 16))
        return cf::fail(CF_EINVAL, "%s: d_o, d_q, d_k, d_v must be 16-byte aligned", who);
    return CF_OK;
}

}  // namespace
