// C ABI of windowed attention: argument checks, kernel selection.
#include "checks.h"

// ---- a window and sinks -----------------------------------------------------------------------------------------
namespace {

// The window of a call, cut to its keys (a longer one hides nothing).
int check_window(const cf_attn_window *w, int32_t n_kv_tokens, const char *who, cf::WindowMask *mask)
{
    if (!w) return cf::fail(CF_EINVAL, "%s: window is NULL", who);
    if (w->window < 1 || w->n_sinks < 0)
        return cf::fail(CF_EINVAL, "%s: need window >= 1 and n_sinks >= 0 (got %d, %d)", who, w->window, w->n_sinks);
    *mask = {std::min(w->window, n_kv_tokens), std::min(w->n_sinks, n_kv_tokens)};
    return CF_OK;
}

// Kernels by the rules of the calls without a window; the backward's list is needed at either head_dim.
bool use_window_mfma(const cf_attn_fwd_params &p) { return mfma_shape(p) && p.softmax_scale > 0.f && narrow(p) && launchable_mfma(p, false); }
bool use_window_mfma(const cf_attn_bwd_params &b, const cf::WindowMask &mask)
{
    return use_window_mfma(b.f) && b.do_stride_tok < kMostStride && cf::window_launch_size(b.f, mask) <= cf::kMostWorkItems;
}
int64_t list_bytes(const cf_attn_fwd_params &p, const cf::WindowMask &mask) { return round_up(256 + cf::window_worklist_capacity(p, mask) * 16, 256); }
int64_t window_scratch(const cf_attn_fwd_params &p, const cf::WindowMask &mask)
{
    // (the scalar kernels' delta, whatever runs; behind it the list of the bf16 kernels and dQ's parts, or the sums of the fp32 one)
    return delta_bytes(p) + (mfma_shape(p) ? list_bytes(p, mask) + cf::window_dq_sums(p, mask) : p.dtype == CF_FP32 ? cf::window_f32_scratch(p, mask) : 0);
}

}  // namespace

extern "C" int cf_attn_window_fwd(const cf_attn_fwd_params *p, const cf_attn_window *w, void *hip_stream)
{
    const char *who = "cf_attn_window_fwd";
    cf::WindowMask mask;
    if (int rc = check_fwd(p, who, false)) return rc;
    if (int rc = check_window(w, p->n_kv_tokens, who, &mask)) return rc;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = use_window_mfma(*p) ? (cf::window_few(*p) ? cf::launch_window_few(*p, mask, s) : cf::launch_window_mfma_fwd(*p, mask, s))
                         : use_f32(*p)       ? cf::launch_window_f32_fwd(*p, mask, s)
                                             : cf::launch_window_simple_fwd(*p, mask, s);
    return e == hipSuccess ? CF_OK : hip_fail(who, e);
}

extern "C" int64_t cf_attn_window_bwd_workspace_bytes(const cf_attn_fwd_params *p, const cf_attn_window *w)
{
    const char *who = "cf_attn_window_bwd_workspace_bytes";
    cf::WindowMask mask;
    if (int rc = check_fwd(p, who, true)) return rc;
    if (p->flags & ~kKnownFlags) return cf::fail(CF_EINVAL, "%s: unknown flags 0x%x", who, p->flags);
    if (int rc = check_window(w, p->n_kv_tokens, who, &mask)) return rc;
    return window_scratch(*p, mask);
}

extern "C" int cf_attn_window_bwd(const cf_attn_bwd_params *b, const cf_attn_window *w, void *hip_stream)
{
    const char *who = "cf_attn_window_bwd";
    cf::WindowMask mask;
    if (int rc = check_bwd_tensors(b, who)) return rc;
    if (int rc = check_window(w, b->f.n_kv_tokens, who, &mask)) return rc;
    const int64_t need = window_scratch(b->f, mask);
    if (!b->workspace || !aligned(b->workspace, 256)) return cf::fail(CF_EINVAL, "%s: workspace must be non-NULL and 256-byte aligned", who);
    if (b->workspace_bytes < need)
        return cf::fail(CF_EINVAL, "%s: workspace has %lld bytes, %lld needed", who, (long long)b->workspace_bytes, (long long)need);
    cf::BwdWorkspace ws = {static_cast<float *>(b->workspace), nullptr, 0};
    if (mfma_shape(b->f)) {
        ws.worklist = reinterpret_cast<int *>(static_cast<char *>(b->workspace) + delta_bytes(b->f));
        ws.worklist_items = cf::window_worklist_capacity(b->f, mask);
    }
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = use_window_mfma(*b, mask) ? cf::launch_window_mfma_bwd(*b, ws, ws.delta + (delta_bytes(b->f) + list_bytes(b->f, mask)) / 4, mask, s)
                         : use_f32(*b)             ? cf::launch_window_f32_bwd(*b, ws.delta + delta_bytes(b->f) / 4, mask, s)
                                                   : cf::launch_window_simple_bwd(*b, ws, mask, s);
    return e == hipSuccess ? CF_OK : hip_fail(who, e);
}
