// Plain scalar kernels of windowed attention for one chunk: fp32 arithmetic, fp32 or bf16 storage, one wavefront per query row
// (forward, dQ) or per key row (dK/dV), pairs one by one; only visible keys are read.  They serve the cross-check flag and what the
// matrix kernels do not cover, as attn_simple.hip does for the causal mask.
//   visible(i, j): j <= p and (j > p - window or j < sinks), p the position of query i;  S = scale * q.k;  P = exp(S - LSE);
//   O = sum_j P v_j;  dV_j += sum_i P dO_i;  delta = sum_j P dP;  dS = P (dO_i.v_j - delta_i);
//   dQ_i = scale sum_j dS k_j;  dK_j += scale sum_i dS q_i.
// What bounds them: a pair is 2 D FMAs on 64 lanes that re-read the key row for every query row and head (2048 rows packed around 300, 8/2 heads,
// D = 128, window 128: forward 125 us, backward 1.39 ms in bf16, 215 us and 1.80 ms in fp32).
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "scalar_rows.h"

namespace cf {
namespace {

constexpr int kWaves = kScalarWaves;

template <typename T, int D>
__device__ inline void keep_row(const T *row, float *kept)
{
    const int lane = threadIdx.x & 63;
    for (int t = 0; t < D / 64; ++t) kept[lane + 64 * t] = ld(row + lane + 64 * t);
}

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void window_fwd_kernel(cf_attn_fwd_params p, WindowMask mask)
{
    __shared__ float sq[kWaves][D];
    const int wave = threadIdx.x >> 6, row = blockIdx.x * kWaves + wave, h = blockIdx.y;
    if (row >= p.n_tokens) return;                   // whole wavefront leaves together; no barrier below
    keep_row<T, D>(row_of<T>(p.q, row, p.q_stride_tok, h, p.q_stride_head), sq[wave]);
    __builtin_amdgcn_wave_barrier();
    scalar_fwd_row<T, D, 0>(p, segment_of_query(p, row), row, h, [&](int x) { return sq[wave][x]; }, mask);
}

// delta of a row: <dO, O>; where the row sees at most 64 keys sum_j P_j dP_j, since the rounding of a stored O would be the largest
// error of its gradients.
template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void window_delta_kernel(cf_attn_bwd_params b, float *delta, WindowMask mask)
{
    const cf_attn_fwd_params &p = b.f;
    __shared__ float sq[kWaves][D], sdo[kWaves][D];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, row = blockIdx.x * kWaves + wave, h = blockIdx.y;
    if (row >= p.n_tokens) return;
    const SegmentRows g = segment_of_query(p, row);
    const int kh = h / (p.n_q_heads / p.n_kv_heads);
    const KeysOfRow<WindowMask> keys(mask, g.lk - g.lq + (row - g.q0));
    keep_row<T, D>(row_of<T>(p.q, row, p.q_stride_tok, h, p.q_stride_head), sq[wave]);
    keep_row<T, D>(row_of<T>(b.d_o, row, b.do_stride_tok, h, b.do_stride_head), sdo[wave]);
    __builtin_amdgcn_wave_barrier();
    float s = 0.f;
    if (keys.n > 64) {
        const T *o = row_of<T>(p.o, row, p.o_stride_tok, h, p.o_stride_head);
        for (int t = 0; t < D / 64; ++t) s += ld(o + lane + 64 * t) * sdo[wave][lane + 64 * t];
    } else if (lane < keys.n) {
        const T *k = row_of<T>(p.k, g.k0 + keys.key(lane), p.kv_stride_tok, kh, p.kv_stride_head);
        const T *v = row_of<T>(p.v, g.k0 + keys.key(lane), p.kv_stride_tok, kh, p.kv_stride_head);
        float sc = 0.f, dp = 0.f;
        for (int x = 0; x < D; ++x) {
            sc += sq[wave][x] * ld(k + x);
            dp += sdo[wave][x] * ld(v + x);
        }
        s = expf(sc * p.softmax_scale - p.lse[(int64_t)h * p.n_tokens + row]) * dp;
    }
    s = wave_sum(s);
    if (lane == 0) delta[(int64_t)h * p.n_tokens + row] = s;
}

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void window_dq_kernel(cf_attn_bwd_params b, const float *delta, WindowMask mask)
{
    const cf_attn_fwd_params &p = b.f;
    __shared__ float sq[kWaves][D], sdo[kWaves][D];
    const int wave = threadIdx.x >> 6, row = blockIdx.x * kWaves + wave, h = blockIdx.y;
    if (row >= p.n_tokens) return;
    keep_row<T, D>(row_of<T>(p.q, row, p.q_stride_tok, h, p.q_stride_head), sq[wave]);
    keep_row<T, D>(row_of<T>(b.d_o, row, b.do_stride_tok, h, b.do_stride_head), sdo[wave]);
    __builtin_amdgcn_wave_barrier();
    scalar_dq_row<T, D, 0>(b, segment_of_query(p, row), row, h, [&](int x) { return sq[wave][x]; }, [&](int x) { return sdo[wave][x]; },
                           delta[(int64_t)h * p.n_tokens + row], mask);
}

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void window_dkv_kernel(cf_attn_bwd_params b, const float *delta, WindowMask mask)
{
    const cf_attn_fwd_params &p = b.f;
    __shared__ float sk[kWaves][D], sv[kWaves][D];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, krow = blockIdx.x * kWaves + wave, kh = blockIdx.y;
    if (krow >= p.n_kv_tokens) return;
    const SegmentRows g = segment_rows(p, find_segment(p.cu_seqlens_k, p.n_segments, krow));
    const int j = krow - g.k0, prefix = g.lk - g.lq;
    if (rows_that_see(mask, j, prefix, g.lq) <= (j > prefix ? j - prefix : 0)) return;      // no row sees it: its gradients stay
    keep_row<T, D>(row_of<T>(p.k, krow, p.kv_stride_tok, kh, p.kv_stride_head), sk[wave]);
    keep_row<T, D>(row_of<T>(p.v, krow, p.kv_stride_tok, kh, p.kv_stride_head), sv[wave]);
    __builtin_amdgcn_wave_barrier();
    float dk[D / 64], dv[D / 64];
    scalar_dkv_row<T, D, 0>(b, g, krow, kh, [&](int x) { return sk[wave][x]; }, [&](int x) { return sv[wave][x]; },
                            [&](int row, int h) { return delta[(int64_t)h * p.n_tokens + row]; }, dk, dv, mask);
    float *gk = b.d_k + (int64_t)krow * b.dkv_stride_tok + (int64_t)kh * b.dkv_stride_head;
    float *gv = b.d_v + (int64_t)krow * b.dkv_stride_tok + (int64_t)kh * b.dkv_stride_head;
    for (int t = 0; t < D / 64; ++t) {
        gk[lane + 64 * t] += dk[t] * p.softmax_scale;
        gv[lane + 64 * t] += dv[t];
    }
}

template <typename T, int D>
hipError_t run_fwd(const cf_attn_fwd_params &p, const WindowMask &mask, hipStream_t s)
{
    window_fwd_kernel<T, D><<<dim3((p.n_tokens + kWaves - 1) / kWaves, p.n_q_heads), kWaves * 64, 0, s>>>(p, mask);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t run_bwd(const cf_attn_bwd_params &b, const BwdWorkspace &ws, const WindowMask &mask, hipStream_t s)
{
    const cf_attn_fwd_params &p = b.f;
    const dim3 rows((p.n_tokens + kWaves - 1) / kWaves, p.n_q_heads), keys((p.n_kv_tokens + kWaves - 1) / kWaves, p.n_kv_heads);
    window_delta_kernel<T, D><<<rows, kWaves * 64, 0, s>>>(b, ws.delta, mask);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    window_dq_kernel<T, D><<<rows, kWaves * 64, 0, s>>>(b, ws.delta, mask);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    window_dkv_kernel<T, D><<<keys, kWaves * 64, 0, s>>>(b, ws.delta, mask);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_window_simple_fwd(const cf_attn_fwd_params &p, const WindowMask &mask, hipStream_t s)
{
    if (p.dtype == CF_FP32) return p.head_dim == 64 ? run_fwd<float, 64>(p, mask, s) : run_fwd<float, 128>(p, mask, s);
    return p.head_dim == 64 ? run_fwd<unsigned short, 64>(p, mask, s) : run_fwd<unsigned short, 128>(p, mask, s);
}
hipError_t launch_window_simple_bwd(const cf_attn_bwd_params &b, const BwdWorkspace &ws, const WindowMask &mask, hipStream_t s)
{
    if (b.f.dtype == CF_FP32) return b.f.head_dim == 64 ? run_bwd<float, 64>(b, ws, mask, s) : run_bwd<float, 128>(b, ws, mask, s);
    return b.f.head_dim == 64 ? run_bwd<unsigned short, 64>(b, ws, mask, s) : run_bwd<unsigned short, 128>(b, ws, mask, s);
}

}  // namespace cf
