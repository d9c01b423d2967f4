// Attention of new tokens over a paged cache of 8 bits: entry points, scalar kernel (as that of attn_paged.hip; for calls that ask for it and those that
// the matrix kernels do not hold: 64 tokens behind up to 16384 keys, 32/8 heads x 128, take 7.3 ms with it).
#include <hip/hip_runtime.h>

#include "paged8.h"
#include "paged_checks.h"

namespace cf {
namespace {

constexpr int kWaves = 4;        // wavefronts per workgroup

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void paged8_rows_kernel(Paged8Args c)
{
    const PagedArgs &a = c.a;
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
    const RowSums<float, D> r = paged8_row<D, 0, 64>(c, table, position, h / (p.n_q_heads / p.n_kv_heads), tiles, 0, tiles.n, [&](int x) { return sq[wave][x]; });
    T *o = (T *)p.o + row * p.o_stride_tok + (int64_t)h * p.o_stride_head;
    const bool none = r.m == -INFINITY && r.z == 0.f;
    for (int t = 0; t < D / 64; ++t) st(o + lane + 64 * t, none ? 0.f : r.acc[t] / r.z);
    if (lane == 0 && p.lse) p.lse[(int64_t)h * p.n_tokens + row] = none ? -INFINITY : r.m + logf(r.z);
}

template <typename T, int D>
hipError_t run_rows(const Paged8Args &a, hipStream_t s)
{
    const dim3 grid((unsigned)(((int64_t)a.a.p.n_tokens + kWaves - 1) / kWaves), (unsigned)a.a.p.n_q_heads);
    paged8_rows_kernel<T, D><<<grid, kWaves * 64, 0, s>>>(a);
    return hipGetLastError();
}

// The matrix kernels' offsets inside a group of 16 keys have 32 bits, and a HIP launch holds fewer than 2^32 work-items.  (Wider rows and
// larger calls: a wavefront to a row.)
bool on_matrix_kernel(const PagedArgs &a)
{
    return !(a.p.flags & CF_FLAG_SCALAR_KERNELS) && a.p.kv_stride_tok < (1 << 25) && paged8_mfma_launch_size(a) <= 0xffffffffLL;
}
// Chooses the parts; bytes of workspace.
int64_t cut(PagedArgs &a)
{
    a.part_o = nullptr, a.part_ml = nullptr;
    cut_paged8_mfma(a);
    if (!on_matrix_kernel(a)) a.parts = 1;
    if (a.parts == 1) return 0;
    const int64_t rows = (int64_t)a.p.n_tokens * a.p.n_q_heads;
    return a.parts * rows * (a.p.head_dim * 4 + 8);
}

int check(const cf_attn_paged8_params *p, const char *who, bool sizes_only, Paged8Args *c)
{
    if (!p) return fail(CF_EINVAL, "%s: params is NULL", who);
    if (int rc = check_paged(&p->a, who, sizes_only, &c->a, true)) return rc;
    c->k_scales = p->k_scales, c->v_scales = p->v_scales, c->scale_page = p->scale_stride_page, c->scale_head = p->scale_stride_head;
    return sizes_only ? CF_OK : check_scales(who, p->k_scales, p->v_scales, p->scale_stride_page, p->scale_stride_head, p->a.page_size);
}

}  // namespace
}  // namespace cf

extern "C" int64_t cf_attn_paged8_workspace_bytes(const cf_attn_paged8_params *p)
{
    cf::Paged8Args c;
    if (int rc = cf::check(p, "cf_attn_paged8_workspace_bytes", true, &c)) return rc;
    return cf::cut(c.a);
}

extern "C" int cf_attn_paged8_fwd(const cf_attn_paged8_params *p8, void *hip_stream)
{
    const char *who = "cf_attn_paged8_fwd";
    cf::Paged8Args c;
    if (int rc = cf::check(p8, who, false, &c)) return rc;
    const cf_attn_paged_params *p = &p8->a;
    const int64_t need = cf::cut(c.a);
    if (int rc = cf::take_workspace(who, need, &c.a)) return rc;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    hipError_t e;
    if (cf::on_matrix_kernel(c.a)) e = cf::launch_paged8_mfma(c, s);
    else if (p->dtype == CF_FP32) e = p->head_dim == 64 ? cf::run_rows<float, 64>(c, s) : cf::run_rows<float, 128>(c, s);
    else e = p->head_dim == 64 ? cf::run_rows<unsigned short, 64>(c, s) : cf::run_rows<unsigned short, 128>(c, s);
    if (e == hipSuccess && c.a.parts > 1) e = cf::launch_paged_join(c.a, s);
    return e == hipSuccess ? CF_OK : cf::fail(CF_EHIP, "%s: %s", who, hipGetErrorString(e));
}
