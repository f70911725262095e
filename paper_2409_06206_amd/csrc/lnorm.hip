// LayerNorm of rows, forward and backward (lnorm.h): the kernels and the C ABI.
#include "../../include/lnorm.h"
#include "args.h"
#include "common.h"
#include "mfma.h"
#include "profile.h"

namespace gswa {
namespace {

constexpr int kThreads = 256;
constexpr int kSlices = 64; // of the rows, in the sums of the parameter gradients

struct Args {
    const void *x, *residual, *gamma, *beta, *dy, *dsum;
    void *y, *sum, *dx;
    float2 *stats;  // backward: mean and 1 / sqrt(var + eps) of every row
    float *part;    // backward: [kSlices][2 C]
    float *dgamma, *dbeta;
    long rows, ldx, ldy, ldr;
    int C, accumulate;
    float eps;
};

__device__ __forceinline__ float block_sum(float v, float *lds)
{
#pragma unroll
    for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// mean and 1 / sqrt(var + eps) of a row: the squares are of distances from the mean, in a second pass
template <typename T> __device__ __forceinline__ float2 row_stats(const T *row, int C, float eps, float *lds)
{
    float s = 0.f, q = 0.f;
    for (int c = threadIdx.x; c < C; c += kThreads) s += to_f32(row[c]);
    const float mean = block_sum(s, lds) / (float)C;
    for (int c = threadIdx.x; c < C; c += kThreads) {
        const float d = to_f32(row[c]) - mean;
        q += d * d;
    }
    return make_float2(mean, rsqrtf(block_sum(q, lds) / (float)C + eps));
}

// One workgroup per row; a row is read again from the caches for each pass over it.
template <typename T> __global__ __launch_bounds__(kThreads) void lnorm_fwd_kernel(Args a)
{
    __shared__ float lds[4];
    const T *gamma = static_cast<const T *>(a.gamma), *beta = static_cast<const T *>(a.beta);
    for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *u = static_cast<const T *>(a.x) + row * a.ldx;
        if (a.residual) {
            const T *r = static_cast<const T *>(a.residual) + row * a.ldr;
            T *s = static_cast<T *>(a.sum) + row * a.ldr;
            for (int c = threadIdx.x; c < a.C; c += kThreads) from_f32(s[c], to_f32(u[c]) + to_f32(r[c]));
            u = s; // (every thread reads back only what it wrote)
        }
        const float2 st = row_stats(u, a.C, a.eps, lds);
        T *y = static_cast<T *>(a.y) + row * a.ldy;
        for (int c = threadIdx.x; c < a.C; c += kThreads)
            from_f32(y[c], (to_f32(u[c]) - st.x) * st.y * (gamma ? to_f32(gamma[c]) : 1.f) + (beta ? to_f32(beta[c]) : 0.f));
    }
}

template <typename T> __global__ __launch_bounds__(kThreads) void lnorm_stats_kernel(Args a)
{
    __shared__ float lds[4];
    for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float2 st = row_stats(static_cast<const T *>(a.x) + row * a.ldx, a.C, a.eps, lds);
        if (threadIdx.x == 0) a.stats[row] = st;
    }
}

template <typename T> __global__ __launch_bounds__(kThreads) void lnorm_bwd_kernel(Args a)
{
    __shared__ float lds[4];
    const T *gamma = static_cast<const T *>(a.gamma);
    for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *u = static_cast<const T *>(a.x) + row * a.ldx, *dy = static_cast<const T *>(a.dy) + row * a.ldy;
        const float2 st = row_stats(u, a.C, a.eps, lds);
        float sg = 0.f, sgx = 0.f;
        for (int c = threadIdx.x; c < a.C; c += kThreads) {
            const float g = to_f32(dy[c]) * (gamma ? to_f32(gamma[c]) : 1.f);
            sg += g;
            sgx += g * ((to_f32(u[c]) - st.x) * st.y);
        }
        sg = block_sum(sg, lds) / (float)a.C;
        sgx = block_sum(sgx, lds) / (float)a.C;
        T *dx = static_cast<T *>(a.dx) + row * a.ldr;
        const T *ds = a.dsum ? static_cast<const T *>(a.dsum) + row * a.ldr : nullptr;
        for (int c = threadIdx.x; c < a.C; c += kThreads) {
            const float g = to_f32(dy[c]) * (gamma ? to_f32(gamma[c]) : 1.f);
            from_f32(dx[c], (g - sg - (to_f32(u[c]) - st.x) * st.y * sgx) * st.y + (ds ? to_f32(ds[c]) : 0.f));
        }
    }
}

// partial sums of dy * xh and dy over a slice of the rows, a thread per column
template <typename T> __global__ __launch_bounds__(kThreads) void lnorm_wgrad_kernel(Args a)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.C) return;
    float dg = 0.f, db = 0.f;
    for (long row = blockIdx.y; row < a.rows; row += kSlices) {
        const float2 st = a.stats[row];
        const float d = to_f32(static_cast<const T *>(a.dy)[row * a.ldy + c]);
        dg += d * ((to_f32(static_cast<const T *>(a.x)[row * a.ldx + c]) - st.x) * st.y);
        db += d;
    }
    float *part = a.part + (size_t)blockIdx.y * 2 * a.C;
    part[c] = dg;
    part[a.C + c] = db;
}

__global__ __launch_bounds__(kThreads) void lnorm_sum_kernel(Args a)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= 2 * a.C) return;
    float s = 0.f;
    for (int i = 0; i < kSlices; ++i) s += a.part[(size_t)i * 2 * a.C + c];
    float *out = c < a.C ? a.dgamma + c : a.dbeta + (c - a.C);
    *out = a.accumulate ? *out + s : s;
}

struct Plan {
    size_t elem, stats, part;
    long ldx, ldy, ldr;
};

int make_plan(const lnorm_desc *d, Plan *p)
{
    if (!d) return GSWA_EINVAL;
    if (d->rows <= 0 || d->C <= 0 || (d->dtype != GSWA_F32 && d->dtype != GSWA_BF16)) return GSWA_EINVAL;
    if (!(d->eps >= 0.f) || (d->flags & ~(uint32_t)LNORM_ACCUM_WGRAD)) return GSWA_EINVAL;
    p->ldx = d->x_stride ? d->x_stride : d->C;
    p->ldy = d->y_stride ? d->y_stride : d->C;
    p->ldr = d->r_stride ? d->r_stride : d->C;
    if (p->ldx < d->C || p->ldy < d->C || p->ldr < d->C) return GSWA_EINVAL;
    p->elem = d->dtype == GSWA_F32 ? 4 : 2;
    if (d->C > (int)(65536 / p->elem)) return GSWA_EUNSUPPORTED;
    const long widest = p->ldx > p->ldy ? (p->ldx > p->ldr ? p->ldx : p->ldr) : (p->ldy > p->ldr ? p->ldy : p->ldr);
    if (d->rows > (1L << 40) / widest) return GSWA_EUNSUPPORTED;
    p->stats = to_256((size_t)d->rows * sizeof(float2));
    p->part = to_256((size_t)kSlices * 2 * d->C * sizeof(float));
    return GSWA_OK;
}

// bytes from the first row's first value to the last row's last one
size_t span(const lnorm_desc *d, const Plan &p, long ld) { return ((size_t)(d->rows - 1) * ld + d->C) * p.elem; }

unsigned row_blocks(long rows) { return (unsigned)(rows < 65536 ? rows : 65536); }

} // namespace
} // namespace gswa

using namespace gswa;

#define LN_LAUNCHED()                                             \
    do {                                                          \
        const hipError_t e_ = hipGetLastError();                  \
        if (e_ != hipSuccess) return report_hip_error(e_);        \
    } while (0)

extern "C" {

int lnorm_query_bytes(const lnorm_desc *desc, size_t *bwd_ws_bytes)
{
    Plan p;
    const int rc = make_plan(desc, &p);
    if (rc != GSWA_OK) return rc;
    if (bwd_ws_bytes) *bwd_ws_bytes = p.stats + p.part;
    return GSWA_OK;
}

int lnorm_forward(const lnorm_desc *desc, const void *x, const void *residual, const void *gamma, const void *beta,
                  void *y, void *sum, void *hip_stream)
{
    Plan p;
    const int rc = make_plan(desc, &p);
    if (rc != GSWA_OK) return rc;
    if (!x || !y || !residual != !sum || !aligned_to(16, x, residual, gamma, beta, y, sum)) return GSWA_EINVAL;
    const size_t row = (size_t)desc->C * p.elem;
    const Range rx(x, span(desc, p, p.ldx)), rr(residual, span(desc, p, p.ldr)), rg(gamma, row), rb(beta, row),
        ry(y, span(desc, p, p.ldy)), rs(sum, span(desc, p, p.ldr));
    if (overlaps_any(ry, rx, rr, rg, rb, rs) || overlaps_any(rs, rg, rb)) return GSWA_EINVAL;
    if (overlaps_any(rs, rx) && !(sum == x && p.ldx == p.ldr)) return GSWA_EINVAL;
    if (overlaps_any(rs, rr) && sum != residual) return GSWA_EINVAL;
    Args a{};
    a.x = x; a.residual = residual; a.gamma = gamma; a.beta = beta; a.y = y; a.sum = sum;
    a.rows = desc->rows; a.ldx = p.ldx; a.ldy = p.ldy; a.ldr = p.ldr; a.C = desc->C; a.eps = desc->eps;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    KernelTimer t(K_LNORM_FWD, st);
    if (desc->dtype == GSWA_F32) hipLaunchKernelGGL(lnorm_fwd_kernel<float>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL(lnorm_fwd_kernel<bf16_t>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, st, a);
    LN_LAUNCHED();
    return GSWA_OK;
}

int lnorm_backward(const lnorm_desc *desc, const void *x, const void *dy, const void *gamma, const void *dsum,
                   void *dx, float *dgamma, float *dbeta, void *ws, void *hip_stream)
{
    Plan p;
    const int rc = make_plan(desc, &p);
    if (rc != GSWA_OK) return rc;
    if (!x || !dy || !dx || !dgamma != !dbeta || (dgamma && !ws)) return GSWA_EINVAL;
    if (!aligned_to(16, x, dy, gamma, dsum, dx, dgamma, dbeta) || !aligned_to(256, ws)) return GSWA_EINVAL;
    const size_t row = (size_t)desc->C * p.elem, vec = (size_t)desc->C * sizeof(float);
    const Range rx(x, span(desc, p, p.ldx)), ry(dy, span(desc, p, p.ldy)), rg(gamma, row), rs(dsum, span(desc, p, p.ldr)),
        rd(dx, span(desc, p, p.ldr)), wg(dgamma, vec), wb(dbeta, vec), rw(dgamma ? ws : nullptr, p.stats + p.part);
    if (overlaps_any(rd, rx, rg, wg, wb, rw) || overlaps_any(wg, rx, ry, rg, rs, wb, rw) ||
        overlaps_any(wb, rx, ry, rg, rs, rw) || overlaps_any(rw, rx, ry, rg, rs))
        return GSWA_EINVAL;
    if (overlaps_any(rd, ry) && !(dx == dy && p.ldy == p.ldr)) return GSWA_EINVAL;
    if (overlaps_any(rd, rs) && dx != dsum) return GSWA_EINVAL;
    Args a{};
    a.x = x; a.dy = dy; a.gamma = gamma; a.dsum = dsum; a.dx = dx; a.dgamma = dgamma; a.dbeta = dbeta;
    a.rows = desc->rows; a.ldx = p.ldx; a.ldy = p.ldy; a.ldr = p.ldr; a.C = desc->C; a.eps = desc->eps;
    a.accumulate = (desc->flags & LNORM_ACCUM_WGRAD) != 0;
    if (dgamma) {
        a.stats = static_cast<float2 *>(ws);
        a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + p.stats);
    }
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool f32 = desc->dtype == GSWA_F32;
    // (dx may go over dy: the parameter gradients come first)
    if (dgamma) {
        const dim3 cols((desc->C + kThreads - 1) / kThreads, kSlices), both((2 * desc->C + kThreads - 1) / kThreads);
        KernelTimer t(K_LNORM_SUM, st);
        if (f32) hipLaunchKernelGGL(lnorm_stats_kernel<float>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL(lnorm_stats_kernel<bf16_t>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, st, a);
        LN_LAUNCHED();
        if (f32) hipLaunchKernelGGL(lnorm_wgrad_kernel<float>, cols, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL(lnorm_wgrad_kernel<bf16_t>, cols, dim3(kThreads), 0, st, a);
        LN_LAUNCHED();
        hipLaunchKernelGGL(lnorm_sum_kernel, both, dim3(kThreads), 0, st, a);
        LN_LAUNCHED();
    }
    KernelTimer t(K_LNORM_BWD, st);
    if (f32) hipLaunchKernelGGL(lnorm_bwd_kernel<float>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL(lnorm_bwd_kernel<bf16_t>, dim3(row_blocks(a.rows)), dim3(kThreads), 0, st, a);
    LN_LAUNCHED();
    return GSWA_OK;
}

} // extern "C"
