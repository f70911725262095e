// Learned relative position bias by buckets of offsets, with its gradient (relpos.h): the kernels and the C ABI.
#include "../../include/relpos.h"
#include "args.h"
#include "common.h"
#include "profile.h"

#include <math.h>
#include <vector>

namespace gswa {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 64; // rows of a gradient (one image and head) that one workgroup sums

struct Args {
    const void *table, *dout;
    void *out;
    float *dtable, *part; // part: [heads][slices][buckets]
    long ld, slices;
    int heads, batch, q, k, start, window, buckets, bidirectional, causal, accumulate, n;
    int edges[RELPOS_MAX_EDGES];
};

// edges <= d
__device__ __forceinline__ int edges_up_to(const Args &a, int d)
{
    int lo = 0, hi = a.n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.edges[mid] <= d) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// bucket of r = key - query
__device__ __forceinline__ int bucket_of(const Args &a, int r)
{
    if (!a.bidirectional) return edges_up_to(a, r < 0 ? -r : 0);
    return edges_up_to(a, r < 0 ? -r : r) + (r > 0 ? a.n + 1 : 0);
}

__device__ __forceinline__ int window_bucket(const Args &a, int offset)
{
    const int side = 2 * a.window - 1;
    const int dr = offset / side - (a.window - 1), dc = offset % side - (a.window - 1);
    return bucket_of(a, -dr) * 2 * (a.n + 1) + bucket_of(a, -dc);
}

template <typename T> __global__ __launch_bounds__(kThreads) void window_fwd_kernel(Args a)
{
    const int side = 2 * a.window - 1, total = side * side * a.heads;
    const int e = blockIdx.x * kThreads + threadIdx.x;
    if (e >= total) return;
    const int offset = e / a.heads, h = e - offset * a.heads;
    static_cast<T *>(a.out)[e] = static_cast<const T *>(a.table)[(long)window_bucket(a, offset) * a.heads + h];
}

// a thread per learned value goes over the offsets of its pair of buckets
__global__ __launch_bounds__(kThreads) void window_bwd_kernel(Args a)
{
    const int side = 2 * a.window - 1;
    const int e = blockIdx.x * kThreads + threadIdx.x;
    if (e >= a.buckets * a.heads) return;
    const int b = e / a.heads, h = e - b * a.heads;
    float s = 0.f;
    for (int o = 0; o < side * side; ++o)
        if (window_bucket(a, o) == b) s += static_cast<const float *>(a.dout)[(long)o * a.heads + h];
    a.dtable[e] = a.accumulate ? a.dtable[e] + s : s;
}

template <typename T> __global__ __launch_bounds__(kThreads) void sequence_fwd_kernel(Args a)
{
    const int h = blockIdx.y;
    for (int i = blockIdx.x; i < a.q; i += gridDim.x) {
        T *row = static_cast<T *>(a.out) + ((long)h * a.q + i) * a.ld;
        for (int j = threadIdx.x; j < a.k; j += kThreads) {
            const int r = j - i - a.start;
            if (a.causal && r > 0) from_f32(row[j], -INFINITY);
            else row[j] = static_cast<const T *>(a.table)[(long)bucket_of(a, r) * a.heads + h];
        }
    }
}

// A workgroup sums kRows rows of one image and head.  A thread walks down a diagonal (key - query = const, one bucket), neighbours next to
// each other in every row; 256 diagonals at a time go to LDS, where a thread per bucket adds those of its bucket in their order.
template <typename T> __global__ __launch_bounds__(kThreads) void sequence_bwd_kernel(Args a)
{
    __shared__ float sums[kThreads];
    __shared__ int of[kThreads];
    const int h = blockIdx.y;
    const int slices_q = (a.q + kRows - 1) / kRows;
    for (long slice = blockIdx.x; slice < a.slices; slice += gridDim.x) {
        const int b = (int)(slice / slices_q), i0 = (int)(slice % slices_q) * kRows, i1 = i0 + kRows < a.q ? i0 + kRows : a.q;
        const T *d = static_cast<const T *>(a.dout) + ((long)b * a.heads + h) * a.q * a.ld;
        // the diagonals that meet these rows: from the last row's first key to the first row's last one (or to the query itself)
        const int first = -(i1 - 1), last = a.causal && a.start < a.k - 1 - i0 ? a.start : a.k - 1 - i0; // j - i
        float mine = 0.f;
        for (int c0 = first; c0 <= last; c0 += kThreads) {
            const int diag = c0 + (int)threadIdx.x;
            float s = 0.f;
            if (diag <= last)
                for (int i = i0; i < i1; ++i) {
                    const int j = i + diag;
                    if (j >= 0 && j < a.k) s += to_f32(d[(long)i * a.ld + j]);
                }
            __syncthreads();
            sums[threadIdx.x] = s;
            of[threadIdx.x] = diag <= last ? bucket_of(a, diag - a.start) : -1;
            __syncthreads();
            if ((int)threadIdx.x < a.buckets)
                for (int t = 0; t < kThreads; ++t)
                    if (of[t] == (int)threadIdx.x) mine += sums[t];
        }
        if ((int)threadIdx.x < a.buckets) a.part[((long)h * a.slices + slice) * a.buckets + threadIdx.x] = mine;
        __syncthreads();
    }
}

__global__ __launch_bounds__(64) void sequence_sum_kernel(Args a)
{
    const int b = blockIdx.x, h = blockIdx.y;
    double s = 0.;
    for (long i = threadIdx.x; i < a.slices; i += 64) s += a.part[((long)h * a.slices + i) * a.buckets + b];
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    if (threadIdx.x == 0) {
        float *out = a.dtable + (long)b * a.heads + h;
        *out = (float)(a.accumulate ? *out + s : s);
    }
}

struct Plan {
    size_t elem, out, dout, table, dtable, ws;
    long ld, slices;
    int buckets;
};

int make_plan(const relpos_desc *d, Plan *p)
{
    if (!d) return GSWA_EINVAL;
    if (d->heads <= 0 || d->heads > 65535 || (d->dtype != GSWA_F32 && d->dtype != GSWA_BF16)) return GSWA_EINVAL;
    if (d->flags & ~(uint32_t)(RELPOS_BIDIRECTIONAL | RELPOS_CAUSAL | RELPOS_ACCUM_WGRAD)) return GSWA_EINVAL;
    if (d->n_edges < 0 || d->n_edges > RELPOS_MAX_EDGES || d->window < 0 || d->window > 64) return GSWA_EINVAL;
    for (int i = 0; i < d->n_edges; ++i)
        if (d->edges[i] < (i ? d->edges[i - 1] : 1)) return GSWA_EINVAL;
    const bool both = d->flags & RELPOS_BIDIRECTIONAL;
    const int side = (d->n_edges + 1) * (both ? 2 : 1);
    p->elem = d->dtype == GSWA_F32 ? 4 : 2;
    if (d->window > 0) {
        if (!both || (d->flags & RELPOS_CAUSAL)) return GSWA_EINVAL;
        if (d->heads > 4096) return GSWA_EUNSUPPORTED;
        const long offsets = (2L * d->window - 1) * (2L * d->window - 1);
        p->buckets = side * side;
        p->out = (size_t)offsets * d->heads * p->elem;
        p->dout = (size_t)offsets * d->heads * sizeof(float);
        p->slices = 0;
        p->ws = 0;
        p->ld = 0;
    } else {
        if (d->batch <= 0 || d->q_len <= 0 || d->k_len <= 0 || d->q_start < 0) return GSWA_EINVAL;
        if ((long)d->q_start + d->q_len > (1L << 30) || d->k_len > (1 << 30)) return GSWA_EUNSUPPORTED;
        p->ld = d->row_stride ? d->row_stride : d->k_len;
        if (p->ld < d->k_len) return GSWA_EINVAL;
        const long rows = (long)d->batch * d->heads;
        if ((unsigned __int128)rows * d->q_len * p->ld > (1UL << 44)) return GSWA_EUNSUPPORTED;
        p->buckets = side;
        p->out = (((size_t)d->heads * d->q_len - 1) * p->ld + d->k_len) * p->elem;
        p->dout = (((size_t)rows * d->q_len - 1) * p->ld + d->k_len) * p->elem;
        p->slices = (long)d->batch * ((d->q_len + kRows - 1) / kRows);
        p->ws = to_256((size_t)d->heads * p->slices * side * sizeof(float));
    }
    p->table = (size_t)p->buckets * d->heads * p->elem;
    p->dtable = (size_t)p->buckets * d->heads * sizeof(float);
    return GSWA_OK;
}

void fill(const relpos_desc *d, const Plan &p, Args *a)
{
    *a = Args{};
    a->heads = d->heads; a->batch = d->batch; a->q = d->q_len; a->k = d->k_len; a->start = d->q_start;
    a->window = d->window; a->buckets = p.buckets; a->ld = p.ld; a->slices = p.slices;
    a->bidirectional = (d->flags & RELPOS_BIDIRECTIONAL) != 0;
    a->causal = (d->flags & RELPOS_CAUSAL) != 0;
    a->accumulate = (d->flags & RELPOS_ACCUM_WGRAD) != 0;
    a->n = d->n_edges;
    for (int i = 0; i < d->n_edges; ++i) a->edges[i] = d->edges[i];
}

// base^n as a whole number of 32-bit digits, times another one
std::vector<uint32_t> power(uint32_t base, int n, std::vector<uint32_t> x)
{
    for (; n > 0; --n) {
        uint64_t carry = 0;
        for (auto &digit : x) {
            carry += (uint64_t)digit * base;
            digit = (uint32_t)carry;
            carry >>= 32;
        }
        if (carry) x.push_back((uint32_t)carry);
    }
    return x;
}

// r >= E (D / E)^(k / n), i.e. r^n E^k >= D^k E^n
bool reaches(uint32_t r, uint32_t E, uint32_t D, int k, int n)
{
    const auto left = power(E, k, power(r, n, {1u})), right = power(E, n, power(D, k, {1u}));
    if (left.size() != right.size()) return left.size() > right.size();
    for (size_t i = left.size(); i-- > 0;)
        if (left[i] != right[i]) return left[i] > right[i];
    return true;
}

} // namespace
} // namespace gswa

using namespace gswa;

#define RP_LAUNCHED()                                             \
    do {                                                          \
        const hipError_t e_ = hipGetLastError();                  \
        if (e_ != hipSuccess) return report_hip_error(e_);        \
    } while (0)

extern "C" {

int relpos_log_edges(int32_t buckets, int32_t max_distance, int32_t bidirectional, int32_t *n_edges, int32_t *edges)
{
    if (!n_edges || !edges || buckets <= 0 || (bidirectional && buckets % 2)) return GSWA_EINVAL;
    const int side = bidirectional ? buckets / 2 : buckets, exact = side / 2, n = side - exact;
    if (side < 2 || side > RELPOS_MAX_EDGES + 1 || max_distance <= exact) return GSWA_EINVAL;
    try {
        for (int r = 1; r <= exact; ++r) edges[r - 1] = r;
        for (int k = 1; k < n; ++k) {
            const double t = exact * pow((double)max_distance / exact, (double)k / n);
            long r = (long)floor(t);
            // the logarithm names the border to within far less than one; whole numbers decide where it falls next to one
            if (r < 1) r = 1;
            while (r > 1 && reaches((uint32_t)(r - 1), exact, max_distance, k, n)) --r;
            while (!reaches((uint32_t)r, exact, max_distance, k, n)) ++r;
            edges[exact + k - 1] = (int32_t)r;
        }
    } catch (...) {
        return GSWA_EINVAL;
    }
    *n_edges = side - 1;
    return GSWA_OK;
}

int relpos_query_bytes(const relpos_desc *desc, size_t *bwd_ws_bytes)
{
    Plan p;
    const int rc = make_plan(desc, &p);
    if (rc != GSWA_OK) return rc;
    if (bwd_ws_bytes) *bwd_ws_bytes = p.ws;
    return GSWA_OK;
}

int relpos_forward(const relpos_desc *desc, const void *table, void *out, void *hip_stream)
{
    Plan p;
    const int rc = make_plan(desc, &p);
    if (rc != GSWA_OK) return rc;
    if (!table || !out || !aligned_to(16, table, out)) return GSWA_EINVAL;
    if (overlaps_any(Range(out, p.out), Range(table, p.table))) return GSWA_EINVAL;
    Args a;
    fill(desc, p, &a);
    a.table = table; a.out = out;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    KernelTimer t(K_RELPOS_FWD, st);
    if (desc->window > 0) {
        const long total = (2L * desc->window - 1) * (2L * desc->window - 1) * desc->heads;
        const dim3 grid((unsigned)((total + kThreads - 1) / kThreads));
        if (desc->dtype == GSWA_F32) hipLaunchKernelGGL(window_fwd_kernel<float>, grid, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL(window_fwd_kernel<bf16_t>, grid, dim3(kThreads), 0, st, a);
    } else {
        const dim3 grid(desc->q_len < 8192 ? desc->q_len : 8192, desc->heads);
        if (desc->dtype == GSWA_F32) hipLaunchKernelGGL(sequence_fwd_kernel<float>, grid, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL(sequence_fwd_kernel<bf16_t>, grid, dim3(kThreads), 0, st, a);
    }
    RP_LAUNCHED();
    return GSWA_OK;
}

int relpos_backward(const relpos_desc *desc, const void *dout, float *dtable, void *ws, void *hip_stream)
{
    Plan p;
    const int rc = make_plan(desc, &p);
    if (rc != GSWA_OK) return rc;
    if (!dout || !dtable || (p.ws && !ws) || !aligned_to(16, dout, dtable) || !aligned_to(256, ws)) return GSWA_EINVAL;
    const Range rd(dout, p.dout), rt(dtable, p.dtable), rw(ws, p.ws);
    if (overlaps_any(rt, rd, rw) || overlaps_any(rw, rd)) return GSWA_EINVAL;
    Args a;
    fill(desc, p, &a);
    a.dout = dout; a.dtable = dtable; a.part = static_cast<float *>(ws);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (desc->window > 0) {
        KernelTimer t(K_RELPOS_BWD, st);
        hipLaunchKernelGGL(window_bwd_kernel, dim3((unsigned)(((long)p.buckets * desc->heads + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, a);
        RP_LAUNCHED();
        return GSWA_OK;
    }
    const dim3 grid((unsigned)(p.slices < 65536 ? p.slices : 65536), desc->heads);
    {
        KernelTimer t(K_RELPOS_BWD, st);
        if (desc->dtype == GSWA_F32) hipLaunchKernelGGL(sequence_bwd_kernel<float>, grid, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL(sequence_bwd_kernel<bf16_t>, grid, dim3(kThreads), 0, st, a);
        RP_LAUNCHED();
    }
    KernelTimer t(K_RELPOS_SUM, st);
    hipLaunchKernelGGL(sequence_sum_kernel, dim3(p.buckets, desc->heads), dim3(64), 0, st, a);
    RP_LAUNCHED();
    return GSWA_OK;
}

} // extern "C"
