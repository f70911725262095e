// LayerNorm of rows, forward and backward (lnorm.h): the kernels and the C ABI.
//
// Both passes are bound by memory: about ten operations an element against 4 to 14 bytes.  So a row is read once, stays in the registers
// of L lanes (P vectors of 16 bytes each), and all of a row's sums are formed there: the mean, then the squares of the distances from it (in a second
// round, so that a mean far from zero costs the variance no digits).
#include "../../include/lnorm.h"
#include "args.h"
#include "common.h"
#include "mfma.h"
#include "profile.h"

#include <type_traits>

namespace gswa {
namespace {

constexpr int kSumThreads = 1024, kSumColumns = 32;
// Rounds of rows that one workgroup takes where it then has them all, and no second launch adds partial sums (bf16 rows of 768: 16 of them, two rounds, 6.8 us, with the
// second launch 8.3; 32, four rounds, 9.0, with it 8.6).
constexpr int kAlone = 2;
constexpr long kBalance = 500000; // see make_plan
constexpr int N_MAX = 3; // sums of a row that are formed at once

struct Args {
    const void *x, *residual, *gamma, *beta, *dy, *dsum;
    void *y, *sum, *dx;
    float *part;    // backward: [workgroups][2 C], null where no parameter gradients are wanted or one workgroup has all rows
    float *dgamma, *dbeta;
    long rows, ldx, ldy, ldr;
    int C, accumulate, parts;
    float eps;
};

// V values as they lie in memory; a row starts anywhere, so only the alignment of an element is promised (the wide loads and stores take any).
template <typename T, int V> struct Raw {
    typename std::conditional<V * sizeof(T) == 16, uint4, T>::type w;
};
template <typename T, int V> __device__ __forceinline__ Raw<T, V> load(const T *p)
{
    Raw<T, V> r;
    __builtin_memcpy(&r.w, p, V * sizeof(T));
    return r;
}
__device__ __forceinline__ void unpack(const Raw<bf16_t, 8> &r, float *f)
{
    f[0] = bf16_lo(r.w.x); f[1] = bf16_hi(r.w.x); f[2] = bf16_lo(r.w.y); f[3] = bf16_hi(r.w.y);
    f[4] = bf16_lo(r.w.z); f[5] = bf16_hi(r.w.z); f[6] = bf16_lo(r.w.w); f[7] = bf16_hi(r.w.w);
}
__device__ __forceinline__ void unpack(const Raw<float, 4> &r, float *f)
{
    f[0] = __uint_as_float(r.w.x); f[1] = __uint_as_float(r.w.y); f[2] = __uint_as_float(r.w.z); f[3] = __uint_as_float(r.w.w);
}
template <typename T> __device__ __forceinline__ void unpack(const Raw<T, 1> &r, float *f) { f[0] = to_f32(r.w); }
__device__ __forceinline__ Raw<bf16_t, 8> pack(const float *f, Raw<bf16_t, 8>)
{
    return {make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]))};
}
__device__ __forceinline__ Raw<float, 4> pack(const float *f, Raw<float, 4>)
{
    return {make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]))};
}
template <typename T> __device__ __forceinline__ Raw<T, 1> pack(const float *f, Raw<T, 1> r)
{
    from_f32(r.w, f[0]);
    return r;
}
template <typename T, int V> __device__ __forceinline__ void store(T *p, const float *f)
{
    const Raw<T, V> r = pack(f, Raw<T, V>{});
    __builtin_memcpy(p, &r.w, V * sizeof(T));
}

// The compiler may not carry what it unpacked from these over this point (it would hold a register for each value, where unpacking again is one
// instruction).
__device__ __forceinline__ void again(Raw<bf16_t, 8> &r) { asm volatile("" : "+v"(r.w.x), "+v"(r.w.y), "+v"(r.w.z), "+v"(r.w.w)); }
__device__ __forceinline__ void again(Raw<float, 4> &r) { asm volatile("" : "+v"(r.w.x), "+v"(r.w.y), "+v"(r.w.z), "+v"(r.w.w)); }
template <typename T> __device__ __forceinline__ void again(Raw<T, 1> &) {}

// V ones or zeros where gamma or beta is not given: the loop over the rows has no branch for it
template <typename T, int V> __device__ __forceinline__ Raw<T, V> all(float v)
{
    float f[V];
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = v;
    return pack(f, Raw<T, V>{});
}

template <int CTRL> __device__ __forceinline__ float dpp_add(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
// v_permlane16_swap(v, v) and v_permlane32_swap(v, v) leave v and its partner of the other row of 16 lanes, or half of the wavefront, in the two results
__device__ __forceinline__ float rows_add(float v)
{
    const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float halves_add(float v)
{
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// sum over groups of 8 to 64 lanes: pairs, quads, halves of a row of 16 lanes (a mirrored lane holds what the exchanged one holds), rows, halves
template <int L> __device__ __forceinline__ float lanes_sum(float v)
{
    v = dpp_add<0xB1>(v);
    v = dpp_add<0x4E>(v);
    v = dpp_add<0x141>(v);
    if constexpr (L >= 16) v = dpp_add<0x140>(v);
    if constexpr (L >= 32) v = rows_add(v);
    if constexpr (L >= 64) v = halves_add(v);
    return v;
}

// The L lanes of a row, and what each holds of it: vector p of a lane is columns [column(p), column(p) + V).  The row's last vector ends
// at column C: where C is no multiple of V it begins inside the one before it, whose columns it reads as well but does not own.  (So no load is ever
// narrower than a vector.  Within a wavefront the stores are not either: both lanes store the same values.  Across wavefronts a lane stores what it owns: in a
// call that works in place the other one may have read its vector again after this one stored.)
template <int L, int P, int V, int THREADS> struct Place {
    static constexpr int kBlock = THREADS, kGroups = kBlock / L, kWaves = kBlock / 64;
    int C, lane;
    __device__ __forceinline__ Place(int C_) : C(C_), lane((int)threadIdx.x % L) {}
    __device__ __forceinline__ int column(int p) const
    {
        const int c = (p * L + lane) * V;
        return c < C - V ? c : C - V;
    }
    __device__ __forceinline__ bool any(int p) const { return p < P - 1 || (p * L + lane) * V < C; }
    // whether element i of vector p is this lane's (P is the least that holds a row: only a lane's last vector can be short)
    __device__ __forceinline__ bool own(int p, int i) const { return p < P - 1 || column(p) + i >= (p * L + lane) * V; }
    template <typename T> __device__ __forceinline__ void fetch(const T *row, Raw<T, V> (&r)[P]) const
    {
#pragma unroll
        for (int p = 0; p < P; ++p) r[p] = load<T, V>(row + column(p));
    }
    // `without` throughout where there is no vector
    template <typename T> __device__ __forceinline__ void fetch_or(const void *row, float without, Raw<T, V> (&r)[P]) const
    {
#pragma unroll
        for (int p = 0; p < P; ++p) r[p] = row ? load<T, V>(static_cast<const T *>(row) + column(p)) : all<T, V>(without);
    }
    template <typename T> __device__ __forceinline__ void put(T *row, int p, const float *f) const
    {
        if (!any(p)) return;
        if (L <= 64 || own(p, 0)) {
            store<T, V>(row + column(p), f);
        } else {
#pragma unroll
            for (int i = 1; i < V; ++i)
                if (own(p, i)) from_f32(row[column(p) + i], f[i]);
        }
    }
    template <typename T> __device__ __forceinline__ void put(T *row, const float (&f)[P * V]) const
    {
#pragma unroll
        for (int p = 0; p < P; ++p) put(row, p, f + p * V);
    }
    // Sums over the lanes of a row, of N values at once.  Rows of more than a wavefront go through LDS; `half` alternates between
    // the two halves of it, so that one barrier a sum is enough.
    template <int N> __device__ __forceinline__ void sum(float (&v)[N], float (*lds)[N_MAX][kWaves], int half) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = lanes_sum<(L < 64 ? L : 64)>(v[n]);
        if constexpr (L > 64) {
            const int wave = threadIdx.x >> 6, first = (int)threadIdx.x / L * (L / 64);
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int n = 0; n < N; ++n) lds[half][n][wave] = v[n];
            }
            __syncthreads();
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < L / 64; ++w) s += lds[half][n][first + w];
                v[n] = s;
            }
        }
    }
};

// Threads of a workgroup.  The backward pass leaves one vector of partial sums per workgroup, so where no barrier ties its rows together it has half as many,
// of twice the size, if the registers allow four wavefronts on a SIMD anyway.
template <int L> constexpr int fwd_threads() { return L > 256 ? L : 256; }
constexpr int bwd_threads(int L, int values, int V) { return L > 256 || (L <= 64 && values <= (V == 4 ? 8 : 16)) ? 512 : 256; }

template <typename T, int L, int P, int V>
__global__ __launch_bounds__((fwd_threads<L>())) void lnorm_fwd_kernel(Args a)
{
    using Pl = Place<L, P, V, fwd_threads<L>()>;
    __shared__ float lds[2][N_MAX][Pl::kWaves];
    const Pl pl(a.C);
    const T *x = static_cast<const T *>(a.x), *res = static_cast<const T *>(a.residual);
    const long stride = (long)gridDim.x * Pl::kGroups;
    long row = (long)blockIdx.x * Pl::kGroups + (Pl::kGroups == 1 ? 0 : threadIdx.x / L);
    Raw<T, V> gamma[P], beta[P], rx[P], rr[P];
    pl.fetch_or(a.gamma, 1.f, gamma);
    pl.fetch_or(a.beta, 0.f, beta);
    // (a group of lanes past the last row goes along on that row and stores nothing)
    const auto fetch = [&](long r) {
        const long at = r < a.rows ? r : a.rows - 1;
        pl.fetch(x + at * a.ldx, rx);
        if (res) pl.fetch(res + at * a.ldr, rr);
    };
    const float per = 1.f / (float)a.C;
    fetch(row);
    for (long base = (long)blockIdx.x * Pl::kGroups; base < a.rows; base += stride, row += stride) {
        float u[P * V];
        const bool live = Pl::kGroups == 1 || row < a.rows;
#pragma unroll
        for (int p = 0; p < P; ++p) unpack(rx[p], u + p * V);
        if (res) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                float r[V];
                unpack(rr[p], r);
#pragma unroll
                for (int i = 0; i < V; ++i) u[p * V + i] += r[i];
                const Raw<T, V> held = pack(u + p * V, Raw<T, V>{}); // the norm is of what is stored
                unpack(held, u + p * V);
                if (live) pl.put(static_cast<T *>(a.sum) + row * a.ldr, p, u + p * V); // (exact: the values are of the type)
            }
        }
        if (base + stride < a.rows) fetch(row + stride);
        float s[1] = {0.f}, q[1] = {0.f};
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += pl.own(p, i) ? u[p * V + i] : 0.f;
        pl.sum(s, lds, 0);
        const float mean = s[0] / (float)a.C;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                u[p * V + i] -= mean;
                q[0] += pl.own(p, i) ? u[p * V + i] * u[p * V + i] : 0.f;
            }
        pl.sum(q, lds, 1);
        const float rstd = rsqrtf(q[0] * per + a.eps);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float f[V], e[V];
            unpack(gamma[p], f);
            unpack(beta[p], e);
#pragma unroll
            for (int i = 0; i < V; ++i) u[p * V + i] = u[p * V + i] * rstd * f[i] + e[i];
        }
        if (live) pl.put(static_cast<T *>(a.y) + row * a.ldy, u);
    }
}

// dx of every row, and over the rows of a workgroup the sums of dy * xh and dy, a column in one place of one lane's registers throughout; they
// leave as one vector of 2 C partial sums.
template <typename T, int L, int P, int V, bool DSUM>
__global__ __launch_bounds__((bwd_threads(L, P * V, V))) void lnorm_bwd_kernel(Args a)
{
    using Pl = Place<L, P, V, bwd_threads(L, P * V, V)>;
    __shared__ float lds[2][N_MAX][Pl::kWaves];
    Pl pl(a.C);
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy), *ds = static_cast<const T *>(a.dsum);
    const long stride = (long)gridDim.x * Pl::kGroups;
    long row = (long)blockIdx.x * Pl::kGroups + (Pl::kGroups == 1 ? 0 : threadIdx.x / L);
    Raw<T, V> gamma[P], rx[P], ry[P], rs[P];
    pl.fetch_or(a.gamma, 1.f, gamma);
    const auto fetch = [&](long r) {
        const long at = r < a.rows ? r : a.rows - 1;
        pl.fetch(x + at * a.ldx, rx);
        pl.fetch(dy + at * a.ldy, ry);
    };
    float dg[P * V] = {}, db[P * V] = {};
    const float per = 1.f / (float)a.C;
    constexpr bool kAhead = P * V <= (V == 8 ? 24 : 16); // (the next row's vectors beside this one's values: too much for the widest rows' registers)
    if (kAhead) fetch(row);
    for (long base = (long)blockIdx.x * Pl::kGroups; base < a.rows; base += stride, row += stride) {
        float u[P * V], d[P * V];
        const bool live = Pl::kGroups == 1 || row < a.rows;
        if (!kAhead) fetch(row);
        if constexpr (DSUM && kAhead) pl.fetch(ds + (live ? row : a.rows - 1) * a.ldr, rs);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            unpack(rx[p], u + p * V);
            unpack(ry[p], d + p * V);
        }
        if (kAhead && base + stride < a.rows) fetch(row + stride);
        if (!live) {
#pragma unroll
            for (int k = 0; k < P * V; ++k) d[k] = 0.f;
        }
        float s[1] = {0.f};
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += pl.own(p, i) ? u[p * V + i] : 0.f;
        pl.sum(s, lds, 0);
        const float mean = s[0] / (float)a.C;
        // sums of the squared distances, of g and of g times the distance, in one round
        float t[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float f[V];
            unpack(gamma[p], f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int k = p * V + i;
                u[k] -= mean;
                const float g = d[k] * f[i];
                t[0] += pl.own(p, i) ? u[k] * u[k] : 0.f;
                t[1] += pl.own(p, i) ? g : 0.f;
                t[2] += pl.own(p, i) ? g * u[k] : 0.f;
            }
        }
        pl.sum(t, lds, 1);
        if constexpr (DSUM && !kAhead) pl.fetch(ds + (live ? row : a.rows - 1) * a.ldr, rs);
        const float rstd = rsqrtf(t[0] * per + a.eps), sg = t[1] * per, sgx = t[2] * per * rstd;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float f[V], e[V];
            again(gamma[p]);
            unpack(gamma[p], f);
            if constexpr (DSUM) unpack(rs[p], e);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int k = p * V + i;
                const float xh = u[k] * rstd, g = d[k] * f[i];
                dg[k] += d[k] * xh;
                db[k] += d[k];
                u[k] = (g - sg - xh * sgx) * rstd;
                if constexpr (DSUM) u[k] += e[i];
            }
        }
        if (live) pl.put(static_cast<T *>(a.dx) + row * a.ldr, u);
    }
    if (!a.dgamma) return;
    asm("" : "+v"(pl.lane)); // (or the places of what follows would be found before the loop and held through it)
    float *const out_g = a.part ? a.part + (size_t)blockIdx.x * 2 * a.C : a.dgamma, *const out_b = a.part ? out_g + a.C : a.dbeta;
    const bool add = !a.part && a.accumulate;
    if constexpr (L > 64 && Pl::kGroups > 1) { // the other wavefronts' sums to those of the first row
        static_assert(L <= 64 || Pl::kGroups <= 2, "two rows at once");
        __shared__ float other[2][L * P * V];
        if ((int)threadIdx.x >= L) {
#pragma unroll
            for (int k = 0; k < P * V; ++k) other[0][k * L + pl.lane] = dg[k], other[1][k * L + pl.lane] = db[k];
        }
        __syncthreads();
        if ((int)threadIdx.x >= L) return;
#pragma unroll
        for (int k = 0; k < P * V; ++k) dg[k] += other[0][k * L + pl.lane], db[k] += other[1][k * L + pl.lane];
    }
    const auto leave = [&](float *out, float (&f)[P * V]) {
        if constexpr (L <= 64) {
            // Groups of a wavefront by exchanges between its lanes; then each wavefront lays its sums into LDS, and a thread adds up a column in their
            // order.  (Columns that a row's last vector reads again have the same sums in both lanes.)
            __shared__ __align__(16) float sums[Pl::kWaves][L * P * V];
#pragma unroll
            for (int k = 0; k < P * V; ++k) {
                if constexpr (L == 8) f[k] = dpp_add<0x128>(f[k]); // (row_ror 8)
                if constexpr (L <= 16) f[k] = rows_add(f[k]);
                if constexpr (L <= 32) f[k] = halves_add(f[k]);
            }
            __syncthreads(); // (the sums before these have been read)
            float *mine = sums[threadIdx.x >> 6];
            if ((threadIdx.x & 63) < L) {
#pragma unroll
                for (int p = 0; p < P; ++p)
                    if (pl.any(p)) __builtin_memcpy(mine + pl.column(p), f + p * V, V * sizeof(float));
            }
            __syncthreads();
            for (int c = threadIdx.x; c < a.C; c += Pl::kBlock) {
                float s = sums[0][c];
#pragma unroll
                for (int w = 1; w < Pl::kWaves; ++w) s += sums[w][c];
                out[c] = add ? out[c] + s : s;
            }
        } else {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (!pl.any(p)) continue;
                if (pl.own(p, 0) && !add) { // a whole vector of its own
                    __builtin_memcpy(out + pl.column(p), f + p * V, V * sizeof(float));
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (pl.own(p, i)) out[pl.column(p) + i] = add ? out[pl.column(p) + i] + f[p * V + i] : f[p * V + i];
                }
            }
        }
    };
    leave(out_g, dg);
    leave(out_b, db);
}

// The partial sums of kSumColumns columns: a slice of the workgroups per 32 threads, then the slices in their order.
__global__ __launch_bounds__(kSumThreads) void lnorm_sum_kernel(Args a)
{
    constexpr int kSlices = kSumThreads / kSumColumns;
    __shared__ float lds[kSlices][kSumColumns];
    const int col = threadIdx.x % kSumColumns, slice = threadIdx.x / kSumColumns, c = blockIdx.x * kSumColumns + col;
    float s = 0.f;
    if (c < 2 * a.C) {
#pragma unroll 8
        for (int i = slice; i < a.parts; i += kSlices) s += a.part[(size_t)i * 2 * a.C + c];
    }
    lds[slice][col] = s;
    __syncthreads();
    if (slice || c >= 2 * a.C) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < kSlices; ++i) s += lds[i][col];
    float *out = c < a.C ? a.dgamma + c : a.dbeta + (c - a.C);
    *out = a.accumulate ? *out + s : s;
}

struct Plan {
    size_t elem, ws;
    long ldx, ldy, ldr;
    int lanes, vectors; // L and P; lanes = 0: rows shorter than a vector
    unsigned fwd_blocks, bwd_blocks, sum_blocks; // sum_blocks: of the backward pass where it leaves partial sums
};

// Lanes of a row: as few as hold it in 24 values of bf16 or 16 of fp32 each, at most 512, which hold the widest rows in 32.  (Fewer lanes with more
// values keep more loads in flight and leave fewer lanes idle behind the row's end; the backward pass has two fp32 sums for each value in registers as
// well.  Backward of 8192 x 5120 bf16 without parameter gradients: 640 vectors on 256 lanes 48.2 us, on 512 58.1 us; 4096 x 12288: on 512
// 57.5 us, on 1024 74.2 us.)
int lanes_of(int C, int V)
{
    int L = 8;
    while (L * (V == 8 ? 24 : 16) < C && L < 512) L *= 2;
    return L;
}

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
    if (d->C > 16384) return GSWA_EUNSUPPORTED;
    const long widest = p->ldx > p->ldy ? (p->ldx > p->ldr ? p->ldx : p->ldr) : (p->ldy > p->ldr ? p->ldy : p->ldr);
    if (d->rows > (1L << 40) / widest) return GSWA_EUNSUPPORTED;
    const int V = (int)(16 / p->elem), n = (d->C + V - 1) / V;
    p->lanes = d->C < V ? 0 : lanes_of(d->C, V);
    const int L = p->lanes ? p->lanes : 8;
    p->vectors = p->lanes ? (n + L - 1) / L : 1;
    const int values = p->vectors * (p->lanes ? V : 1);
    // workgroups: what the compute units hold at once, going on to further rows
    const auto blocks = [&](int threads, long most) {
        const long rounds = (d->rows + threads / L - 1) / (threads / L);
        return (unsigned)(rounds < most ? rounds : most);
    };
    p->fwd_blocks = blocks(L > 256 ? L : 256, (L > 256 ? 4 : 8) * kSizingCus);
    const long together = bwd_threads(L, values, p->lanes ? V : 1) / L; // rows of a workgroup at once
    p->bwd_blocks = blocks(bwd_threads(L, values, p->lanes ? V : 1), (L > 256 && values > 16 ? 1 : L <= 64 && V == 4 && values > 8 ? 3 : 2) * kSizingCus);
    // With partial sums a workgroup takes at least r rounds of rows, such that r round times are what writing and reading the sums takes, 16 C bytes a workgroup: r^2 =
    // rounds C / kBalance (8192 values in bf16: 512 rows in 512 workgroups 21.8 us, in 128 to 171 16.8 to 18.3, in 86 20.5; fp32, 1024 rows 36.1 and 27).
    const long rounds = (d->rows + together - 1) / together;
    long r = 1;
    while (r * r * kBalance < rounds * d->C) ++r;
    p->sum_blocks = rounds <= kAlone ? 1 : (unsigned)((rounds + r - 1) / r < p->bwd_blocks ? (rounds + r - 1) / r : p->bwd_blocks);
    p->ws = to_256((size_t)p->sum_blocks * 2 * d->C * sizeof(float));
    return GSWA_OK;
}

template <typename T, int L, int P, int V> void launch(const Args &a, const Plan &p, bool forward, hipStream_t st)
{
    const dim3 fwd(fwd_threads<L>()), bwd(bwd_threads(L, P * V, V));
    if (forward) hipLaunchKernelGGL((lnorm_fwd_kernel<T, L, P, V>), dim3(p.fwd_blocks), fwd, 0, st, a);
    else if (a.dsum) hipLaunchKernelGGL((lnorm_bwd_kernel<T, L, P, V, true>), dim3(a.parts), bwd, 0, st, a);
    else hipLaunchKernelGGL((lnorm_bwd_kernel<T, L, P, V, false>), dim3(a.parts), bwd, 0, st, a);
}

// The numbers of vectors that lanes_of leads to: more than half of the most, but on 8 lanes, and up to 32 values on 512.
template <typename T, int L> void launch_vectors(const Args &a, const Plan &p, bool forward, hipStream_t st)
{
    constexpr int V = 16 / sizeof(T);
    switch (p.vectors) {
    case 1: if constexpr (L == 8) launch<T, L, 1, V>(a, p, forward, st); break;
    case 2: if constexpr (L == 8 || V == 8) launch<T, L, 2, V>(a, p, forward, st); break;
    case 3: launch<T, L, 3, V>(a, p, forward, st); break;
    case 4: if constexpr (L == 512 || V == 4) launch<T, L, 4, V>(a, p, forward, st); break;
    case 5: if constexpr (L == 512 && V == 4) launch<T, L, 5, V>(a, p, forward, st); break;
    case 6: if constexpr (L == 512 && V == 4) launch<T, L, 6, V>(a, p, forward, st); break;
    case 7: if constexpr (L == 512 && V == 4) launch<T, L, 7, V>(a, p, forward, st); break;
    case 8: if constexpr (L == 512 && V == 4) launch<T, L, 8, V>(a, p, forward, st); break;
    }
}

template <typename T> void launch_type(const Args &a, const Plan &p, bool forward, hipStream_t st)
{
    switch (p.lanes) {
    case 0: launch<T, 8, 1, 1>(a, p, forward, st); break;
    case 8: launch_vectors<T, 8>(a, p, forward, st); break;
    case 16: launch_vectors<T, 16>(a, p, forward, st); break;
    case 32: launch_vectors<T, 32>(a, p, forward, st); break;
    case 64: launch_vectors<T, 64>(a, p, forward, st); break;
    case 128: launch_vectors<T, 128>(a, p, forward, st); break;
    case 256: launch_vectors<T, 256>(a, p, forward, st); break;
    case 512: launch_vectors<T, 512>(a, p, forward, st); break;
    }
}

// bytes from the first row's first value to the last row's last one
size_t span(const lnorm_desc *d, const Plan &p, long ld) { return ((size_t)(d->rows - 1) * ld + d->C) * p.elem; }

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
    if (bwd_ws_bytes) *bwd_ws_bytes = p.ws;
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
    if (desc->dtype == GSWA_F32) launch_type<float>(a, p, true, st);
    else launch_type<bf16_t>(a, p, true, st);
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
        rd(dx, span(desc, p, p.ldr)), wg(dgamma, vec), wb(dbeta, vec), rw(dgamma ? ws : nullptr, p.ws);
    if (overlaps_any(rd, rx, rg, wg, wb, rw) || overlaps_any(wg, rx, ry, rg, rs, wb, rw) ||
        overlaps_any(wb, rx, ry, rg, rs, rw) || overlaps_any(rw, rx, ry, rg, rs))
        return GSWA_EINVAL;
    if (overlaps_any(rd, ry) && !(dx == dy && p.ldy == p.ldr)) return GSWA_EINVAL;
    if (overlaps_any(rd, rs) && dx != dsum) return GSWA_EINVAL;
    Args a{};
    a.x = x; a.dy = dy; a.gamma = gamma; a.dsum = dsum; a.dx = dx; a.dgamma = dgamma; a.dbeta = dbeta;
    a.rows = desc->rows; a.ldx = p.ldx; a.ldy = p.ldy; a.ldr = p.ldr; a.C = desc->C; a.eps = desc->eps;
    a.accumulate = (desc->flags & LNORM_ACCUM_WGRAD) != 0;
    a.part = dgamma && p.sum_blocks > 1 ? static_cast<float *>(ws) : nullptr;
    a.parts = (int)(dgamma ? p.sum_blocks : p.bwd_blocks);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    {
        KernelTimer t(K_LNORM_BWD, st);
        if (desc->dtype == GSWA_F32) launch_type<float>(a, p, false, st);
        else launch_type<bf16_t>(a, p, false, st);
        LN_LAUNCHED();
    }
    if (a.part) {
        KernelTimer t(K_LNORM_SUM, st);
        hipLaunchKernelGGL(lnorm_sum_kernel, dim3((2 * desc->C + kSumColumns - 1) / kSumColumns), dim3(kSumThreads), 0, st, a);
        LN_LAUNCHED();
    }
    return GSWA_OK;
}

} // extern "C"
