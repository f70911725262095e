// One AdamW step over many tensors (adamw.h): the plan, the norm of the gradients, the step, the read-back of
// 8-bit states, and the C ABI.
#include "../../include/adamw.h"
#include "args.h"
#include "common.h"
#include "mfma.h"
#include "profile.h"

#include <algorithm>
#include <vector>

namespace gswa {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kBlock = 256;             // elements that share an exponent: four for each lane of a wavefront
constexpr int kChunkBlocks = 8;         // blocks of one piece of work: two for each wavefront of a workgroup
constexpr long kChunk = (long)kBlock * kChunkBlocks;
constexpr int kNormBlocks = 1024;

// A tensor as the kernels see it.
struct Tensor {
    void *p;
    float *master;
    const void *g;
    void *m, *v;
    uint8_t *m_exp, *v_exp;
    long n;
    long first_block; // its place among all blocks
    int first_chunk;  // and among all pieces of work
    float decay;
    int p_bf16, g_bf16;
};

// The plan's buffer: [Tensor * n][tensor of every piece of work, int][partial sums of the norm][counter]
struct Layout {
    size_t owner, part, counter, bytes;
};
Layout layout(int n, long chunks)
{
    Layout l;
    l.owner = to_256((size_t)n * sizeof(Tensor));
    l.part = l.owner + to_256((size_t)chunks * sizeof(int));
    l.counter = l.part + to_256(kNormBlocks * sizeof(double));
    l.bytes = l.counter + 256;
    return l;
}

struct Step {
    const Tensor *tensors;
    const int *owner;
    double *part;
    unsigned *counter;
    long chunks;
    int64_t *step;
    const float *lr_scale, *norm;
    float *norm_out;
    double beta1, beta2;
    float lr, max_norm, b1, b1c, b2, b2c, eps; // beta and 1 - beta, each rounded once
    int eight, skip;
    uint32_t seed_lo, seed_hi;
    uint16_t *m_out, *v_out;
};

constexpr int kPerLaunch = 40; // tensors whose places fit the arguments of one launch
struct PlanArgs {
    Tensor t[kPerLaunch];
    Tensor *tensors;
    int *owner;
    unsigned *counter;
    int first;
};

__global__ __launch_bounds__(kThreads) void plan_kernel(PlanArgs a)
{
    const Tensor &t = a.t[blockIdx.x];
    const int index = a.first + (int)blockIdx.x;
    if (threadIdx.x == 0) {
        a.tensors[index] = t;
        if (index == 0) *a.counter = 0;
    }
    const int chunks = (int)((t.n + kChunk - 1) / kChunk);
    for (int c = threadIdx.x; c < chunks; c += kThreads) a.owner[t.first_chunk + c] = index;
}

__device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x9E3779B9u;
    x ^= x >> 15;
    x *= 0x6A09E667u;
    return x ^ x >> 16;
}

// A lane's four elements of a block, from `i` on, as many of them as the tensor has; a whole four by one wide access.
template <typename T> __device__ __forceinline__ void load4(const T *p, int left, T (&v)[4])
{
    if (left >= 4) {
        __builtin_memcpy(v, __builtin_assume_aligned(p, 4 * sizeof(T) < 16 ? 4 * sizeof(T) : 16), 4 * sizeof(T));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = j < left ? p[j] : T{};
    }
}
template <typename T> __device__ __forceinline__ void store4(T *p, int left, const T (&v)[4])
{
    if (left >= 4) {
        __builtin_memcpy(__builtin_assume_aligned(p, 4 * sizeof(T) < 16 ? 4 * sizeof(T) : 16), v, 4 * sizeof(T));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[j] = v[j];
    }
}
// (bf16 or fp32 by a flag of the tensor, the same for a whole wavefront)
__device__ __forceinline__ void load4_as(const void *p, long i, bool bf16, int left, float (&f)[4])
{
    if (bf16) {
        bf16_t v[4];
        load4(static_cast<const bf16_t *>(p) + i, left, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = to_f32(v[j]);
    } else {
        load4(static_cast<const float *>(p) + i, left, f);
    }
}

// a wavefront's largest pattern
template <int CTRL> __device__ __forceinline__ uint32_t dpp_max(uint32_t v)
{
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
    return o > v ? o : v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    v = dpp_max<0xB1>(v);
    v = dpp_max<0x4E>(v);
    v = dpp_max<0x141>(v);
    v = dpp_max<0x140>(v);
    u32x2 r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = r[0] > r[1] ? r[0] : r[1];
    r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return r[0] > r[1] ? r[0] : r[1];
}

// Value of code c (without its sign) in a block of exponent E, and the code of a magnitude's pattern rounded by 16 random bits.
template <int TOP> __device__ __forceinline__ float decode(uint32_t c, int E)
{
    const int T = 8 * (E + 1) - TOP + (int)c;
    const uint32_t bits = c ? (uint32_t)(T > 1 ? T : 1) << 20 : 0u;
    return __uint_as_float(E == 255 ? 0x7fc00000u : bits);
}
template <int TOP> __device__ __forceinline__ uint32_t encode(uint32_t bits, int E, uint32_t noise)
{
    constexpr int least = TOP == 255 ? 1 : 0; // (a second moment that is not 0 is not stored as 0)
    int T = (int)((bits + (noise << 4)) >> 20);
    const bool none = least ? bits == 0 : T < 1;
    T = T > 1 ? T : 1;
    const int c = T - (8 * (E + 1) - TOP), most = E == 254 ? TOP - 1 : TOP;
    return none || E == 255 ? 0u : (uint32_t)(c < least ? least : c > most ? most : c);
}

// What a step needs of its number and rates, the same for all elements.
struct Rates {
    float lr, rate, root, clip; // learning rate; over 1 - beta1^t; sqrt(1 - beta2^t); factor of the gradients
    uint32_t key;
};
__device__ __forceinline__ Rates rates_of(const Step &a, float norm)
{
    const uint64_t t = (uint64_t)*a.step + 1;
    double b1 = 1., b2 = 1., f1 = a.beta1, f2 = a.beta2; // beta^t by squares
    for (uint64_t e = t; e; e >>= 1) {
        if (e & 1) b1 *= f1, b2 *= f2;
        f1 *= f1;
        f2 *= f2;
    }
    Rates r;
    r.lr = a.lr_scale ? a.lr * *a.lr_scale : a.lr;
    r.rate = r.lr / (float)(1. - b1);
    r.root = sqrtf((float)(1. - b2));
    r.clip = a.max_norm > 0.f && norm > a.max_norm ? a.max_norm / norm : 1.f;
    r.key = mix(mix(a.seed_hi ^ 0x510E527Fu) ^ a.seed_lo);
    r.key = mix(mix(r.key ^ (uint32_t)(t >> 32)) ^ (uint32_t)t);
    return r;
}

// What the next step sees of the states is rounded from m' and v', so these are formed by products and sums that are rounded one by one
// (no fused multiply-add): the result does not hang on how a compiler joins them.
__device__ __forceinline__ void moments(const Step &a, float g, float &m, float &v)
{
#pragma clang fp contract(off)
    m = m * a.b1 + g * a.b1c;
    v = v * a.b2 + g * g * a.b2c;
}

// Bound by memory: 16 to 30 bytes an element against some 40 operations.  A workgroup takes pieces of 8 blocks, a wavefront two of them with all loads of both
// in flight together; a block's largest magnitude comes from exchanges between its lanes.
template <bool EIGHT> __global__ __launch_bounds__(kThreads) void step_kernel(Step a)
{
    constexpr int kEach = kChunkBlocks / kWaves;
    const float norm = a.norm ? *a.norm : 0.f;
    if (a.skip && !(fabsf(norm) < INFINITY)) return;
    const Rates r = rates_of(a, norm);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (long chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        const Tensor T = a.tensors[a.owner[chunk]];
        const long first = (chunk - T.first_chunk) * kChunkBlocks + wave;
        float g[kEach][4], p[kEach][4], m[kEach][4], v[kEach][4];
        uint8_t cm[kEach][4], cv[kEach][4];
        int em[kEach], ev[kEach], left[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const long block = first + k * kWaves, i = block * kBlock + lane * 4, n = T.n - i;
            left[k] = n < 0 ? 0 : n < 4 ? (int)n : 4;
            if (block * kBlock >= T.n) continue;
            load4_as(T.g, i, T.g_bf16, left[k], g[k]);
            if (T.master) load4(T.master + i, left[k], p[k]);
            else load4_as(T.p, i, T.p_bf16, left[k], p[k]);
            if (EIGHT) {
                load4(static_cast<const uint8_t *>(T.m) + i, left[k], cm[k]);
                load4(static_cast<const uint8_t *>(T.v) + i, left[k], cv[k]);
                em[k] = T.m_exp[block];
                ev[k] = T.v_exp[block];
            } else {
                load4(static_cast<const float *>(T.m) + i, left[k], m[k]);
                load4(static_cast<const float *>(T.v) + i, left[k], v[k]);
            }
        }
        const float keep = 1.f - r.lr * T.decay;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const long block = first + k * kWaves, i = block * kBlock + lane * 4;
            if (block * kBlock >= T.n) continue;
            uint32_t mmax = 0, vmax = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (EIGHT) {
                    m[k][j] = decode<127>(cm[k][j] & 127, em[k]);
                    if (cm[k][j] & 128) m[k][j] = -m[k][j];
                    v[k][j] = decode<255>(cv[k][j], ev[k]);
                }
                moments(a, g[k][j] * r.clip, m[k][j], v[k][j]);
                p[k][j] = p[k][j] * keep - r.rate * m[k][j] / (sqrtf(v[k][j]) / r.root + a.eps);
                if (EIGHT && j < left[k]) {
                    const uint32_t mb = __float_as_uint(m[k][j]) & 0x7fffffffu, vb = __float_as_uint(v[k][j]) & 0x7fffffffu;
                    mmax = mb > mmax ? mb : mmax;
                    vmax = vb > vmax ? vb : vmax;
                }
            }
            const uint64_t number = (uint64_t)(T.first_block + block) * kBlock + lane * 4;
            uint32_t h[4];
            const bool noisy = T.p_bf16 && !T.master;
            if (EIGHT || noisy) {
                const uint32_t key = mix(r.key ^ (uint32_t)(number >> 32));
#pragma unroll
                for (int j = 0; j < 4; ++j) h[j] = mix(((uint32_t)number + j) ^ key);
            }
            if (T.p_bf16) {
                bf16_t q[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (noisy) {
                        uint32_t bits = __float_as_uint(p[k][j]);
                        if ((bits & 0x7f800000u) != 0x7f800000u) bits += mix(h[j] ^ 0xBB67AE85u) & 0xffffu;
                        q[j].bits = p[k][j] == p[k][j] ? (uint16_t)(bits >> 16) : (uint16_t)0x7fc0;
                    } else {
                        from_f32(q[j], p[k][j]);
                    }
                }
                store4(static_cast<bf16_t *>(T.p) + i, left[k], q);
                if (T.master) store4(T.master + i, left[k], p[k]);
            } else {
                store4(static_cast<float *>(T.p) + i, left[k], p[k]);
            }
            if (EIGHT) {
                const int Em = (int)(wave_max(mmax) >> 23), Ev = (int)(wave_max(vmax) >> 23);
                if (lane == 0) {
                    T.m_exp[block] = (uint8_t)Em;
                    T.v_exp[block] = (uint8_t)Ev;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t mb = __float_as_uint(m[k][j]);
                    const uint32_t c = encode<127>(mb & 0x7fffffffu, Em, h[j] & 0xffffu);
                    cm[k][j] = (uint8_t)(c | (c ? mb >> 24 & 128u : 0u));
                    cv[k][j] = (uint8_t)encode<255>(__float_as_uint(v[k][j]) & 0x7fffffffu, Ev, h[j] >> 16);
                }
                store4(static_cast<uint8_t *>(T.m) + i, left[k], cm[k]);
                store4(static_cast<uint8_t *>(T.v) + i, left[k], cv[k]);
            } else {
                store4(static_cast<float *>(T.m) + i, left[k], m[k]);
                store4(static_cast<float *>(T.v) + i, left[k], v[k]);
            }
        }
    }
}

// behind the step, on the same stream
__global__ void count_kernel(Step a)
{
    if (a.skip && !(fabsf(*a.norm) < INFINITY)) return;
    *a.step += 1;
}

// Squares are summed in fp64, which costs nothing beside the reads: no gradient's square overflows or is lost.
__global__ __launch_bounds__(kThreads) void norm_kernel(Step a)
{
    constexpr int kEach = kChunkBlocks / kWaves;
    __shared__ double lds[kWaves];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    double s = 0.;
    for (long chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        const Tensor T = a.tensors[a.owner[chunk]];
        const long first = (chunk - T.first_chunk) * kChunkBlocks + wave;
        float g[kEach][4];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const long i = (first + k * kWaves) * kBlock + lane * 4, n = T.n - i;
            load4_as(T.g, i, T.g_bf16, n < 0 ? 0 : n < 4 ? (int)n : 4, g[k]);
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) s += (double)g[k][j] * (double)g[k][j];
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) lds[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0) a.part[blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__global__ __launch_bounds__(64) void norm_sum_kernel(Step a, int parts)
{
    double s = 0.;
    for (int i = threadIdx.x; i < parts; i += 64) s += a.part[i];
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    if (threadIdx.x == 0) *a.norm_out = (float)sqrt(s);
}

__global__ __launch_bounds__(kThreads) void unpack_kernel(Step a)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (long chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        const Tensor T = a.tensors[a.owner[chunk]];
        const long first = (chunk - T.first_chunk) * kChunkBlocks + wave;
#pragma unroll
        for (int k = 0; k < kChunkBlocks / kWaves; ++k) {
            const long block = first + k * kWaves, i = block * kBlock + lane * 4, n = T.n - i, at = T.first_block * kBlock + i;
            if (block * kBlock >= T.n) break;
            const int left = n < 0 ? 0 : n < 4 ? (int)n : 4;
            uint8_t cm[4] = {}, cv[4] = {};
            if (a.m_out) load4(static_cast<const uint8_t *>(T.m) + i, left, cm);
            if (a.v_out) load4(static_cast<const uint8_t *>(T.v) + i, left, cv);
            const int em = T.m_exp[block], ev = T.v_exp[block];
            uint16_t m[4], v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) { // (zeros behind the tensor's end)
                m[j] = j < left ? (uint16_t)(__float_as_uint(decode<127>(cm[j] & 127, em)) >> 16 | (cm[j] & 128) << 8) : 0;
                v[j] = j < left ? (uint16_t)(__float_as_uint(decode<255>(cv[j], ev)) >> 16) : 0;
            }
            if (a.m_out) store4(a.m_out + at, 4, m);
            if (a.v_out) store4(a.v_out + at, 4, v);
        }
    }
}

bool desc_ok(const adamw_desc *d)
{
    return d && d->beta1 >= 0. && d->beta1 < 1. && d->beta2 >= 0. && d->beta2 < 1. && d->eps >= 0.f && d->eps < INFINITY &&
           (d->state_bits == 32 || d->state_bits == 8) && !(d->flags & ~(uint32_t)ADAMW_SKIP_NONFINITE);
}

// What the host knows of the list: places among all blocks and pieces of work.
int count(const adamw_desc *d, const adamw_tensor *t, int n, long *chunks, long *blocks)
{
    if (!desc_ok(d) || !t || n <= 0) return GSWA_EINVAL;
    *chunks = *blocks = 0;
    for (int i = 0; i < n; ++i) {
        if (t[i].n < 0) return GSWA_EINVAL;
        if (t[i].n > 1L << 40) return GSWA_EUNSUPPORTED;
        *chunks += (t[i].n + kChunk - 1) / kChunk;
        *blocks += (t[i].n + kBlock - 1) / kBlock;
        if (*chunks > 0x7fffffffL) return GSWA_EUNSUPPORTED;
    }
    return GSWA_OK;
}

uint64_t checksum(const adamw_plan_t *p)
{
    uint64_t h = 0x41646157u;
    for (uint64_t x : {(uint64_t)p->n_tensors, (uint64_t)p->chunks, (uint64_t)p->blocks, (uint64_t)reinterpret_cast<uintptr_t>(p->buffer),
                       (uint64_t)p->desc.state_bits, (uint64_t)p->desc.flags, p->desc.seed})
        h = (h ^ x) * 0x9E3779B97F4A7C15u, h ^= h >> 29;
    return h;
}

bool plan_ok(const adamw_plan_t *p) { return p && p->buffer && desc_ok(&p->desc) && p->check == checksum(p); }

void fill(const adamw_plan_t *p, Step *a)
{
    *a = Step{};
    char *b = static_cast<char *>(p->buffer);
    const Layout l = layout(p->n_tensors, p->chunks);
    a->tensors = reinterpret_cast<const Tensor *>(b);
    a->owner = reinterpret_cast<const int *>(b + l.owner);
    a->part = reinterpret_cast<double *>(b + l.part);
    a->counter = reinterpret_cast<unsigned *>(b + l.counter);
    a->chunks = p->chunks;
    a->beta1 = p->desc.beta1; a->beta2 = p->desc.beta2; a->eps = p->desc.eps;
    a->b1 = (float)a->beta1; a->b1c = (float)(1. - a->beta1); a->b2 = (float)a->beta2; a->b2c = (float)(1. - a->beta2);
    a->eight = p->desc.state_bits == 8;
    a->skip = (p->desc.flags & ADAMW_SKIP_NONFINITE) != 0;
    a->seed_lo = (uint32_t)p->desc.seed; a->seed_hi = (uint32_t)(p->desc.seed >> 32);
}

// No writable array may share a byte with another array of the list or with the buffer, but for a gradient shared by tensors.
int check_ranges(const adamw_desc *d, const adamw_tensor *t, int n, const void *buffer, size_t bytes)
{
    struct Piece {
        uintptr_t lo, hi;
        bool written;
    };
    try {
        std::vector<Piece> all;
        all.reserve((size_t)n * 7 + 1);
        const auto add = [&](const void *p, size_t size, bool written) {
            if (p && size) all.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + size, written});
        };
        const size_t state = d->state_bits == 8 ? 1 : 4;
        for (int i = 0; i < n; ++i) {
            const size_t k = (size_t)t[i].n;
            add(t[i].p, k * (t[i].p_dtype == GSWA_F32 ? 4 : 2), true);
            add(t[i].master, k * 4, true);
            add(t[i].m, k * state, true);
            add(t[i].v, k * state, true);
            add(t[i].m_exp, (k + kBlock - 1) / kBlock, true);
            add(t[i].v_exp, (k + kBlock - 1) / kBlock, true);
            add(t[i].g, k * (t[i].g_dtype == GSWA_F32 ? 4 : 2), false);
        }
        add(buffer, bytes, true);
        std::sort(all.begin(), all.end(), [](const Piece &a, const Piece &b) { return a.lo < b.lo; });
        uintptr_t end = 0, written_end = 0; // of what has begun so far, and of the written ones among it
        for (const Piece &x : all) {
            if (x.lo < (x.written ? end : written_end)) return GSWA_EINVAL;
            end = std::max(end, x.hi);
            if (x.written) written_end = std::max(written_end, x.hi);
        }
    } catch (...) { // (no host memory for the list)
        return GSWA_EUNSUPPORTED;
    }
    return GSWA_OK;
}

unsigned grid_of(long chunks, long most) { return (unsigned)(chunks < most ? chunks : most); }

} // namespace
} // namespace gswa

using namespace gswa;

#define AW_LAUNCHED()                                             \
    do {                                                          \
        const hipError_t e_ = hipGetLastError();                  \
        if (e_ != hipSuccess) return report_hip_error(e_);        \
    } while (0)

extern "C" {

int adamw_query_bytes(const adamw_desc *desc, const adamw_tensor *tensors, int32_t n_tensors, size_t *plan_bytes)
{
    long chunks, blocks;
    const int rc = count(desc, tensors, n_tensors, &chunks, &blocks);
    if (rc != GSWA_OK) return rc;
    if (plan_bytes) *plan_bytes = layout(n_tensors, chunks).bytes;
    return GSWA_OK;
}

int adamw_plan(const adamw_desc *desc, const adamw_tensor *tensors, int32_t n_tensors, void *buffer, adamw_plan_t *plan,
               void *hip_stream)
{
    long chunks, blocks;
    int rc = count(desc, tensors, n_tensors, &chunks, &blocks);
    if (rc != GSWA_OK) return rc;
    if (!buffer || !plan || !aligned_to(256, buffer)) return GSWA_EINVAL;
    const bool eight = desc->state_bits == 8;
    for (int i = 0; i < n_tensors; ++i) {
        const adamw_tensor &t = tensors[i];
        if ((t.p_dtype != GSWA_F32 && t.p_dtype != GSWA_BF16) || (t.g_dtype != GSWA_F32 && t.g_dtype != GSWA_BF16)) return GSWA_EINVAL;
        if (!(t.weight_decay >= 0.f && t.weight_decay < INFINITY) || (t.master && t.p_dtype != GSWA_BF16)) return GSWA_EINVAL;
        if (t.n == 0) continue;
        if (!t.p || !t.g || !t.m || !t.v || !t.m_exp != !eight || !t.v_exp != !eight) return GSWA_EINVAL;
        if (!aligned_to(16, t.p, t.master, t.g, t.m, t.v)) return GSWA_EINVAL;
    }
    const Layout l = layout(n_tensors, chunks);
    rc = check_ranges(desc, tensors, n_tensors, buffer, l.bytes);
    if (rc != GSWA_OK) return rc;
    *plan = adamw_plan_t{};
    plan->desc = *desc;
    plan->n_tensors = n_tensors; plan->chunks = chunks; plan->blocks = blocks; plan->buffer = buffer;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    char *b = static_cast<char *>(buffer);
    PlanArgs a;
    a.tensors = reinterpret_cast<Tensor *>(b);
    a.owner = reinterpret_cast<int *>(b + l.owner);
    a.counter = reinterpret_cast<unsigned *>(b + l.counter);
    long block = 0;
    int chunk = 0;
    for (int first = 0; first < n_tensors; first += kPerLaunch) {
        const int now = n_tensors - first < kPerLaunch ? n_tensors - first : kPerLaunch;
        a.first = first;
        for (int i = 0; i < now; ++i) {
            const adamw_tensor &t = tensors[first + i];
            a.t[i] = Tensor{t.p, t.master, t.g, t.m, t.v, t.m_exp, t.v_exp, t.n, block, chunk, t.weight_decay,
                            t.p_dtype == GSWA_BF16, t.g_dtype == GSWA_BF16};
            block += (t.n + kBlock - 1) / kBlock;
            chunk += (int)((t.n + kChunk - 1) / kChunk);
        }
        KernelTimer timer(K_ADAMW_PLAN, st);
        hipLaunchKernelGGL(plan_kernel, dim3(now), dim3(kThreads), 0, st, a);
        AW_LAUNCHED();
    }
    plan->check = checksum(plan);
    return GSWA_OK;
}

int adamw_norm(const adamw_plan_t *plan, float *norm, void *hip_stream)
{
    if (!plan_ok(plan) || !norm || !aligned_to(4, norm)) return GSWA_EINVAL;
    Step a;
    fill(plan, &a);
    a.norm_out = norm;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const unsigned grid = grid_of(plan->chunks, kNormBlocks);
    KernelTimer t(K_ADAMW_NORM, st);
    if (grid) {
        hipLaunchKernelGGL(norm_kernel, dim3(grid), dim3(kThreads), 0, st, a);
        AW_LAUNCHED();
    }
    hipLaunchKernelGGL(norm_sum_kernel, dim3(1), dim3(64), 0, st, a, (int)grid);
    AW_LAUNCHED();
    return GSWA_OK;
}

int adamw_step(const adamw_plan_t *plan, int64_t *step, float lr, const float *lr_scale, const float *norm, float max_norm,
               void *hip_stream)
{
    if (!plan_ok(plan) || !step || !aligned_to(8, step) || !aligned_to(4, lr_scale, norm)) return GSWA_EINVAL;
    if (!(lr >= 0.f && lr < INFINITY) || !(max_norm >= 0.f && max_norm < INFINITY)) return GSWA_EINVAL;
    if ((max_norm > 0.f || (plan->desc.flags & ADAMW_SKIP_NONFINITE)) && !norm) return GSWA_EINVAL;
    Step a;
    fill(plan, &a);
    a.step = step; a.lr = lr; a.lr_scale = lr_scale; a.norm = norm; a.max_norm = max_norm;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    KernelTimer t(K_ADAMW_STEP, st);
    if (plan->chunks) {
        const dim3 grid(grid_of(plan->chunks, 65536));
        if (a.eight) hipLaunchKernelGGL(step_kernel<true>, grid, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL(step_kernel<false>, grid, dim3(kThreads), 0, st, a);
        AW_LAUNCHED();
    }
    hipLaunchKernelGGL(count_kernel, dim3(1), dim3(1), 0, st, a);
    AW_LAUNCHED();
    return GSWA_OK;
}

int adamw_unpack(const adamw_plan_t *plan, void *m_out, void *v_out, void *hip_stream)
{
    if (!plan_ok(plan) || plan->desc.state_bits != 8 || (!m_out && !v_out) || !aligned_to(16, m_out, v_out)) return GSWA_EINVAL;
    const size_t bytes = (size_t)plan->blocks * kBlock * 2;
    if (overlaps_any(Range(m_out, bytes), Range(v_out, bytes), Range(plan->buffer, layout(plan->n_tensors, plan->chunks).bytes)) ||
        overlaps_any(Range(v_out, bytes), Range(plan->buffer, layout(plan->n_tensors, plan->chunks).bytes)))
        return GSWA_EINVAL;
    if (!plan->chunks) return GSWA_OK;
    Step a;
    fill(plan, &a);
    a.m_out = static_cast<uint16_t *>(m_out);
    a.v_out = static_cast<uint16_t *>(v_out);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    KernelTimer t(K_ADAMW_UNPACK, st);
    hipLaunchKernelGGL(unpack_kernel, dim3(grid_of(plan->chunks, 65536)), dim3(kThreads), 0, st, a);
    AW_LAUNCHED();
    return GSWA_OK;
}

} // extern "C"
