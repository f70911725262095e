// One AdamW step over many tensors (adamw.h): the plan, the norm of the gradients, the step, the read-back of
// 8-bit states, and the C ABI.
#include "../../include/adamw.h"
#include "args.h"
#include "common.h"
#include "mfma.h"
#include "profile.h"

#include <algorithm>
#include <type_traits>
#include <vector>

namespace gswa {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kBlock = 256;             // elements that share an exponent: four for each lane of a wavefront
constexpr int kNormBlocks = 1024;       // workgroups of the norm, at most
constexpr unsigned kAlone = 64;         // workgroups of the norm whose last one adds up what they leave (see norm_kernel)
constexpr int kStepBlocks = 65536;      // and of the others: a workgroup a piece of work up to 268 M elements (201 M, fp32: 1042 us; 4096 workgroups that
                                        // go on to further pieces 1127 us, 16384 1082 us)
constexpr int kGroups = 32;             // of the workgroups that are counted together (see last_of_all)
constexpr int kCounterStep = 32;        // counters stand in lines of their own

// Blocks of a piece of work that a wavefront takes at once.  Four for large lists, whose loads then keep the memory busy (201 M elements, steps one after another:
// fp32 states 1042 us, with two blocks 1075; 8-bit states and bf16 alone 458 and 482, the read-back 197 and 262; beside an fp32 copy 589 and 591; 7.7 M
// elements in 8 bits the same either way, 26).  One for lists that do not fill the card, where the time of one wavefront counts (8-bit states, 13 tensors of a
// layer, 25 K elements: 5.4 us, with four 7.1; 0.9 M elements in 468 tensors: 8.5, with four 9.7).
constexpr int kMany = 4;
constexpr long kSmall = 8192;           // blocks of a list that does not: up to 2 M elements, 8 workgroups a compute unit
constexpr long chunk_of(int each) { return (long)kBlock * kWaves * each; }

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

// The plan's buffer: [Tensor * n][tensor of every piece of work, int][partial sums of the norm][counters]
struct Layout {
    size_t owner, part, counter, bytes;
};
Layout layout(int n, long chunks)
{
    Layout l;
    l.owner = to_256((size_t)n * sizeof(Tensor));
    l.part = l.owner + to_256((size_t)chunks * sizeof(int));
    l.counter = l.part + to_256(kNormBlocks * sizeof(double));
    l.bytes = l.counter + to_256((kGroups + 1) * kCounterStep * sizeof(unsigned));
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
    int eight, skip, alone;
    uint32_t seed_key;
    uint16_t *m_out, *v_out;
};

constexpr int kPerLaunch = 40; // tensors whose places fit the arguments of one launch
struct PlanArgs {
    Tensor t[kPerLaunch];
    Tensor *tensors;
    int *owner;
    unsigned *counter;
    int first, each;
};

__global__ __launch_bounds__(kThreads) void plan_kernel(PlanArgs a)
{
    const Tensor &t = a.t[blockIdx.x];
    const int index = a.first + (int)blockIdx.x;
    if (threadIdx.x == 0) a.tensors[index] = t;
    if (index == 0 && threadIdx.x <= kGroups) a.counter[threadIdx.x * kCounterStep] = 0;
    const long chunk = chunk_of(a.each);
    const int chunks = (int)((t.n + chunk - 1) / chunk);
    for (int c = threadIdx.x; c < chunks; c += kThreads) a.owner[t.first_chunk + c] = index;
}

__host__ __device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x9E3779B9u;
    x ^= x >> 15;
    x *= 0x6A09E667u;
    return x ^ x >> 16;
}

// Four elements of a lane.  Pointers come out of the plan, so the compiler has to be told that they point at global memory; `base` is the same for a
// wavefront.  FULL: all four are there, one wide access; else the first `left` of them, zeros for the others.
template <typename E> using Global = __attribute__((address_space(1))) E;
template <typename E> struct Four;
template <> struct Four<float> { typedef u32x4 V; };
template <> struct Four<bf16_t> { typedef u32x2 V; };
template <> struct Four<uint8_t> { typedef uint32_t V; };
template <typename E, bool FULL> __device__ __forceinline__ typename Four<E>::V load4(const void *base, int lane, int left)
{
    typedef typename Four<E>::V V;
    if constexpr (FULL) {
        return ((const Global<V> *)base)[lane];
    } else {
        typedef typename std::conditional<sizeof(E) == 1, uint8_t, typename std::conditional<sizeof(E) == 2, uint16_t, uint32_t>::type>::type Bits;
        Bits e[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = j < left ? ((const Global<Bits> *)base)[lane * 4 + j] : Bits(0);
        V v;
        __builtin_memcpy(&v, e, sizeof(v));
        return v;
    }
}
template <typename E, bool FULL> __device__ __forceinline__ void store4(void *base, int lane, int left, typename Four<E>::V v)
{
    typedef typename Four<E>::V V;
    if constexpr (FULL) {
        ((Global<V> *)base)[lane] = v;
    } else {
        typedef typename std::conditional<sizeof(E) == 1, uint8_t, typename std::conditional<sizeof(E) == 2, uint16_t, uint32_t>::type>::type Bits;
        Bits e[4];
        __builtin_memcpy(e, &v, sizeof(v));
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) ((Global<Bits> *)base)[lane * 4 + j] = e[j];
    }
}
__device__ __forceinline__ void floats(u32x4 v, float (&f)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(v[j]);
}
__device__ __forceinline__ void floats(u32x2 v, float (&f)[4])
{
    f[0] = bf16_lo(v[0]); f[1] = bf16_hi(v[0]);
    f[2] = bf16_lo(v[1]); f[3] = bf16_hi(v[1]);
}
__device__ __forceinline__ u32x4 patterns(const float (&f)[4])
{
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
}
template <typename E> __device__ __forceinline__ const void *at(const void *p, long i) { return static_cast<const char *>(p) + i * (long)sizeof(E); }
template <typename E> __device__ __forceinline__ void *at(void *p, long i) { return static_cast<char *>(p) + i * (long)sizeof(E); }

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

// Codes of a block.  Its exponent is the same for a wavefront (for half of one where it is read back), `base` the pattern (upper 12 bits) of code 0.  Codes
// and patterns fit 16 bits, so two elements go through each operation: elements 0 and 2 of a lane in one register, 1 and 3 in another.  (A step with 8-bit
// states and bf16 parameters without a copy is bound by its operations: 75 an element so, 94 with one element at a time.  201 M elements with bf16
// gradients: 456 to 474 us, 514 to 519 before; 7.7 M: 26 us, 30.)
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 pair(uint32_t v) { return __builtin_bit_cast(u16x2, v); }
__device__ __forceinline__ uint32_t word(u16x2 v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ u16x2 least(u16x2 a, uint16_t b) { return __builtin_elementwise_min(a, u16x2{b, b}); }
__device__ __forceinline__ u16x2 most_signed(u16x2 a, int16_t b) // (patterns below 0 are met where a block holds next to nothing)
{
    return __builtin_bit_cast(u16x2, __builtin_elementwise_max(__builtin_bit_cast(i16x2, a), i16x2{b, b}));
}
template <int TOP> __device__ __forceinline__ u16x2 base_of(int E)
{
    const uint16_t base = (uint16_t)(8 * (E + 1) - TOP);
    return u16x2{base, base};
}
// 0 for 0, 1 for anything else (of the least with a plain 1 the compiler would make comparisons and choices, element by element)
__device__ __forceinline__ u16x2 some(u16x2 a)
{
    uint32_t ones = 0x00010001u;
    asm("" : "+s"(ones));
    return __builtin_elementwise_min(a, pair(ones));
}
__device__ __forceinline__ uint32_t upper_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// What four codes stand for, as bf16 patterns: elements 0 and 2, 1 and 3.
__device__ __forceinline__ uint32_t decode(uint32_t codes, u16x2 base) // the magnitudes
{
    const u16x2 c = pair(codes);
    return word(most_signed(c + base, 1) * some(c)) << 4;
}
__device__ __forceinline__ u32x2 decode_m(uint32_t codes, int E)
{
    const u16x2 base = base_of<127>(E);
    const u32x2 q = {decode(codes & 0x007f007fu, base) | (codes << 8 & 0x80008000u), decode(codes >> 8 & 0x007f007fu, base) | (codes & 0x80008000u)};
    return E == 255 ? u32x2{0x7fc07fc0u, 0x7fc07fc0u} : q;
}
__device__ __forceinline__ u32x2 decode_v(uint32_t codes, int E)
{
    const u16x2 base = base_of<255>(E);
    const u32x2 q = {decode(codes & 0x00ff00ffu, base), decode(codes >> 8 & 0x00ff00ffu, base)};
    return E == 255 ? u32x2{0x7fc07fc0u, 0x7fc07fc0u} : q;
}
__device__ __forceinline__ void as_floats(u32x2 q, float (&f)[4])
{
    f[0] = bf16_lo(q[0]); f[2] = bf16_hi(q[0]);
    f[1] = bf16_lo(q[1]); f[3] = bf16_hi(q[1]);
}
__device__ __forceinline__ u32x2 in_order(u32x2 q) // four bf16 as they lie in memory
{
    return u32x2{__builtin_amdgcn_perm(q[1], q[0], 0x05040100u), upper_halves(q[0], q[1])};
}

// bits + 16 times the lower or the upper half of h
__device__ __forceinline__ uint32_t add_lower(uint32_t bits, uint32_t h)
{
    uint32_t r;
    asm("v_mad_u32_u16 %0, %1, 16, %2" : "=v"(r) : "v"(h), "v"(bits));
    return r;
}
__device__ __forceinline__ uint32_t add_upper(uint32_t bits, uint32_t h)
{
    uint32_t r;
    asm("v_mad_u32_u16 %0, %1, 16, %2 op_sel:[1,0,0,0]" : "=v"(r) : "v"(h), "v"(bits));
    return r;
}

// m's codes, the low 16 bits of h against what is cut off, and v's, the high ones (what is not 0 is not stored as 0).  Signs go along: nothing but a NaN
// reaches them by the sum, and its block has E = 255.
__device__ __forceinline__ uint32_t encode_m(const float (&m)[4], int E, const uint32_t (&h)[4])
{
    const u16x2 base = base_of<127>(E);
    const uint16_t most = E == 254 ? 126 : 127;
    uint32_t t[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) t[j] = add_lower(__float_as_uint(m[j]), h[j]);
    const auto codes = [&](uint32_t x) {
        const u16x2 T = pair(x >> 4 & 0x07ff07ffu), c = least(most_signed(T - base, 0), most) * some(T);
        return word(pair(x >> 8 & 0x00800080u) * some(c) + c);
    };
    const uint32_t w = codes(upper_halves(t[0], t[2])) | codes(upper_halves(t[1], t[3])) << 8;
    return E == 255 ? 0u : w;
}
__device__ __forceinline__ uint32_t encode_v(const float (&v)[4], int E, const uint32_t (&h)[4])
{
    const u16x2 base = base_of<255>(E);
    const uint16_t most = E == 254 ? 254 : 255;
    uint32_t t[4], held[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t bits = __float_as_uint(v[j]);
        uint32_t one = 1u;
        asm("" : "+s"(one));
        t[j] = add_upper(bits, h[j]);
        held[j] = bits < one ? bits : one;
    }
    const auto codes = [&](uint32_t x, uint32_t held) {
        const u16x2 T = most_signed(pair(x >> 4 & 0x07ff07ffu), 1);
        return word(least(most_signed(T - base, 1), most) * pair(held));
    };
    const uint32_t w = codes(upper_halves(t[0], t[2]), held[0] | held[2] << 16) | codes(upper_halves(t[1], t[3]), held[1] | held[3] << 16) << 8;
    return E == 255 ? 0u : w;
}

// sqrt to a unit of its last place, of subnormal numbers too (the instruction takes those for 0)
__device__ __forceinline__ float root_of(float v)
{
    const bool small = v < 0x1p-96f;
    const float s = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v);
    return small ? s * 0x1p-32f : s;
}

// What a step needs of its number and rates, the same for all elements.
struct Rates {
    float lr, rate, root, clip; // learning rate; over 1 - beta1^t; 1 / sqrt(1 - beta2^t); factor of the gradients
    uint32_t key;
};
__device__ __forceinline__ Rates rates_of(const Step &a, float norm)
{
    const uint64_t steps = (uint64_t)*a.step;
    const uint32_t t_lo = __builtin_amdgcn_readfirstlane((uint32_t)steps), t_hi = __builtin_amdgcn_readfirstlane((uint32_t)(steps >> 32));
    const uint64_t t = ((uint64_t)t_hi << 32 | t_lo) + 1;
    double b = 1., f = threadIdx.x & 1 ? a.beta2 : a.beta1; // beta^t by squares: of beta1 in the even lanes, of beta2 in the odd ones
    for (uint64_t e = t; e; e >>= 1) {
        if (e & 1) b *= f;
        f *= f;
    }
    const int rest = __float_as_int((float)(1. - b));
    Rates r;
    r.lr = a.lr_scale ? a.lr * *a.lr_scale : a.lr;
    r.rate = r.lr / __int_as_float(__builtin_amdgcn_readlane(rest, 0));
    r.root = 1.f / sqrtf(__int_as_float(__builtin_amdgcn_readlane(rest, 1)));
    r.clip = a.max_norm > 0.f && norm > a.max_norm ? a.max_norm / norm : 1.f;
    r.key = mix(mix(a.seed_key ^ (uint32_t)(t >> 32)) ^ (uint32_t)t);
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

// Whether this workgroup is the last of its launch to come here (one thread of each does, when it needs nothing more that the last one changes).  Arrivals at
// one address take 15 ns each, whatever they overlap with, so those of a large launch are counted in 32 groups first (a step over 468 tensors, 792 workgroups:
// 14.8 -> 9.1 us).  Nothing but the count is handed over, so no order of memory is asked for.  Counters are left at 0 for the next launch.
__device__ __forceinline__ bool arrived_last(unsigned *counter, unsigned all)
{
    if (__hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != all - 1) return false;
    *counter = 0;
    return true;
}
__device__ __forceinline__ bool last_of_all(unsigned *counters)
{
    if (gridDim.x <= 2 * kGroups) return arrived_last(counters, gridDim.x);
    const unsigned group = blockIdx.x % kGroups, members = (gridDim.x - group + kGroups - 1) / kGroups;
    return arrived_last(counters + (1 + group) * kCounterStep, members) && arrived_last(counters, kGroups);
}

enum { kP32 = 0, kP16 = 1, kPBoth = 2 }; // the parameter: fp32; bf16; bf16 with an fp32 copy

// N blocks of a tensor in a row; all of their loads first.
template <int P, typename G, bool EIGHT, int N, bool FULL>
__device__ __forceinline__ void step_blocks(const Step &a, const Rates &r, const Tensor &T, long first, int lane)
{
    typedef typename std::conditional<P == kP16, bf16_t, float>::type Held; // what the parameter is read from
    typename Four<G>::V g4[N];
    typename Four<Held>::V p4[N];
    u32x4 m4[N], v4[N];
    uint32_t cm[N], cv[N];
    int em[N], ev[N], left[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const long block = first + k, i = block * kBlock;
        const long n = T.n - i - lane * 4;
        left[k] = FULL ? 4 : n < 0 ? 0 : n < 4 ? (int)n : 4;
        g4[k] = load4<G, FULL>(at<G>(T.g, i), lane, left[k]);
        p4[k] = load4<Held, FULL>(at<Held>(P == kPBoth ? (const void *)T.master : T.p, i), lane, left[k]);
        if constexpr (EIGHT) {
            cm[k] = load4<uint8_t, FULL>(at<uint8_t>(T.m, i), lane, left[k]);
            cv[k] = load4<uint8_t, FULL>(at<uint8_t>(T.v, i), lane, left[k]);
            em[k] = ((const Global<uint8_t> *)T.m_exp)[block];
            ev[k] = ((const Global<uint8_t> *)T.v_exp)[block];
        } else {
            m4[k] = load4<float, FULL>(at<float>(T.m, i), lane, left[k]);
            v4[k] = load4<float, FULL>(at<float>(T.v, i), lane, left[k]);
        }
    }
    const float keep = 1.f - r.lr * T.decay;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const long block = first + k, i = block * kBlock;
        float g[4], p[4], m[4], v[4];
        floats(g4[k], g);
        floats(p4[k], p);
        if constexpr (EIGHT) {
            as_floats(decode_m(cm[k], __builtin_amdgcn_readfirstlane(em[k])), m);
            as_floats(decode_v(cv[k], __builtin_amdgcn_readfirstlane(ev[k])), v);
        } else {
            floats(m4[k], m);
            floats(v4[k], v);
        }
        uint32_t mmax = 0, vmax = 0; // (elements behind the tensor's end are zeros throughout)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            moments(a, g[j] * r.clip, m[j], v[j]);
            // (quotient and root to a unit of their last places: the update is some 1e-3 of the parameter)
            p[j] = p[j] * keep - r.rate * m[j] * __builtin_amdgcn_rcpf(root_of(v[j]) * r.root + a.eps);
            if constexpr (EIGHT) {
                const uint32_t mb = __float_as_uint(m[j]) & 0x7fffffffu, vb = __float_as_uint(v[j]); // (v is not negative, but for a NaN)
                mmax = mb > mmax ? mb : mmax;
                vmax = vb > vmax ? vb : vmax;
            }
        }
        uint32_t h[4];
        if constexpr (EIGHT || P == kP16) {
            const uint64_t number = (uint64_t)(T.first_block + block) * kBlock; // of the block's first element: no block crosses 2^32
            const uint32_t key = mix(r.key ^ (uint32_t)(number >> 32)), low = (uint32_t)number + lane * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) h[j] = mix((low + j) ^ key);
        }
        if constexpr (P == kP16) {
            uint32_t q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) { // (an infinity stays one: its 16 bits behind are 0)
                const uint32_t bits = __float_as_uint(p[j]) + (mix(h[j] ^ 0xBB67AE85u) & 0xffffu);
                q[j] = p[j] == p[j] ? bits : 0x7fc00000u;
            }
            store4<bf16_t, FULL>(at<bf16_t>(T.p, i), lane, left[k], u32x2{q[0] >> 16 | (q[1] & 0xffff0000u), q[2] >> 16 | (q[3] & 0xffff0000u)});
        } else if constexpr (P == kPBoth) {
            store4<bf16_t, FULL>(at<bf16_t>(T.p, i), lane, left[k], u32x2{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3])});
            store4<float, FULL>(at<float>((void *)T.master, i), lane, left[k], patterns(p));
        } else {
            store4<float, FULL>(at<float>(T.p, i), lane, left[k], patterns(p));
        }
        if constexpr (EIGHT) {
            const int Em = __builtin_amdgcn_readfirstlane(wave_max(mmax) >> 23), Ev = __builtin_amdgcn_readfirstlane(wave_max(vmax) >> 23) & 255;
            if (lane == 0) {
                ((Global<uint8_t> *)T.m_exp)[block] = (uint8_t)Em;
                ((Global<uint8_t> *)T.v_exp)[block] = (uint8_t)Ev;
            }
            store4<uint8_t, FULL>(at<uint8_t>(T.m, i), lane, left[k], encode_m(m, Em, h));
            store4<uint8_t, FULL>(at<uint8_t>(T.v, i), lane, left[k], encode_v(v, Ev, h));
        } else {
            store4<float, FULL>(at<float>(T.m, i), lane, left[k], patterns(m));
            store4<float, FULL>(at<float>(T.v, i), lane, left[k], patterns(v));
        }
    }
}

// The N blocks of a piece of work that a wavefront takes: all at once where they are whole, one by one at a tensor's end.
template <int N, typename F, typename H> __device__ __forceinline__ void each_block(const Tensor &T, long chunk, int wave, F whole, H partly)
{
    const long first = ((chunk - T.first_chunk) * kWaves + wave) * N;
    if ((first + N) * kBlock <= T.n) return whole(first);
    for (long b = first; b < first + N; ++b)
        if (b * kBlock < T.n) partly(b);
}

// Bound by memory, but with 8-bit states and no fp32 copy: 10 to 30 bytes an element against 75 operations with 8-bit states, half of that with 32.  A wavefront has all loads of
// N blocks in flight together; a block's largest magnitude comes from exchanges between its lanes.
template <bool EIGHT, int N> __global__ __launch_bounds__(kThreads) void step_kernel(Step a)
{
    const float norm = a.norm ? *a.norm : 0.f;
    if (a.skip && !(fabsf(norm) < INFINITY)) return;
    const Rates r = rates_of(a, norm);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (long chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        const Tensor T = a.tensors[a.owner[chunk]];
        const auto go = [&](auto p, auto g) {
            typedef decltype(g) G;
            constexpr int P = decltype(p)::value;
            each_block<N>(T, chunk, wave, [&](long b) { step_blocks<P, G, EIGHT, N, true>(a, r, T, b, lane); },
                          [&](long b) { step_blocks<P, G, EIGHT, 1, false>(a, r, T, b, lane); });
        };
        const auto by_gradient = [&](auto p) {
            if (T.g_bf16) go(p, bf16_t{});
            else go(p, float{});
        };
        if (!T.p_bf16) by_gradient(std::integral_constant<int, kP32>{});
        else if (T.master) by_gradient(std::integral_constant<int, kPBoth>{});
        else by_gradient(std::integral_constant<int, kP16>{});
    }
    __syncthreads(); // (all wavefronts of this workgroup have read the number of steps, with all others that have come here)
    if (threadIdx.x == 0 && last_of_all(a.counter)) *a.step += 1;
}

__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double lds[kWaves];
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Four squares are added in fp32 and go on in fp64, so no sum over many elements loses digits; where a square could overflow or be lost (the sum of four
// is out of bounds or hardly above 0) they are formed in fp64 too.  What the workgroups leave is added in their order: by the last of a few of them, by a launch
// of its own after many.  For the last one each has to write its caches back first, which many wait for: norm and step of 36 workgroups 8.8 us, with the second
// launch 11.6; of 144 both 11.6; the norm of 792 alone 16 and 10.
template <int N> __global__ __launch_bounds__(kThreads) void norm_kernel(Step a)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    double s = 0.;
    const auto add = [&](const float (&g)[4]) {
        const float q = (g[0] * g[0] + g[1] * g[1]) + (g[2] * g[2] + g[3] * g[3]);
        if (q > 1e-30f && q < 3e38f) {
            s += (double)q;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) s += (double)g[j] * (double)g[j];
        }
    };
    for (long chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        const Tensor T = a.tensors[a.owner[chunk]];
        const auto go = [&](auto g) {
            typedef decltype(g) G;
            each_block<N>(T, chunk, wave,
                          [&](long b) {
                              typename Four<G>::V v[N];
#pragma unroll
                              for (int k = 0; k < N; ++k) v[k] = load4<G, true>(at<G>(T.g, (b + k) * kBlock), lane, 4);
#pragma unroll
                              for (int k = 0; k < N; ++k) {
                                  float f[4];
                                  floats(v[k], f);
                                  add(f);
                              }
                          },
                          [&](long b) {
                              const long n = T.n - b * kBlock - lane * 4;
                              float f[4];
                              floats(load4<G, false>(at<G>(T.g, b * kBlock), lane, n < 0 ? 0 : n < 4 ? (int)n : 4), f);
                              add(f);
                          });
        };
        if (T.g_bf16) go(bf16_t{});
        else go(float{});
    }
    s = block_sum(s);
    if (threadIdx.x == 0) a.part[blockIdx.x] = s;
    if (!a.alone) return;
    __shared__ int last;
    if (threadIdx.x == 0) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
        last = arrived_last(a.counter, gridDim.x);
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    }
    __syncthreads();
    if (!last) return;
    s = block_sum(threadIdx.x < gridDim.x ? a.part[threadIdx.x] : 0.);
    if (threadIdx.x == 0) *a.norm_out = (float)sqrt(s);
}

__global__ __launch_bounds__(kThreads) void norm_sum_kernel(Step a, int parts)
{
    double s = 0.;
    for (int i = threadIdx.x; i < parts; i += kThreads) s += a.part[i];
    s = block_sum(s);
    if (threadIdx.x == 0) *a.norm_out = (float)sqrt(s);
}

// N whole blocks: two at a time, eight codes a lane, half a wavefront a block (a single one with four a lane).
template <int N, typename Decode>
__device__ __forceinline__ void unpack_whole(const void *codes, const uint8_t *exp, uint16_t *out, long block, int lane, Decode decode)
{
    if constexpr (N == 1) {
        ((Global<u32x2> *)out)[lane] = in_order(decode(((const Global<uint32_t> *)at<uint8_t>(codes, block * kBlock))[lane], ((const Global<uint8_t> *)exp)[block]));
    } else {
        u32x2 c[N / 2];
        int E[N / 2];
#pragma unroll
        for (int k = 0; k < N / 2; ++k) {
            c[k] = ((const Global<u32x2> *)at<uint8_t>(codes, (block + 2 * k) * kBlock))[lane];
            E[k] = ((const Global<uint8_t> *)exp)[block + 2 * k + lane / 32];
        }
#pragma unroll
        for (int k = 0; k < N / 2; ++k) {
            const u32x2 lo = in_order(decode(c[k][0], E[k])), hi = in_order(decode(c[k][1], E[k]));
            ((Global<u32x4> *)at<uint16_t>((void *)out, 2 * k * kBlock))[lane] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
}
// The block at a tensor's end, zeros behind it.
template <typename Decode> __device__ __forceinline__ void unpack_end(const void *codes, const uint8_t *exp, uint16_t *out, long block, long n, int lane, Decode decode)
{
    const long over = n - block * kBlock - lane * 4;
    const int left = over < 0 ? 0 : over < 4 ? (int)over : 4;
    u32x2 q = in_order(decode(load4<uint8_t, false>(at<uint8_t>(codes, block * kBlock), lane, left), ((const Global<uint8_t> *)exp)[block]));
    q[0] &= left > 1 ? 0xffffffffu : left ? 0x0000ffffu : 0u; // (in a block of NaN they are not)
    q[1] &= left > 3 ? 0xffffffffu : left > 2 ? 0x0000ffffu : 0u;
    ((Global<u32x2> *)out)[lane] = q;
}

template <int N> __global__ __launch_bounds__(kThreads) void unpack_kernel(Step a)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const auto of_m = [](uint32_t codes, int E) { return decode_m(codes, E); };
    const auto of_v = [](uint32_t codes, int E) { return decode_v(codes, E); };
    for (long chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        const Tensor T = a.tensors[a.owner[chunk]];
        each_block<N>(T, chunk, wave,
                   [&](long b) {
                       const long to = (T.first_block + b) * kBlock;
                       if (a.m_out) unpack_whole<N>(T.m, T.m_exp, a.m_out + to, b, lane, of_m);
                       if (a.v_out) unpack_whole<N>(T.v, T.v_exp, a.v_out + to, b, lane, of_v);
                   },
                   [&](long b) {
                       const long to = (T.first_block + b) * kBlock;
                       if (a.m_out) unpack_end(T.m, T.m_exp, a.m_out + to, b, T.n, lane, of_m);
                       if (a.v_out) unpack_end(T.v, T.v_exp, a.v_out + to, b, T.n, lane, of_v);
                   });
    }
}

bool desc_ok(const adamw_desc *d)
{
    return d && d->beta1 >= 0. && d->beta1 < 1. && d->beta2 >= 0. && d->beta2 < 1. && (d->eps == 0.f || d->eps >= 0x1p-126f) && d->eps < INFINITY &&
           (d->state_bits == 32 || d->state_bits == 8) && !(d->flags & ~(uint32_t)ADAMW_SKIP_NONFINITE);
}

// What the host knows of the list: places among all blocks and pieces of work.
int count(const adamw_desc *d, const adamw_tensor *t, int n, int *each, long *chunks, long *blocks)
{
    if (!desc_ok(d) || !t || n <= 0) return GSWA_EINVAL;
    *chunks = *blocks = 0;
    for (int i = 0; i < n; ++i) {
        if (t[i].n < 0) return GSWA_EINVAL;
        if (t[i].n > 1L << 40) return GSWA_EUNSUPPORTED;
        *blocks += (t[i].n + kBlock - 1) / kBlock;
        if (*blocks > 1L << 32) return GSWA_EUNSUPPORTED; // (2^40 elements)
    }
    *each = *blocks <= kSmall ? 1 : kMany;
    for (int i = 0; i < n; ++i) *chunks += (t[i].n + chunk_of(*each) - 1) / chunk_of(*each);
    return *chunks > 0x7fffffffL ? GSWA_EUNSUPPORTED : GSWA_OK;
}

uint64_t checksum(const adamw_plan_t *p)
{
    uint64_t h = 0x41646157u;
    for (uint64_t x : {(uint64_t)p->n_tensors, (uint64_t)p->each, (uint64_t)p->chunks, (uint64_t)p->blocks, (uint64_t)reinterpret_cast<uintptr_t>(p->buffer),
                       (uint64_t)p->desc.state_bits, (uint64_t)p->desc.flags, p->desc.seed})
        h = (h ^ x) * 0x9E3779B97F4A7C15u, h ^= h >> 29;
    return h;
}

// the plan's own memory, which no other argument of a call may lie in
Range buffer_of(const adamw_plan_t *p) { return Range(p->buffer, layout(p->n_tensors, p->chunks).bytes); }

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
    a->seed_key = mix(mix((uint32_t)(p->desc.seed >> 32) ^ 0x510E527Fu) ^ (uint32_t)p->desc.seed);
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

unsigned grid_of(long chunks, long most) { return (unsigned)(chunks < 1 ? 1 : chunks < most ? chunks : most); }

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
    int each;
    long chunks, blocks;
    const int rc = count(desc, tensors, n_tensors, &each, &chunks, &blocks);
    if (rc != GSWA_OK) return rc;
    if (plan_bytes) *plan_bytes = layout(n_tensors, chunks).bytes;
    return GSWA_OK;
}

int adamw_plan(const adamw_desc *desc, const adamw_tensor *tensors, int32_t n_tensors, void *buffer, adamw_plan_t *plan,
               void *hip_stream)
{
    int each;
    long chunks, blocks;
    int rc = count(desc, tensors, n_tensors, &each, &chunks, &blocks);
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
    plan->n_tensors = n_tensors; plan->each = each; plan->chunks = chunks; plan->blocks = blocks; plan->buffer = buffer;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    char *b = static_cast<char *>(buffer);
    PlanArgs a;
    a.tensors = reinterpret_cast<Tensor *>(b);
    a.owner = reinterpret_cast<int *>(b + l.owner);
    a.counter = reinterpret_cast<unsigned *>(b + l.counter);
    a.each = each;
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
            chunk += (int)((t.n + chunk_of(each) - 1) / chunk_of(each));
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
    if (!plan_ok(plan) || !norm || !aligned_to(4, norm) || overlaps_any(Range(norm, 4), buffer_of(plan))) return GSWA_EINVAL;
    Step a;
    fill(plan, &a);
    a.norm_out = norm;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const unsigned grid = grid_of(plan->chunks, kNormBlocks);
    a.alone = grid <= kAlone;
    {
        KernelTimer t(K_ADAMW_NORM, st);
        if (plan->each == 1) hipLaunchKernelGGL(norm_kernel<1>, dim3(grid), dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL(norm_kernel<kMany>, dim3(grid), dim3(kThreads), 0, st, a);
        AW_LAUNCHED();
    }
    if (a.alone) return GSWA_OK;
    KernelTimer t(K_ADAMW_NORM, st);
    hipLaunchKernelGGL(norm_sum_kernel, dim3(1), dim3(kThreads), 0, st, a, (int)grid);
    AW_LAUNCHED();
    return GSWA_OK;
}

int adamw_step(const adamw_plan_t *plan, int64_t *step, float lr, const float *lr_scale, const float *norm, float max_norm,
               void *hip_stream)
{
    if (!plan_ok(plan) || !step || !aligned_to(8, step) || !aligned_to(4, lr_scale, norm)) return GSWA_EINVAL;
    if (overlaps_any(Range(step, 8), Range(norm, 4), Range(lr_scale, 4)) || overlaps_any(buffer_of(plan), Range(step, 8), Range(norm, 4), Range(lr_scale, 4)))
        return GSWA_EINVAL;
    if (!(lr >= 0.f && lr < INFINITY) || !(max_norm >= 0.f && max_norm < INFINITY)) return GSWA_EINVAL;
    if ((max_norm > 0.f || (plan->desc.flags & ADAMW_SKIP_NONFINITE)) && !norm) return GSWA_EINVAL;
    Step a;
    fill(plan, &a);
    a.step = step; a.lr = lr; a.lr_scale = lr_scale; a.norm = norm; a.max_norm = max_norm;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    KernelTimer t(K_ADAMW_STEP, st);
    const dim3 grid(grid_of(plan->chunks, kStepBlocks));
    if (plan->each == 1) {
        if (a.eight) hipLaunchKernelGGL((step_kernel<true, 1>), grid, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL((step_kernel<false, 1>), grid, dim3(kThreads), 0, st, a);
    } else {
        if (a.eight) hipLaunchKernelGGL((step_kernel<true, kMany>), grid, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL((step_kernel<false, kMany>), grid, dim3(kThreads), 0, st, a);
    }
    AW_LAUNCHED();
    return GSWA_OK;
}

int adamw_unpack(const adamw_plan_t *plan, void *m_out, void *v_out, void *hip_stream)
{
    if (!plan_ok(plan) || plan->desc.state_bits != 8 || (!m_out && !v_out) || !aligned_to(16, m_out, v_out)) return GSWA_EINVAL;
    const size_t bytes = (size_t)plan->blocks * kBlock * 2;
    if (overlaps_any(Range(m_out, bytes), Range(v_out, bytes), buffer_of(plan)) ||
        overlaps_any(Range(v_out, bytes), buffer_of(plan)))
        return GSWA_EINVAL;
    if (!plan->chunks) return GSWA_OK;
    Step a;
    fill(plan, &a);
    a.m_out = static_cast<uint16_t *>(m_out);
    a.v_out = static_cast<uint16_t *>(v_out);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    KernelTimer t(K_ADAMW_UNPACK, st);
    const dim3 grid(grid_of(plan->chunks, kStepBlocks));
    if (plan->each == 1) hipLaunchKernelGGL(unpack_kernel<1>, grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL(unpack_kernel<kMany>, grid, dim3(kThreads), 0, st, a);
    AW_LAUNCHED();
    return GSWA_OK;
}

} // extern "C"
