// Learned relative position bias by buckets of offsets, with its gradient (relpos.h): the kernels and the C ABI.
#include "../../include/relpos.h"
#include "args.h"
#include "common.h"
#include "mfma.h"
#include "profile.h"

#include <math.h>
#include <type_traits>
#include <vector>

namespace gswa {
namespace {

constexpr int kThreads = 256;
constexpr int kMostRows = 32;     // rows of a tile of the gradient, at most (64 lanes hold what leaves it)
constexpr int kMostFwdRows = 64;  // rows of a tile of the bias, at most

struct Args {
    const void *table, *dout;
    void *out;
    float *dtable, *part; // part: [heads][slices][buckets], null where one workgroup has all of a head
    long ld;
    int heads, batch, q, k, start, window, buckets, bidirectional, causal, accumulate, n;
    int rows, grad_rows;  // of a tile of the bias and of the gradient
    int spread;           // logarithm of the XCDs over which the bands of rows of the bias are spread
    int slices;           // workgroups of a head in the sums of the gradient
    int edges[RELPOS_MAX_EDGES];
};

// ---- the table of a window --------------------------------------------------------------------------------------------------------
// A few thousand values: what counts is the chain of dependent steps.  The buckets of the 2 M - 1 offsets of an axis are found side by side and kept
// in LDS; a pair of buckets is a rectangle of offsets, which one workgroup sums.

template <typename T> __global__ __launch_bounds__(kThreads) void window_fwd_kernel(Args a)
{
    __shared__ int axis[128];
    const int side = 2 * a.window - 1, total = side * side * a.heads, B = 2 * (a.n + 1);
    if ((int)threadIdx.x < side) {
        const int r = a.window - 1 - (int)threadIdx.x, d = r < 0 ? -r : r; // key - query of the offset query - key = threadIdx.x - (M - 1)
        int n = 0;
        for (int e = 0; e < a.n; ++e) n += a.edges[e] <= d;
        axis[threadIdx.x] = n + (r > 0 ? a.n + 1 : 0);
    }
    __syncthreads();
    const int e = blockIdx.x * kThreads + threadIdx.x;
    if (e >= total) return;
    const int offset = e / a.heads, h = e - offset * a.heads, dr = offset / side, dc = offset - dr * side;
    static_cast<T *>(a.out)[e] = static_cast<const T *>(a.table)[((long)axis[dr] * B + axis[dc]) * a.heads + h];
}

// The places [lo, hi) of an axis of the table whose offsets fall into bucket b.
__device__ __forceinline__ void bucket_places(const Args &a, int b, int &lo, int &hi)
{
    const int M = a.window, behind = b > a.n, n = behind ? b - a.n - 1 : b;
    const int from = n ? a.edges[n - 1] : behind, to = n < a.n ? a.edges[n] - 1 : M - 1; // distances; key behind the query: r > 0
    const int first = from, last = to < M - 1 ? to : M - 1;
    // place = query - key + M - 1 = M - 1 - r
    lo = behind ? M - 1 - last : M - 1 + first;
    hi = behind ? M - first : M + last;
    if (first > last) lo = hi = 0;
}

// A workgroup per pair of buckets: its threads take the heads of as many places at once as there is room for, places in their order; the threads of
// a head are summed in their order.
__global__ __launch_bounds__(kThreads) void window_bwd_kernel(Args a)
{
    __shared__ float lds[kThreads];
    const int B = 2 * (a.n + 1), side = 2 * a.window - 1, pair = blockIdx.x;
    int r0, r1, c0, c1;
    bucket_places(a, pair / B, r0, r1);
    bucket_places(a, pair % B, c0, c1);
    const int heads = a.heads < kThreads ? a.heads : kThreads, width = c1 - c0, places = (r1 - r0) * width;
    const int slots = kThreads / heads, slot = threadIdx.x / heads, used = slots < places ? slots : places;
    const float *dout = static_cast<const float *>(a.dout);
    for (int h0 = 0; h0 < a.heads; h0 += heads) {
        const int h = h0 + threadIdx.x % heads;
        float s = 0.f;
        if (slot < slots && h < a.heads)
#pragma unroll 4
            for (int p = slot; p < places; p += slots) {
                const int r = p / width;
                s += dout[((long)(r0 + r) * side + c0 + (p - r * width)) * a.heads + h];
            }
        lds[threadIdx.x] = s;
        __syncthreads();
        if ((int)threadIdx.x < heads && h < a.heads) {
            s = 0.f;
            for (int i = 0; i < used; ++i) s += lds[i * heads + threadIdx.x];
            float *out = a.dtable + (long)pair * a.heads + h;
            *out = a.accumulate ? *out + s : s;
        }
        __syncthreads();
    }
}

// ---- the bias of a sequence -------------------------------------------------------------------------------------------------------
// Bound by the writes of the bias.  out[h, i, j] depends on j - i: a tile of R rows and C columns has R + C - 1 different values, which go to LDS
// once.  A lane writes the same V columns of every row; from one row to the next its
// values move up by one place, so a row costs a lane one value out of LDS, a shift of its vector and one wide store.

template <typename T> struct Vector;
template <> struct Vector<bf16_t> {
    static constexpr int V = 8;
    typedef uint16_t Bits;
    uint4 w;
    __device__ __forceinline__ void shift(uint32_t v)
    {
        w.w = __builtin_amdgcn_alignbit(w.w, w.z, 16);
        w.z = __builtin_amdgcn_alignbit(w.z, w.y, 16);
        w.y = __builtin_amdgcn_alignbit(w.y, w.x, 16);
        w.x = w.x << 16 | v;
    }
    __device__ __forceinline__ uint32_t at(int i) const
    {
        const uint32_t u = i < 4 ? (i < 2 ? w.x : w.y) : (i < 6 ? w.z : w.w);
        return i & 1 ? u >> 16 : u & 0xffffu;
    }
    // 8 values from c + u on; c is a multiple of 8, values of 16, and u the same for all lanes
    static __device__ __forceinline__ Vector from(const Bits *values, int c, int u)
    {
        const uint32_t *p = reinterpret_cast<const uint32_t *>(values) + c / 2 + u / 2;
        const uint32_t x[5] = {p[0], p[1], p[2], p[3], p[4]};
        Vector v;
        v.w = u & 1 ? make_uint4(__builtin_amdgcn_alignbit(x[1], x[0], 16), __builtin_amdgcn_alignbit(x[2], x[1], 16), __builtin_amdgcn_alignbit(x[3], x[2], 16),
                                 __builtin_amdgcn_alignbit(x[4], x[3], 16))
                    : make_uint4(x[0], x[1], x[2], x[3]);
        return v;
    }
    static constexpr uint32_t kMinusInf = 0xff80u;
};
template <> struct Vector<float> {
    static constexpr int V = 4;
    typedef uint32_t Bits;
    uint4 w;
    __device__ __forceinline__ void shift(uint32_t v)
    {
        w.w = w.z;
        w.z = w.y;
        w.y = w.x;
        w.x = v;
    }
    __device__ __forceinline__ uint32_t at(int i) const { return i < 2 ? (i ? w.y : w.x) : (i == 2 ? w.z : w.w); }
    static __device__ __forceinline__ Vector from(const Bits *values, int c, int u)
    {
        const uint32_t *p = values + c + u;
        Vector v;
        v.w = make_uint4(p[0], p[1], p[2], p[3]);
        return v;
    }
    static constexpr uint32_t kMinusInf = 0xff800000u;
};

// Where a row starts.
enum {
    kAligned, // at a 128-byte line
    kJoined,  // anywhere, one row right behind the other
    kApart,   // anywhere, with something between them
    kSingle   // anywhere, one a head
};

// A line that is written in part costs more than its bytes, also if another instruction writes the rest soon after.  So neighbouring rows are one XCD's, and
// where rows do not start at lines, a lane's columns move with the row to where lines start and its vector is read out of LDS anew:
//   joined  forward; a row has the lines that start in it, the last one with the next row's first columns, whose values wait in `starts`, and one
//           instruction writes it (16 x 4096 rows of 4001 in bf16: 5.1 TB/s; with a row's own vectors and then what reaches over its end 4.4, with rows
//           as apart 4.3; rows of 4032 5.4)
//   apart   back to the line that the row starts in; elements before the first aligned vector and behind the last one are stored one by one, by a lane
//           each, of all rows at once
//   single  as apart, by the lanes that have them in a vector (one token against 8190 keys: 5.3 us, as apart 6.4)
template <typename T, int THREADS, int ROWS> __global__ __launch_bounds__(THREADS) void sequence_fwd_kernel(Args a)
{
    typedef Vector<T> Vec;
    typedef typename Vec::Bits Bits;
    constexpr int V = Vec::V, kColumns = THREADS * V, kLine = 128 / sizeof(T), kBefore = ROWS == kApart || ROWS == kSingle ? kLine : 0, kMore = ROWS == kAligned ? 0 : kLine;
    constexpr int kValues = kColumns + kMore + kMostFwdRows, kStarts = ROWS == kJoined ? kLine + kMostFwdRows : 0;
    __shared__ __align__(16) Bits values[kValues + kStarts + 4];
    [[maybe_unused]] const Bits *const starts = values + kValues;
    __shared__ Bits learned[2 * (RELPOS_MAX_EDGES + 1)];
    __shared__ int edges[2 * (RELPOS_MAX_EDGES + 1)]; // (behind the last edge none is ever reached)
    const int h = blockIdx.y;
    int top = 1; // the largest power of two up to n
    while (2 * top <= a.n) top *= 2;
    for (int b = threadIdx.x; b < a.buckets; b += THREADS) learned[b] = static_cast<const Bits *>(a.table)[(long)b * a.heads + h];
    for (int e = threadIdx.x; e < 2 * top; e += THREADS) edges[e] = e < a.n ? a.edges[e] : 0x7fffffff;
    const int tiles_k = (a.k + (kBefore ? kLine - 1 : 0) + kColumns - 1) / kColumns;
    const int bands = (a.q + a.rows - 1) / a.rows, per = (bands + (1 << a.spread) - 1) >> a.spread; // bands of rows, and those of an XCD (workgroups go to them in turn)
    const long tiles = (long)per * tiles_k << a.spread;
    for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const long t = tile >> a.spread;
        const int down = t >> 32 ? (int)(t / tiles_k) : (int)((uint32_t)t / (uint32_t)tiles_k), band = (int)(tile & ((1 << a.spread) - 1)) * per + down;
        if (band >= bands) continue;
        const int i0 = band * a.rows, j0 = (int)(t - (long)down * tiles_k) * kColumns;
        const int i1 = i0 + a.rows < a.q ? i0 + a.rows : a.q, R = i1 - i0;
        __syncthreads();
        // all of a thread's offsets are searched for side by side: one chain of a few reads of LDS, not one for each
        constexpr int kMine = (kValues + kStarts + THREADS - 1) / THREADS;
        const int lowest = j0 - kBefore - (i1 - 1) - a.start, count = kColumns + kMore + R - 1;
        const auto offset = [&](int x) { return kStarts && x >= kValues ? x - kValues - i1 - a.start : x + lowest; };
        int n[kMine];
#pragma unroll
        for (int k = 0; k < kMine; ++k) n[k] = 0;
        for (int step = top; step; step >>= 1) {
#pragma unroll
            for (int k = 0; k < kMine; ++k) {
                const int r = offset(threadIdx.x + k * THREADS), d = r < 0 ? -r : a.bidirectional ? r : 0;
                n[k] += edges[n[k] + step - 1] <= d ? step : 0;
            }
        }
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const int x = threadIdx.x + k * THREADS, r = offset(x);
            if (x < count || (kStarts && x >= kValues && x < kValues + kStarts))
                values[x] = a.causal && r > 0 ? (Bits)Vec::kMinusInf : learned[a.bidirectional && r > 0 ? n[k] + a.n + 1 : n[k]];
        }
        __syncthreads();
        const int c = threadIdx.x * V;
        Bits *const first = static_cast<Bits *>(a.out) + ((long)h * a.q + i0) * a.ld + j0; // the tile's corner
        // elements from the last line's start up to this row's column j0, which is a multiple of a line
        const auto into_line = [&](const Bits *row) { return (int)(reinterpret_cast<uintptr_t>(row) / sizeof(Bits)) & (kLine - 1); };
        if constexpr (ROWS == kAligned) {
            const int j = j0 + c;
            if (j >= a.k) continue;
            Vec v;
#pragma unroll
            for (int e = V - 1; e >= 0; --e) v.shift(values[c + R - 1 + e]);
            Bits *row = first + c;
            if (j + V <= a.k) {
#pragma unroll 4
                for (int i = R - 1;; --i) {
                    __builtin_memcpy(row, &v.w, 16);
                    if (i == 0) break;
                    row += a.ld;
                    v.shift(values[c + i - 1]);
                }
            } else {
                for (int i = R - 1;; --i) {
#pragma unroll
                    for (int e = 0; e < V - 1; ++e)
                        if (j + e < a.k) row[e] = (Bits)v.at(e);
                    if (i == 0) break;
                    row += a.ld;
                    v.shift(values[c + i - 1]);
                }
            }
        } else if constexpr (ROWS == kJoined) {
            if (i0 == 0 && j0 == 0) { // what lies before the head's first line
                const int ahead = (kLine - into_line(first)) & (kLine - 1);
                for (int e = threadIdx.x; e < ahead; e += THREADS) first[e] = values[e + R - 1];
            }
            // the rows' last lines, side by side
            for (int t = threadIdx.x; t < R * (kLine / V); t += THREADS) {
                const int i = t / (kLine / V);
                Bits *row = first + (long)i * a.ld;
                const int ahead = (kLine - into_line(row)) & (kLine - 1), line = (a.k - 1 - ahead) / kLine * kLine - j0; // from the tile's first one on
                const int col = line + ahead + t % (kLine / V) * V, left = a.k - j0 - col;                               // columns of this row from there on
                if (line < 0 || line >= kColumns) continue;
                if (i0 + i + 1 < a.q) {
                    Bits e[V];
#pragma unroll
                    for (int k = 0; k < V; ++k) e[k] = k < left ? values[col + k + R - 1 - i] : starts[k - left + R - 1 - i];
                    __builtin_memcpy(__builtin_assume_aligned(row + col, 16), e, 16);
                } else {
                    for (int k = 0; k < left && k < V; ++k) row[col + k] = values[col + k + R - 1 - i];
                }
            }
            if (j0 + (c & -64 * V) >= a.k) continue; // (nothing for this wavefront)
#pragma unroll 2
            for (int i = 0; i < R; ++i) {
                Bits *row = first + (long)i * a.ld;
                const int ahead = (kLine - into_line(row)) & (kLine - 1);
                const Vec v = Vec::from(values, c, ahead + R - 1 - i);
                if (j0 + (c & -kLine) + ahead + kLine < a.k) *reinterpret_cast<uint4 *>(row + c + ahead) = v.w;
            }
        } else {
#pragma unroll 2
            for (int i = 0; i < R; ++i) {
                Bits *row = first + (long)i * a.ld;
                const int m = into_line(row), col = c - m;
                const Vec v = Vec::from(values, c, kLine + R - 1 - i - m);
                if (j0 + col >= 0 && j0 + col + V <= a.k) {
                    *reinterpret_cast<uint4 *>(row + col) = v.w;
                } else if (ROWS == kSingle) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (j0 + col + e >= 0 && j0 + col + e < a.k) row[col + e] = (Bits)v.at(e);
                }
            }
            for (int t = threadIdx.x; ROWS == kApart && t < R * 2 * V; t += THREADS) {
                const int i = t / (2 * V), head = t % (2 * V);
                Bits *row = first + (long)i * a.ld;
                const int m = into_line(row), above = kLine + R - 1 - i, o = m & (V - 1), last = ((a.k + o) & ~(V - 1)) - o - j0, tail = last + head - V;
                if (head < V) {
                    if (j0 == 0 && o > 0 && head < V - o && head < a.k) row[head] = values[head + above];
                } else if (j0 + last >= 0 && last + m >= 0 && last + m < kColumns && j0 + tail < a.k) {
                    row[tail] = values[tail + above];
                }
            }
        }
    }
}

// ---- its gradient -------------------------------------------------------------------------------------------------------------------
// Bound by the reads of dout.  A wavefront takes 8 to 32 rows of 64 V columns, a lane V columns of every row, and keeps one sum for each of its
// columns' diagonals (j - i = const: one offset, one bucket).  From one row to the next the sums move up by one place, from a lane's last to the next lane's
// first; what leaves the last lane is the whole sum of a diagonal of this tile and waits in a lane of a register of its own.  So every value costs one
// addition, in the same order every run, wherever its bucket's borders lie; only the sums of a tile's diagonals, some 64 V, are sorted into buckets, and most
// tiles meet one bucket alone.

// V columns of dout from column j on.  The vector that reaches over a row's end is read with what stands behind it, in the last row of all, where there may
// be nothing, V columns before the end; keep() takes away what is not the row's.  That is done when the values are used and not before: the loads stay in flight.
template <typename T, int V> struct Columns {
    uint4 w;
    static __device__ __forceinline__ int place(int j, int k, bool last) { return last ? (j < k - V ? j : k - V) : j < k ? j : k - 1; }
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (V == 1) w.x = sizeof(T) == 2 ? (uint32_t)*reinterpret_cast<const uint16_t *>(p) : *reinterpret_cast<const uint32_t *>(p);
        else __builtin_memcpy(&w, p, 16);
    }
    __device__ __forceinline__ void keep(int j, int k, bool last)
    {
        constexpr int kBits = 8 * sizeof(T);
        if constexpr (V == 1) {
            w.x = j < k ? w.x : 0u;
        } else if (last) { // the columns from j on to the front, zeros behind them
            const int bits = (j - place(j, k, true)) * kBits < 128 ? (j - place(j, k, true)) * kBits : 128;
            const uint64_t lo = (uint64_t)w.y << 32 | w.x, hi = (uint64_t)w.w << 32 | w.z;
            const uint64_t l = bits == 0 ? lo : bits < 64 ? lo >> bits | hi << (64 - bits) : bits < 128 ? hi >> (bits - 64) : 0;
            const uint64_t u = bits < 64 ? hi >> bits : 0;
            w = make_uint4((uint32_t)l, (uint32_t)(l >> 32), (uint32_t)u, (uint32_t)(u >> 32));
        } else {
            const int bits = (k - j) * kBits; // that are the row's
            const auto part = [&](uint32_t v, int from) { return bits >= from + 32 ? v : bits > from ? v & 0xffffffffu >> (from + 32 - bits) : 0u; };
            w = make_uint4(part(w.x, 0), part(w.y, 32), part(w.z, 64), part(w.w, 96));
        }
    }
    __device__ __forceinline__ float at(int i) const
    {
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
        if constexpr (sizeof(T) == 4) return __uint_as_float(word[i]);
        return i & 1 ? __uint_as_float(word[i / 2] & 0xffff0000u) : __uint_as_float(word[i / 2] << 16);
    }
};

template <int CTRL> __device__ __forceinline__ float dpp_move(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v += dpp_move<0xB1>(v);
    v += dpp_move<0x4E>(v);
    v += dpp_move<0x141>(v);
    v += dpp_move<0x140>(v);
    return qgroup_sum(v);
}

template <typename T, int V> __global__ __launch_bounds__(kThreads) void sequence_bwd_kernel(Args a)
{
    constexpr int kWaves = kThreads / 64, kColumns = 64 * V, kAtOnce = 4; // rows whose loads are in flight together
    constexpr int kLong = 48; // a run of more diagonals than this is summed by all lanes, a shorter one by one
    __shared__ float sums[kWaves][2 * (RELPOS_MAX_EDGES + 1)];
    __shared__ float diagonal[kWaves][kColumns + 64];
    __shared__ int edges[RELPOS_MAX_EDGES];
    const int h = blockIdx.y, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (int b = lane; b < a.buckets; b += 64) sums[wave][b] = 0.f;
    for (int e = threadIdx.x; e < a.n; e += kThreads) edges[e] = a.edges[e];
    __syncthreads();
    const int R = a.grad_rows, tiles_q = (a.q + R - 1) / R, tiles_k = (a.k + kColumns - 1) / kColumns;
    const long tiles = (long)a.batch * tiles_q * tiles_k;
    for (long tile = (long)blockIdx.x * kWaves + wave; tile < tiles; tile += (long)gridDim.x * kWaves) {
        const long t = tile / tiles_k;
        const int i0 = (int)(t % tiles_q) * R, b = (int)(t / tiles_q), j0 = (int)(tile % tiles_k) * kColumns;
        if (a.causal && j0 > i0 + R - 1 + a.start) continue; // (nothing seen)
        const T *rows = static_cast<const T *>(a.dout) + (((long)b * a.heads + h) * a.q + i0) * a.ld;
        const int i1 = a.q - i0 < R ? a.q - i0 : R, j = j0 + lane * V;
        const bool edge = j0 + kColumns > a.k;
        const int inside = Columns<T, V>::place(j, a.k, false), before = Columns<T, V>::place(j, a.k, true);
        const int last = b == a.batch - 1 && h == a.heads - 1 ? a.q - 1 - i0 : -1; // the last row of all, among these
        float acc[V] = {}, gone = 0.f;
        Columns<T, V> now[kAtOnce], next[kAtOnce];
        const auto fetch = [&](int i, Columns<T, V> (&c)[kAtOnce]) {
#pragma unroll
            for (int r = 0; r < kAtOnce; ++r) {
                c[r].w = make_uint4(0, 0, 0, 0);
                // (a lane all of whose columns are hidden from these rows does without them)
                if (i + r < i1 && !(a.causal && j > i0 + i + kAtOnce - 1 + a.start)) c[r].load(rows + (long)(i + r) * a.ld + (i + r == last ? before : inside));
            }
        };
        fetch(0, now);
        for (int i = 0; i < R; i += kAtOnce) {
            if (i + kAtOnce < i1) fetch(i + kAtOnce, next);
            else {
#pragma unroll
                for (int r = 0; r < kAtOnce; ++r) next[r].w = make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < kAtOnce; ++r) {
                if (i + r > 0) {
                    const float out = acc[V - 1];
                    // (wave_shl 1: what waits moves to the lane before, the last lane takes its own last sum)
                    gone = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, out), __builtin_bit_cast(int, gone), 0x130, 0xF, 0xF,
                                                                                 false));
#pragma unroll
                    for (int e = V - 1; e > 0; --e) acc[e] = acc[e - 1];
                    acc[0] = dpp_move<0x138>(out); // (wave_shr 1: from the lane before; 0 into the first)
                }
                if (edge) now[r].keep(j, a.k, i + r == last);
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += now[r].at(e);
            }
#pragma unroll
            for (int r = 0; r < kAtOnce; ++r) now[r] = next[r];
        }
        // The sums in the order of their diagonals, from offset `low` on: acc[e] of a lane is (lane, e), and what has left stands in the last
        // R - 1 lanes, the farthest offset first.
        const int low = j0 - (i0 + R - 1) - a.start, high = j0 + kColumns - 1 - i0 - a.start, most = a.causal && high > 0 ? 0 : high;
        float *diag = diagonal[wave];
#pragma unroll
        for (int e = 0; e < V; ++e) diag[lane * V + e] = acc[e];
        if (lane > 64 - R) diag[kColumns + 63 - lane] = gone;
        __builtin_amdgcn_wave_barrier();
        // A lane finds the offsets of its bucket among them, and sums them if they are few.
        for (int b0 = 0; b0 < a.buckets; b0 += 64) {
            const int bucket = b0 + lane, behind = bucket > a.n, n = behind ? bucket - a.n - 1 : bucket;
            int from = 1, to = 0;
            if (bucket < a.buckets) {
                const int near = n ? edges[n - 1] : behind, far = n < a.n ? edges[n] - 1 : 0x7fffffff; // distances
                from = behind ? near : -far;
                to = behind ? far : !n && !a.bidirectional ? 0x7fffffff : -near;
                from = (from > low ? from : low) - low;
                to = (to < most ? to : most) - low;
            }
            const int length = to - from + 1;
            if (length > 0 && length <= kLong) {
                float s = 0.f;
#pragma unroll 4
                for (int x = from; x <= to; ++x) s += diag[x];
                sums[wave][bucket] += s;
            }
            for (uint64_t left = __ballot(length > kLong); left; left &= left - 1) {
                const int owner = __builtin_ctzll(left), first = __builtin_amdgcn_readlane(from, owner), last = __builtin_amdgcn_readlane(to, owner);
                float s = 0.f;
#pragma unroll
                for (int x = 0; x < kColumns + kMostRows - 1; x += 64) {
                    const int y = x + lane;
                    s += y >= first && y <= last ? diag[y] : 0.f;
                }
                s = wave_sum(s);
                if (lane == owner) sums[wave][bucket] += s;
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    for (int b = threadIdx.x; b < a.buckets; b += kThreads) {
        const float s = (sums[0][b] + sums[1][b]) + (sums[2][b] + sums[3][b]);
        float *out = a.dtable + (long)b * a.heads + h;
        if (a.part) a.part[((long)h * a.slices + blockIdx.x) * a.buckets + b] = s;
        else *out = a.accumulate ? *out + s : s;
    }
}

// The workgroups' sums of a head: a thread per bucket and group of them, the groups in their order.
__global__ __launch_bounds__(1024) void sequence_sum_kernel(Args a)
{
    __shared__ double lds[1024];
    const int h = blockIdx.x, groups = 1024 / a.buckets, g = threadIdx.x / a.buckets, b = threadIdx.x - g * a.buckets;
    double s = 0.;
    if (g < groups) {
#pragma unroll 8
        for (int i = g; i < a.slices; i += groups) s += a.part[((long)h * a.slices + i) * a.buckets + b];
    }
    lds[threadIdx.x] = s;
    __syncthreads();
    if (g) return;
#pragma unroll 8
    for (int i = 1; i < groups; ++i) s += lds[i * a.buckets + b];
    float *out = a.dtable + (long)b * a.heads + h;
    *out = (float)(a.accumulate ? *out + s : s);
}

struct Plan {
    size_t elem, out, dout, table, dtable, ws;
    long ld;
    int buckets, V;            // V: columns of a lane
    bool narrow;               // workgroups of one wavefront for the bias
    int rows, grad_rows;       // of a tile of the bias and of the gradient
    int spread;                // logarithm of the XCDs over which the bands of rows of the bias are spread
    int slices;
};

long ceil_div(long a, long b) { return (a + b - 1) / b; }

int make_plan(const relpos_desc *d, Plan *p)
{
    if (!d) return GSWA_EINVAL;
    *p = Plan{}; // (the window form has no tiles)
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
        const int wide = (int)(16 / p->elem);
        p->V = d->k_len < wide ? 1 : wide;
        // The bias: as many rows a tile (64 at most, 8 at least) as leave 8 workgroups a compute unit, since a tile's values are found anew for each; where even
        // 8 rows leave few, workgroups of one wavefront and a quarter of the columns.
        const long across = ceil_div(d->k_len, (long)kThreads * wide) * d->heads;
        p->narrow = across * ceil_div(d->q_len, 8) < 2 * kSizingCus || d->k_len <= 64 * wide;
        p->rows = kMostFwdRows;
        while (p->rows > 8 && across * ceil_div(d->q_len, p->rows) < 8 * kSizingCus) p->rows /= 2;
        p->spread = ceil_div(d->q_len, p->rows) < 16 ? 0 : 3; // 8 XCDs (few bands: workgroups of none would outweigh it)
        // Its gradient: tiles of 32 rows, fewer where that leaves less than four a compute unit; 16 workgroups a compute unit, over the
        // heads, more than run at once (tiles near the diagonal take longer, hidden ones no time).
        const long images = (long)d->batch * ceil_div(d->k_len, 64L * p->V);
        p->grad_rows = kMostRows;
        while (p->grad_rows > 8 && images * d->heads * ceil_div(d->q_len, p->grad_rows) < 4 * kSizingCus) p->grad_rows /= 2;
        const long tiles = ceil_div(images * ceil_div(d->q_len, p->grad_rows), kThreads / 64);
        const long most = ceil_div(16 * kSizingCus, d->heads);
        p->slices = (int)(most < tiles ? most : tiles);
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
    a->window = d->window; a->buckets = p.buckets; a->ld = p.ld; a->slices = p.slices; a->rows = p.rows; a->grad_rows = p.grad_rows;
    a->spread = p.spread;
    a->bidirectional = (d->flags & RELPOS_BIDIRECTIONAL) != 0;
    a->causal = (d->flags & RELPOS_CAUSAL) != 0;
    a->accumulate = (d->flags & RELPOS_ACCUM_WGRAD) != 0;
    a->n = d->n_edges;
    for (int i = 0; i < d->n_edges; ++i) a->edges[i] = d->edges[i];
}

template <typename T, int ROWS> void launch_forward(const Args &a, const Plan &p, hipStream_t st)
{
    const int threads = p.narrow ? 64 : kThreads, line = 128 / (int)sizeof(T);
    const long tiles = (ceil_div(ceil_div(a.q, a.rows), 1 << a.spread) << a.spread) * ceil_div((long)a.k + (ROWS == kApart || ROWS == kSingle ? line - 1 : 0), threads * (16L / sizeof(T)));
    const dim3 grid((unsigned)(tiles < (1L << 20) ? tiles : 1L << 20), a.heads);
    if (p.narrow) hipLaunchKernelGGL((sequence_fwd_kernel<T, 64, ROWS>), grid, dim3(64), 0, st, a);
    else hipLaunchKernelGGL((sequence_fwd_kernel<T, kThreads, ROWS>), grid, dim3(kThreads), 0, st, a);
}

template <typename T> void launch_forward(const Args &a, const Plan &p, hipStream_t st)
{
    const int line = 128 / (int)sizeof(T);
    if (p.ld % line == 0 && reinterpret_cast<uintptr_t>(a.out) % 128 == 0) launch_forward<T, kAligned>(a, p, st);
    else if (p.ld == a.k && a.k >= line && a.q >= 8) launch_forward<T, kJoined>(a, p, st); // (a line that starts in a row ends in it or the next; a head's last row is not joined)
    else if (a.q == 1) launch_forward<T, kSingle>(a, p, st);
    else launch_forward<T, kApart>(a, p, st);
}

template <typename T> void launch_backward(const Args &a, const Plan &p, dim3 grid, hipStream_t st)
{
    if (p.V == 1) hipLaunchKernelGGL((sequence_bwd_kernel<T, 1>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((sequence_bwd_kernel<T, 16 / sizeof(T)>), grid, dim3(kThreads), 0, st, a);
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
        if (desc->dtype == GSWA_F32) launch_forward<float>(a, p, st);
        else launch_forward<bf16_t>(a, p, st);
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
    a.dout = dout; a.dtable = dtable; a.part = p.slices > 1 ? static_cast<float *>(ws) : nullptr;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (desc->window > 0) {
        KernelTimer t(K_RELPOS_BWD, st);
        hipLaunchKernelGGL(window_bwd_kernel, dim3(p.buckets), dim3(kThreads), 0, st, a);
        RP_LAUNCHED();
        return GSWA_OK;
    }
    {
        KernelTimer t(K_RELPOS_BWD, st);
        const dim3 grid(p.slices, desc->heads);
        if (desc->dtype == GSWA_F32) launch_backward<float>(a, p, grid, st);
        else launch_backward<bf16_t>(a, p, grid, st);
        RP_LAUNCHED();
    }
    if (!a.part) return GSWA_OK; // (16 x 16 positions: 4.8 us, 7.1 with a second launch)
    KernelTimer t(K_RELPOS_SUM, st);
    hipLaunchKernelGGL(sequence_sum_kernel, dim3(desc->heads), dim3(1024), 0, st, a);
    RP_LAUNCHED();
    return GSWA_OK;
}

} // extern "C"
