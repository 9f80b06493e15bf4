// Layer norm, forward and backward, with the reduction of the weight's and the bias's gradient.
//
//   mean = sum x / D,  rstd = (sum (x - mean)^2 / D + eps)^(-1/2),  xhat = (x - mean) rstd,  y = xhat w + b
//   dx = rstd (g w - mean(g w) - xhat mean(g w xhat)),  dw = sum_n g xhat,  db = sum_n g
//
// Bound: memory for binary32 rows (8192 x 8192: forward 98 us, 5.5 TB/s, gradient 141 us, 5.7 TB/s); the issue rate for
// 16-bit rows forward (16384 x 4096 bfloat16: 53 us, 5.1 TB/s at 68 % of the issue slots, 19 instructions per value); the
// latency between a row's passes for their gradient (16384 x 8192: 160 us, 5.0 TB/s; 55 % of the issue slots at 16384 x
// 4096); the launch for a few rows (1 x 4096: 2.3 us).  So a row is read once, in 16-byte packs, and its arithmetic runs on
// pairs of binary32 values.  The mean, then the centred squares (two reductions, no cancellation), then the output.  All
// statistics and sums are binary32.
//
// Rows that do not start on 16-byte boundaries (an odd width, say) keep the packs: what a thread owns is a 16-byte
// granule of memory, and with it columns shifted by the row's phase, the number of elements between the granule's start
// and the row's.  Phases repeat with a short period (at most 8 rows), so a CTA or warp takes rows of one phase only:
// its threads then own the same columns in every row, as the sums of dw and db over the rows need it.  The first and
// the last granule of a row are masked; where they would reach beyond the operand they are read element by element.
// (8192 x 4097 bfloat16: forward 48 us and gradient 92 us, against 81 and 269 a value at a time.)
#include <atomic>
#include <climits>
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "device_utils.cuh"
#include "operators_internal.cuh"

namespace rsdgc {

constexpr int kNormWarps = 4;              // warps of a CTA whose rows take one warp each, forward
constexpr int kBackWarps = 8;              // ... backward
constexpr int kNormElems = 16;             // columns of a thread (32 in the widest variants)
constexpr int kNormRingThreads = 512;
constexpr int kNormJoin = kNormRingThreads + 4;
constexpr int kNormLongThreads = 1024;
constexpr int kNormMaxStages = 4;
constexpr int kNormMaxTeams = 8;
constexpr int kNormMaxParts = 8;            // CTAs of a row, the portable size of a cluster
constexpr int kNormRingBytes = 200 << 10;  // shared memory of a multiprocessor's rings

// A 16-byte pack as pairs of binary32 values (f32x2 arithmetic: two values per instruction).
template <typename T>
struct Pairs {
    static constexpr int N = 8 / (int)sizeof(T);   // pairs
    static constexpr int V = 16 / (int)sizeof(T);  // elements
    uint32_t w[4];
    __device__ __forceinline__ void load(const T *p)
    {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    }
    __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0u; }
    __device__ __forceinline__ float2 get(int i) const;
    __device__ __forceinline__ void set(int i, float2 v);
    // element j out of / into the pack
    __device__ __forceinline__ T element(int j) const;
    __device__ __forceinline__ void put(int j, T x);
    // keeps the elements of columns 0 .. d - 1, the pack starting at column c
    __device__ __forceinline__ void mask(int c, int d)
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = (unsigned)(c + j) < (unsigned)d ? w[j] : 0u;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[j] &= ((unsigned)(c + 2 * j) < (unsigned)d ? 0x0000FFFFu : 0u) |
                        ((unsigned)(c + 2 * j + 1) < (unsigned)d ? 0xFFFF0000u : 0u);
        }
    }
    // row: column 0 of a row whose granule `c` is wanted; only existing columns are touched
    __device__ __forceinline__ void load_elements(const T *row, int c, int d)
    {
        clear();
#pragma unroll
        for (int j = 0; j < V; ++j)
            if ((unsigned)(c + j) < (unsigned)d) put(j, row[c + j]);
    }
    // whole: all of it exists and lies on a 16-byte boundary
    __device__ __forceinline__ void store(T *row, bool whole, int c, int d) const
    {
        if (whole) {
            if (RSDGC_IN_BOUNDS(c >= 0 && c + V <= d && (reinterpret_cast<uintptr_t>(row + c) & 15) == 0))
                *reinterpret_cast<uint4 *>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if ((unsigned)(c + j) < (unsigned)d) row[c + j] = element(j);
        }
    }
};
template <>
__device__ __forceinline__ float2 Pairs<float>::get(int i) const
{
    return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
}
template <>
__device__ __forceinline__ void Pairs<float>::set(int i, float2 v)
{
    w[2 * i] = __float_as_uint(v.x);
    w[2 * i + 1] = __float_as_uint(v.y);
}
template <>
__device__ __forceinline__ float2 Pairs<__nv_bfloat16>::get(int i) const
{
    return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
template <>
__device__ __forceinline__ void Pairs<__nv_bfloat16>::set(int i, float2 v)
{
    w[i] = pack2<__nv_bfloat16>(v.x, v.y);
}
template <>
__device__ __forceinline__ float2 Pairs<__half>::get(int i) const
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
}
template <>
__device__ __forceinline__ void Pairs<__half>::set(int i, float2 v)
{
    w[i] = pack2<__half>(v.x, v.y);
}
template <>
__device__ __forceinline__ float Pairs<float>::element(int j) const { return __uint_as_float(w[j]); }
template <>
__device__ __forceinline__ void Pairs<float>::put(int j, float x) { w[j] = __float_as_uint(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 Pairs<__nv_bfloat16>::element(int j) const
{
    return __ushort_as_bfloat16((unsigned short)(w[j >> 1] >> (16 * (j & 1))));
}
template <>
__device__ __forceinline__ void Pairs<__nv_bfloat16>::put(int j, __nv_bfloat16 x)
{
    w[j >> 1] |= (uint32_t)__bfloat16_as_ushort(x) << (16 * (j & 1));
}
template <>
__device__ __forceinline__ __half Pairs<__half>::element(int j) const
{
    return __ushort_as_half((unsigned short)(w[j >> 1] >> (16 * (j & 1))));
}
template <>
__device__ __forceinline__ void Pairs<__half>::put(int j, __half x)
{
    w[j >> 1] |= (uint32_t)__half_as_ushort(x) << (16 * (j & 1));
}

// The parameters of the 2 * PAIRS columns from c on (those that exist), or a constant where there is no vector.
template <bool SHIFT, typename P, int PAIRS>
__device__ __forceinline__ void load_params(const P *p, int c, int d, float missing, float2 *out)
{
    if constexpr (SHIFT) {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            const int a = c + 2 * i;
            out[i].x = p && (unsigned)a < (unsigned)d ? to_f32(p[a]) : missing;
            out[i].y = p && (unsigned)(a + 1) < (unsigned)d ? to_f32(p[a + 1]) : missing;
        }
    } else if (p && c < d) {
#pragma unroll
        for (int k = 0; k < PAIRS / Pairs<P>::N; ++k) {
            Pairs<P> v;
            v.load(p + c + k * Pairs<P>::V);
#pragma unroll
            for (int i = 0; i < Pairs<P>::N; ++i) out[k * Pairs<P>::N + i] = v.get(i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) out[i] = make_float2(missing, missing);
    }
}

// Which rows a walker (CTA or warp) takes: those of one phase.
struct PhaseRows {
    int period, phase0, step;   // rows r and r + period have the same phase, (phase0 + r * step) mod V elements
    bool same_out;              // the output's rows too
};
struct Walk {
    int row0, period, phase;    // its rows: row0 + period * j
    int count;                  // rows of this phase
    int first, stride;          // it takes j = first, first + stride, ...
};
template <int V>
__device__ __forceinline__ Walk walk_of(const PhaseRows &p, int walker, int walkers, int n)
{
    Walk w;
    w.period = p.period;
    w.row0 = walker % p.period;
    w.phase = (p.phase0 + w.row0 * p.step) & (V - 1);
    w.count = n > w.row0 ? (n - w.row0 + p.period - 1) / p.period : 0;
    w.first = walker / p.period;
    w.stride = walkers / p.period;  // a multiple of the period is launched
    return w;
}

// The granules of a thread: columns start + i * pitch on.  SHIFT: rows are shifted, or the width is no whole number of
// granules, or an output's rows lie elsewhere; without it every granule that exists is whole.  `fast`: all granules of the
// whole warp exist and are whole, so that its code (FAST) needs no tests; only a row's first and last warps differ.
template <bool SHIFT, int V, int NV>
struct Columns {
    int start, pitch, d;
    unsigned whole_bits, store_bits;
    bool fast;
    __device__ __forceinline__ Columns(int thread, int threads, int phase, int width, bool same_out)
        : start(thread * V - phase), pitch(threads * V), d(width), whole_bits(0)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) whole_bits |= (unsigned)(at(i) >= 0 && at(i) + V <= d) << i;
        store_bits = !SHIFT || same_out ? whole_bits : 0u;
        fast = __all_sync(0xFFFFFFFFu, store_bits == (1u << NV) - 1u);
    }
    __device__ __forceinline__ int at(int i) const { return start + i * pitch; }
    template <bool FAST>
    __device__ __forceinline__ bool any(int i) const { return FAST || at(i) < d; }
    template <bool FAST>
    __device__ __forceinline__ bool whole(int i) const { return FAST || !SHIFT || (whole_bits >> i & 1); }
    template <bool FAST>
    __device__ __forceinline__ bool stored_whole(int i) const { return FAST || !SHIFT || (store_bits >> i & 1); }
};

// Sum over the threads of one row: a warp, or the CTA with one slot of `part` per warp (the caller alternates between
// two buffers, so that one barrier per sum is enough).
template <bool WARP>
__device__ __forceinline__ float row_sum(float x, float *part)
{
    x = warp_sum(x);
    if (WARP) return x;
    const int warps = (int)(blockDim.x >> 5), lane = threadIdx.x & 31;
    if (lane == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    return warp_sum(lane < warps ? part[lane] : 0.0f);
}

// A ring of stages in shared memory, each one or several rows, filled by bulk copies that run ahead of the threads, so
// that a CTA has tens of KB on their way whatever its threads wait for.
struct RowRing {
    uint32_t base, full;   // shared-memory addresses: rows, barriers (8 bytes each)
    uint32_t stage_bytes;
    int stages;
    bool arrived;          // false once a wait has given up: the results are void, as the status says
    int step;              // a wait gives up after kOperatorPolls / step polls
    unsigned int *status;

    __device__ __forceinline__ uint32_t bar(int i) const { return full + 8 * (i % stages); }
    __device__ __forceinline__ uint32_t offset(int i) const { return (i % stages) * stage_bytes; }
    __device__ __forceinline__ uint32_t at(int i) const { return base + offset(i); }
    // Bounded; after one that gave up the others poll once.  `lost` (shared): the stage whose wait gave up, set by the thread
    // that fills the ring; it fills nothing more then, for a stage may be refilled only once its copies have arrived.
    // TRY_FIRST: the loop's form decides how the rows' loop around it gets along with its registers.  Gradient of 16384 x 8192
    // bfloat16 (weight in registers) 161 us with it, 174 without; of 8192 x 4097 (weight in shared memory) 96 and 91.
    template <bool TRY_FIRST>
    __device__ __forceinline__ void wait(int i, bool fills, int &lost)
    {
        int left = arrived ? (int)kOperatorPolls : 1;
        bool here = false;
        if constexpr (TRY_FIRST) {
            do here = barrier_try(bar(i), (uint32_t)(i / stages) & 1u);
            while (!here && (left -= step) > 0);
        } else {
            while (left > 0 && !(here = barrier_try(bar(i), (uint32_t)(i / stages) & 1u))) left -= step;
        }
        if (!here && arrived) {
            arrived = false;
            if (fills) lost = i;
            atomicOr(status, RSDGC_STATUS_TIMEOUT);
        }
    }
    // After a failure, by the thread that filled the ring: the copies under way, of its last stages before `end`, land in this
    // CTA's memory.
    __device__ __forceinline__ void drain(int end) const
    {
        for (int i = max(0, end - stages); i < end; ++i)
            for (unsigned q = 0; q < kOperatorPolls && !barrier_try(bar(i), (uint32_t)(i / stages) & 1u); ++q) {}
    }
};

// The granules of a row that lie inside the operand, as a bulk copy: all of them but the first of the operand's first
// row and the last of its last, where these reach beyond it.
struct RowCopy {
    uint32_t skip, bytes;  // bytes left out at the front, bytes copied
};
template <typename T>
__device__ __forceinline__ RowCopy row_copy(int row, int n, int phase, int d)
{
    constexpr int V = Pairs<T>::V;
    int g0 = 0, g1 = (phase + d + V - 1) / V;
    if (row == 0 && phase) g0 = 1;
    if (row == n - 1 && (phase + d) % V) --g1;
    return {(uint32_t)g0 * 16u, g1 > g0 ? (uint32_t)(g1 - g0) * 16u : 0u};
}
// Granule i of `row` (column 0) from its copy in shared memory; masked at the row's ends.
template <bool FAST, bool SHIFT, typename T, int NV>
__device__ __forceinline__ void take(Pairs<T> &v, const Columns<SHIFT, Pairs<T>::V, NV> &cols, int i,
                                     const unsigned char *copy, int phase, const T *row, bool edge)
{
    const int c = cols.at(i);
    if (edge && !cols.template whole<FAST>(i)) {
        v.load_elements(row, c, cols.d);
        return;
    }
    v.load(reinterpret_cast<const T *>(copy + (c + phase) * (int)sizeof(T)));
    if (!cols.template whole<FAST>(i)) v.mask(c, cols.d);
}
// Whether an operand of n rows of d values has the values [first, first + count), counted from its first one; what lies between
// its rows counts as its own.
__device__ __forceinline__ bool exist(long long first, int count, long long stride, int n, int d)
{
    return first >= 0 && first + count <= (n - 1) * stride + d;
}
// ... and a bulk copy of a row's granules, inside a row of `room` bytes of the ring
template <typename T>
__device__ __forceinline__ bool copy_exists(const T *x, long long stride, int row, int phase, RowCopy copy, uint32_t room, int n, int d)
{
    const long long first = row * stride - phase + copy.skip / (int)sizeof(T);
    return row >= 0 && row < n && exist(first, copy.bytes / (int)sizeof(T), stride, n, d) && copy.skip + copy.bytes <= room &&
           (reinterpret_cast<uintptr_t>(x + first) & 15) == 0;
}
// Rows whose granules may reach beyond the operand's first or last value (one row at either end unless rows are
// shorter than a granule).
template <int V>
__device__ __forceinline__ bool near_end(long long row, int n, int d)
{
    return row * d < V || (n - 1 - row) * d < V;
}
// ... straight from global memory
template <bool FAST, bool SHIFT, typename T, int NV>
__device__ __forceinline__ void take(Pairs<T> &v, const Columns<SHIFT, Pairs<T>::V, NV> &cols, int i, const T *row, bool edge)
{
    const int c = cols.at(i);
    if (edge && !cols.template whole<FAST>(i)) {
        v.load_elements(row, c, cols.d);
        return;
    }
    v.load(row + c);
    if (!cols.template whole<FAST>(i)) v.mask(c, cols.d);
}

// ---- forward ----------------------------------------------------------------------------------
// A thread's share of the passes over a row in registers: the sum, the centred squares (scaled term by term: their sum
// may leave the range where their mean does not), the output.
template <bool FAST, bool SHIFT, typename T, int NV>
__device__ __forceinline__ float sum_of(const Pairs<T> (&in)[NV], const Columns<SHIFT, Pairs<T>::V, NV> &cols)
{
    float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (cols.template any<FAST>(i)) {
#pragma unroll
            for (int k = 0; k < Pairs<T>::N; ++k) sum = add2(sum, in[i].get(k));  // masked columns are zero
        }
    return sum.x + sum.y;
}
template <bool FAST, bool SHIFT, typename T, int NV>
__device__ __forceinline__ float squares_of(const Pairs<T> (&in)[NV], const Columns<SHIFT, Pairs<T>::V, NV> &cols, float mu,
                                            float root_inv_d)
{
    const float2 rr = make_float2(root_inv_d, root_inv_d), m2 = make_float2(-mu, -mu);
    float2 sq = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (cols.template any<FAST>(i)) {
            const int c = cols.at(i);
            const bool whole = cols.template whole<FAST>(i);
#pragma unroll
            for (int k = 0; k < Pairs<T>::N; ++k) {
                float2 e = mul2(add2(in[i].get(k), m2), rr);
                if (!whole) {
                    e.x = (unsigned)(c + 2 * k) < (unsigned)cols.d ? e.x : 0.0f;
                    e.y = (unsigned)(c + 2 * k + 1) < (unsigned)cols.d ? e.y : 0.0f;
                }
                sq = fma2(e, e, sq);
            }
        }
    return sq.x + sq.y;
}
template <bool FAST, bool SHIFT, typename T, int NV>
__device__ __forceinline__ void write_row(const Pairs<T> (&in)[NV], T *row, const Columns<SHIFT, Pairs<T>::V, NV> &cols, float mu,
                                          float r, const float2 (*wv)[Pairs<T>::N], const float2 (*bv)[Pairs<T>::N])
{
    const float2 m2 = make_float2(-mu, -mu), r2 = make_float2(r, r);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (cols.template any<FAST>(i)) {
            Pairs<T> out;
#pragma unroll
            for (int k = 0; k < Pairs<T>::N; ++k) out.set(k, fma2(mul2(add2(in[i].get(k), m2), r2), wv[i][k], bv[i][k]));
            out.store(row, cols.template stored_whole<FAST>(i), cols.at(i), cols.d);
        }
    }
}
// Both forms of a warp's code: f(std::true_type) where all its granules are whole.
template <typename F>
__device__ __forceinline__ void by_warp(bool fast, F f)
{
    if (fast) f(std::true_type{}); else f(std::false_type{});
}

// A CTA per row, rows through the ring; the threads keep their columns' weight and bias as binary32 pairs.  Two barriers
// per row (mean, squares); the next rows arrive meanwhile.
template <bool SHIFT, typename T, typename P, int E>
__global__ void __launch_bounds__(kNormRingThreads, E <= 16 ? 2 : 1)
k_norm_forward_ring(const T *__restrict__ x, long long xs, const P *__restrict__ w, const P *__restrict__ b,
                    T *__restrict__ y, long long ys, float *__restrict__ mean, float *__restrict__ rstd, int n, int d,
                    PhaseRows phases, float inv_d, float root_inv_d, float eps, int stages, uint32_t stage_bytes, int step,
                    unsigned int *status)
{
    constexpr int V = Pairs<T>::V, NV = E / V, NP = Pairs<T>::N;
    extern __shared__ __align__(128) unsigned char rows[];
    __shared__ float part[2][32];
    __shared__ __align__(8) unsigned long long full[kNormMaxStages];
    __shared__ int lost;
    const Walk walk = walk_of<V>(phases, blockIdx.x, gridDim.x, n);
    RowRing ring = {smem_addr(rows), smem_addr(full), stage_bytes, stages, true, step, status};
    if (threadIdx.x < stages) barrier_init(ring.bar(threadIdx.x), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    grid_dependency_wait();
    grid_dependency_launch_next();
    auto load = [&](int i) {
        const int j = walk.first + i * walk.stride;
        if (j >= walk.count) return;
        const int row = walk.row0 + walk.period * j;
        const RowCopy copy = row_copy<T>(row, n, walk.phase, d);
        barrier_expect(ring.bar(i), copy.bytes);
        if (copy.bytes && RSDGC_IN_BOUNDS(copy_exists(x, xs, row, walk.phase, copy, stage_bytes, n, d)))
            bulk_copy(ring.at(i) + copy.skip, reinterpret_cast<const unsigned char *>(x + row * xs - walk.phase) + copy.skip,
                      copy.bytes, ring.bar(i));
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < stages; ++i) load(i);
    const Columns<SHIFT, V, NV> cols(threadIdx.x, blockDim.x, SHIFT ? walk.phase : 0, d, phases.same_out);
    float2 wv[NV][NP], bv[NV][NP];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load_params<SHIFT, P, NP>(w, cols.at(i), d, 1.0f, wv[i]);
        load_params<SHIFT, P, NP>(b, cols.at(i), d, 0.0f, bv[i]);
    }
    int it = 0;
    for (int j = walk.first; j < walk.count; j += walk.stride, ++it) {
        const int row = walk.row0 + walk.period * j;
        const bool edge = row == 0 || row == n - 1;
        ring.wait<true>(it, threadIdx.x == 0, lost);
        Pairs<T> in[NV];
        float sum = 0.0f, sq = 0.0f;
        by_warp(cols.fast, [&](auto fast) {
            constexpr bool FAST = decltype(fast)::value;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (cols.template any<FAST>(i) &&
                    RSDGC_IN_BOUNDS(cols.at(i) + walk.phase >= 0 && (cols.at(i) + walk.phase + V) * (int)sizeof(T) <= (int)stage_bytes))
                    take<FAST>(in[i], cols, i, rows + ring.offset(it), SHIFT ? walk.phase : 0, x + row * xs, edge);
            sum = sum_of<FAST>(in, cols);
        });
        const float mu = row_sum<false>(sum, part[0]) * inv_d;
        by_warp(cols.fast, [&](auto fast) { sq = squares_of<decltype(fast)::value>(in, cols, mu, root_inv_d); });
        const float r = rsqrtf(row_sum<false>(sq, part[1]) + eps);
        if (threadIdx.x == 0) {
            if (ring.arrived) load(it + stages);  // behind the statistics' barriers: every thread has read the stage
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
        by_warp(cols.fast, [&](auto fast) { write_row<decltype(fast)::value>(in, y + row * ys, cols, mu, r, wv, bv); });
    }
    if (!ring.arrived && threadIdx.x == 0)
        ring.drain(min((walk.count - walk.first + walk.stride - 1) / walk.stride, lost + stages));
}

// A warp per row, kNormWarps walkers per CTA; the next row is loaded while this one is reduced.  (16384 x 512 bfloat16:
// 8.0 us, 4.2 TB/s, out of L2 in part.)
template <bool SHIFT, typename T, typename P>
__global__ void __launch_bounds__(32 * kNormWarps)
k_norm_forward_warp(const T *__restrict__ x, long long xs, const P *__restrict__ w, const P *__restrict__ b,
                    T *__restrict__ y, long long ys, float *__restrict__ mean, float *__restrict__ rstd, int n, int d,
                    PhaseRows phases, float inv_d, float root_inv_d, float eps)
{
    constexpr int V = Pairs<T>::V, NV = kNormElems / V, NP = Pairs<T>::N;
    const int lane = threadIdx.x & 31;
    const Walk walk = walk_of<V>(phases, blockIdx.x * kNormWarps + (threadIdx.x >> 5), gridDim.x * kNormWarps, n);
    const Columns<SHIFT, V, NV> cols(lane, 32, SHIFT ? walk.phase : 0, d, phases.same_out);
    grid_dependency_wait();
    grid_dependency_launch_next();
    Pairs<T> next[NV];
    auto fetch = [&](int j) {
        const int row = walk.row0 + walk.period * j;
        if (j >= walk.count) return;
        by_warp(cols.fast, [&](auto fast) {
            constexpr bool FAST = decltype(fast)::value;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (cols.template any<FAST>(i) &&
                    RSDGC_IN_BOUNDS(row < n && ((near_end<V>(row, n, d) && !cols.template whole<FAST>(i)) ||
                                                exist(row * xs + cols.at(i), V, xs, n, d))))
                    take<FAST>(next[i], cols, i, x + row * xs, near_end<V>(row, n, d));
        });
    };
    fetch(walk.first);
    float2 wv[NV][NP], bv[NV][NP];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load_params<SHIFT, P, NP>(w, cols.at(i), d, 1.0f, wv[i]);
        load_params<SHIFT, P, NP>(b, cols.at(i), d, 0.0f, bv[i]);
    }
    for (int j = walk.first; j < walk.count; j += walk.stride) {
        const int row = walk.row0 + walk.period * j;
        Pairs<T> in[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) in[i] = next[i];
        fetch(j + walk.stride);
        float sum = 0.0f, sq = 0.0f;
        by_warp(cols.fast, [&](auto fast) { sum = sum_of<decltype(fast)::value>(in, cols); });
        const float mu = warp_sum(sum) * inv_d;
        by_warp(cols.fast, [&](auto fast) { sq = squares_of<decltype(fast)::value>(in, cols, mu, root_inv_d); });
        const float r = rsqrtf(warp_sum(sq) + eps);
        if (lane == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
        by_warp(cols.fast, [&](auto fast) { write_row<decltype(fast)::value>(in, y + row * ys, cols, mu, r, wv, bv); });
    }
}

// Any layout and width, a value at a time: rows longer than the ring holds, and operands whose rows have different
// phases.  The row is read three times, the last two out of L2.  (8192 x 4097 bfloat16: 81 us against the ring's 48.)
template <typename T, typename P>
__global__ void __launch_bounds__(kNormLongThreads)
k_norm_forward_any(const T *__restrict__ x, long long xs, const P *__restrict__ w, const P *__restrict__ b,
                   T *__restrict__ y, long long ys, float *__restrict__ mean, float *__restrict__ rstd,
                   int d, float inv_d, float root_inv_d, float eps)
{
    __shared__ float part[2][32];
    grid_dependency_wait();
    grid_dependency_launch_next();
    const long long row = blockIdx.x;
    const T *xr = x + row * xs;
    float sum = 0.0f, sq = 0.0f;
    for (int c = threadIdx.x; c < d; c += blockDim.x) sum += to_f32(xr[c]);
    const float mu = row_sum<false>(sum, part[0]) * inv_d;
    for (int c = threadIdx.x; c < d; c += blockDim.x) {
        const float e = (to_f32(xr[c]) - mu) * root_inv_d;
        sq = fmaf(e, e, sq);
    }
    const float r = rsqrtf(row_sum<false>(sq, part[1]) + eps);
    if (threadIdx.x == 0) {
        if (mean) mean[row] = mu;
        if (rstd) rstd[row] = r;
    }
    for (int c = threadIdx.x; c < d; c += blockDim.x)
        y[row * ys + c] = from_f32<T>(fmaf((to_f32(xr[c]) - mu) * r, w ? to_f32(w[c]) : 1.0f, b ? to_f32(b[c]) : 0.0f));
}

// ---- backward ---------------------------------------------------------------------------------
__device__ __forceinline__ int cluster_rank()
{
    int r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ int cluster_size()
{
    int r;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier()  // all threads of all its CTAs
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// *addr = v in the shared memory of a CTA of the cluster
__device__ __forceinline__ void store_cluster(uint32_t addr, int cta, float2 v)
{
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(cta));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(v.x), "f"(v.y) : "memory");
}

// Sums of dw and db: every thread keeps those of its columns over all rows its CTA takes, and writes them to
// `partial` ([2][CTAs][d]) at the end; k_norm_param_gradient adds them up in a fixed order.  No atomics: the same
// bits from run to run.
template <typename T>
struct BackSums {
    float2 s1, s2;
    // g w, its sums, and the columns' sums, for one granule
    __device__ __forceinline__ void add(const Pairs<T> &vx, const Pairs<T> &vg, const float2 *wv, float2 m2, float2 r2,
                                        float2 *dw, float2 *db)
    {
#pragma unroll
        for (int k = 0; k < Pairs<T>::N; ++k) {
            const float2 gv = vg.get(k), xhat = mul2(add2(vx.get(k), m2), r2);
            const float2 gw = mul2(gv, wv[k]);
            s1 = add2(s1, gw);
            s2 = fma2(gw, xhat, s2);
            dw[k] = fma2(gv, xhat, dw[k]);
            db[k] = add2(db[k], gv);
        }
    }
};
// dx = rstd g w - rstd mean(g w) - xhat rstd mean(g w xhat) of one granule; f1 and f2 are the two means times -rstd
template <typename T>
__device__ __forceinline__ Pairs<T> input_gradient(const Pairs<T> &vx, const Pairs<T> &vg, const float2 *wv, float2 m2, float2 r2,
                                                   float2 f1, float2 f2)
{
    Pairs<T> out;
#pragma unroll
    for (int k = 0; k < Pairs<T>::N; ++k) {
        const float2 xhat = mul2(add2(vx.get(k), m2), r2);
        out.set(k, fma2(xhat, f2, fma2(mul2(vg.get(k), wv[k]), r2, f1)));
    }
    return out;
}

// A CTA is made of teams of `team_threads`, each with its own rows, ring and barrier, so that narrow rows still fill the
// multiprocessor while its columns' sums leave it once.  A team takes ROWS rows of x and dy per stage.  One barrier per
// stage: it ends the sums of this stage and, with it, all reads of the one before, which is refilled behind it.  E <= 16:
// weight, x and dy stay in registers between the two passes; E = 32: x and dy are read again, the weight lies in shared
// memory in the threads' order.
//
// SPLIT: a cluster of CTAs per row, each with its own columns (one team, one row per stage): rows that one CTA cannot hold.
// The warps leave their two sums in every CTA of the cluster, and the cluster's barrier takes the place of the team's.
// (Gradient of 4096 x 16384 binary32: 141 us, 5.7 TB/s, against 416 a value at a time.)
template <bool SHIFT, typename T, int E, int ROWS, bool SPLIT, typename P>
__global__ void __launch_bounds__(kNormRingThreads)
k_norm_backward_ring(const T *__restrict__ dy, long long dys, const T *__restrict__ x, long long xs,
                     const P *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd,
                     T *__restrict__ dx, long long dxs, float *__restrict__ partial, int n, int width, PhaseRows phases,
                     float inv_d, int team_threads, int stages, uint32_t row_bytes, int step, unsigned int *status)
{
    static_assert(!SPLIT || ROWS == 1, "a row per stage");
    constexpr int V = Pairs<T>::V, NV = E / V, NP = Pairs<T>::N;
    constexpr bool KEEP = E <= 16;
    extern __shared__ __align__(128) unsigned char rows[];
    __shared__ float2 part[2][ROWS][(SPLIT ? kNormMaxParts : 1) * kNormRingThreads / 32];
    __shared__ __align__(8) unsigned long long full[kNormMaxTeams][kNormMaxStages];
    __shared__ int lost[kNormMaxTeams];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = team_threads >> 5;
    const int team = threadIdx.x / team_threads, teams = blockDim.x / team_threads, tid = threadIdx.x - team * team_threads;
    const int parts = SPLIT ? cluster_size() : 1, rank = SPLIT ? cluster_rank() : 0;
    Walk walk = walk_of<V>(phases, blockIdx.x / parts, gridDim.x / parts, n);  // the CTA's phase, dealt to its teams
    int d = width;
    if constexpr (SPLIT) {  // from here on the CTA's columns are all there is
        const int all = team_threads * E, col0 = rank ? rank * all - walk.phase : 0;
        d = min(width - col0, rank ? all : all - walk.phase);
        if (rank) walk.phase = 0;
        x += col0;
        dy += col0;
        if (w) w += col0;
        if (dx) dx += col0;
        if (partial) partial += col0;
    }
    walk.first = walk.first * teams + team;
    walk.stride *= teams;
    const int groups = (walk.count + ROWS - 1) / ROWS;
    const uint32_t ring_bytes = stages * ROWS * 2 * row_bytes;
    RowRing ring = {smem_addr(rows) + team * ring_bytes, smem_addr(full[team]), ROWS * 2 * row_bytes, stages, true, step, status};
    if (tid < stages) barrier_init(ring.bar(tid), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if constexpr (SPLIT)
        cluster_barrier();  // the others run: their memory may be written
    else
        __syncthreads();
    grid_dependency_wait();
    grid_dependency_launch_next();
    auto team_barrier = [&]() {
        if constexpr (SPLIT)
            cluster_barrier();
        else
            asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(team_threads) : "memory");
    };
    auto row_of = [&](int g, int r) { return walk.row0 + walk.period * (g * ROWS + r); };
    auto load = [&](int i) {  // by one thread
        const int g = walk.first + i * walk.stride;
        if (g >= groups) return;
        const int count = min(ROWS, walk.count - g * ROWS);
        RowCopy copy[ROWS];
        uint32_t bytes = 0;
        for (int r = 0; r < count; ++r) {
            copy[r] = row_copy<T>(row_of(g, r), n, walk.phase, d);
            bytes += 2 * copy[r].bytes;
        }
        barrier_expect(ring.bar(i), bytes);
        for (int r = 0; r < count; ++r) {
            const long long row = row_of(g, r);
            const uint32_t dst = ring.at(i) + 2 * r * row_bytes + copy[r].skip;
            if (!copy[r].bytes || !RSDGC_IN_BOUNDS(copy_exists(x, xs, (int)row, walk.phase, copy[r], row_bytes, n, d) &&
                                                   copy_exists(dy, dys, (int)row, walk.phase, copy[r], row_bytes, n, d)))
                continue;
            bulk_copy(dst, reinterpret_cast<const unsigned char *>(x + row * xs - walk.phase) + copy[r].skip, copy[r].bytes,
                      ring.bar(i));
            bulk_copy(dst + row_bytes, reinterpret_cast<const unsigned char *>(dy + row * dys - walk.phase) + copy[r].skip,
                      copy[r].bytes, ring.bar(i));
        }
    };
    if (tid == 0)
        for (int i = 0; i + 1 < stages; ++i) load(i);

    const Columns<SHIFT, V, NV> cols(tid, team_threads, SHIFT ? walk.phase : 0, d, phases.same_out);
    float2 dw[NV][NP], db[NV][NP], wv[KEEP ? NV : 1][NP];
    float2 *const shared_w = reinterpret_cast<float2 *>(rows + teams * ring_bytes);  // the teams' columns are the same
    auto weight = [&](int i, float2 *out) {
#pragma unroll
        for (int k = 0; k < NP; ++k) out[k] = shared_w[(i * NP + k) * team_threads + tid];
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if constexpr (KEEP) {
            load_params<SHIFT, P, NP>(w, cols.at(i), d, 1.0f, wv[i]);
        } else {
            load_params<SHIFT, P, NP>(w, cols.at(i), d, 1.0f, wv[0]);
#pragma unroll
            for (int k = 0; k < NP; ++k) shared_w[(i * NP + k) * team_threads + tid] = wv[0][k];
        }
#pragma unroll
        for (int k = 0; k < NP; ++k) dw[i][k] = db[i][k] = make_float2(0.0f, 0.0f);
    }
    float nmu[ROWS], nr[ROWS];  // the next stage's statistics
    auto statistics = [&](int g) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const bool there = g * ROWS + r < walk.count && RSDGC_IN_BOUNDS(row_of(g, r) < n);
            nmu[r] = there ? mean[row_of(g, r)] : 0.0f;
            nr[r] = there ? rstd[row_of(g, r)] : 0.0f;
        }
    };
    statistics(walk.first);
    int it = 0;
    for (int g = walk.first; g < groups; g += walk.stride, ++it) {
        const int turn = it & 1;
        float mu[ROWS], rs[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) mu[r] = nmu[r], rs[r] = nr[r];
        statistics(g + walk.stride);
        ring.wait<KEEP>(it, tid == 0, lost[team]);
        Pairs<T> px[KEEP ? ROWS : 1][KEEP ? NV : 1], pg[KEEP ? ROWS : 1][KEEP ? NV : 1];
        auto operands = [&](auto fast, int r, int i, Pairs<T> &vx, Pairs<T> &vg) {
            constexpr bool FAST = decltype(fast)::value;
            const long long row = row_of(g, r);
            const bool edge = row == 0 || row == n - 1;
            const unsigned char *copy = rows + team * ring_bytes + ring.offset(it) + 2 * r * row_bytes;
            if (!RSDGC_IN_BOUNDS(row < n && cols.at(i) + walk.phase >= 0 &&
                                 (cols.at(i) + walk.phase + V) * (int)sizeof(T) <= (int)row_bytes))
                return;
            take<FAST>(vx, cols, i, copy, SHIFT ? walk.phase : 0, x + row * xs, edge);
            take<FAST>(vg, cols, i, copy + row_bytes, SHIFT ? walk.phase : 0, dy + row * dys, edge);
        };
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float2 m2 = make_float2(-mu[r], -mu[r]), r2 = make_float2(rs[r], rs[r]);
            BackSums<T> sums = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
            if (g * ROWS + r < walk.count)
                by_warp(cols.fast, [&](auto fast) {
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        if (cols.template any<decltype(fast)::value>(i)) {
                            Pairs<T> vx, vg;
                            operands(fast, r, i, vx, vg);
                            if constexpr (KEEP) {
                                px[r][i] = vx, pg[r][i] = vg;
                                sums.add(vx, vg, wv[i], m2, r2, dw[i], db[i]);
                            } else {
                                float2 wl[NP];
                                weight(i, wl);
                                sums.add(vx, vg, wl, m2, r2, dw[i], db[i]);
                            }
                        }
                    }
                });
            const float a = warp_sum(sums.s1.x + sums.s1.y), b = warp_sum(sums.s2.x + sums.s2.y);
            if constexpr (SPLIT) {
                if (lane < parts) store_cluster(smem_addr(&part[turn][r][rank * warps + warp]), lane, make_float2(a, b));
            } else {
                if (lane == 0) part[turn][r][warp] = make_float2(a, b);
            }
        }
        team_barrier();
        if (tid == 0 && ring.arrived) load(it + stages - 1);
        if (!dx) continue;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (g * ROWS + r >= walk.count) break;
            float2 t = make_float2(0.0f, 0.0f);
            if constexpr (SPLIT) {
                for (int i = lane; i < parts * warps; i += 32) t = add2(t, part[turn][r][i]);
            } else {
                if (lane < warps) t = part[turn][r][team * warps + lane];
            }
            const float c1 = -rs[r] * (warp_sum(t.x) * inv_d), c2 = -rs[r] * (warp_sum(t.y) * inv_d);
            const float2 m2 = make_float2(-mu[r], -mu[r]), r2 = make_float2(rs[r], rs[r]), f1 = make_float2(c1, c1),
                         f2 = make_float2(c2, c2);
            T *dst = dx + (long long)row_of(g, r) * dxs;
            by_warp(cols.fast, [&](auto fast) {
                constexpr bool FAST = decltype(fast)::value;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if (cols.template any<FAST>(i)) {
                        Pairs<T> out;
                        if constexpr (KEEP) {
                            out = input_gradient<T>(px[r][i], pg[r][i], wv[i], m2, r2, f1, f2);
                        } else {
                            Pairs<T> vx, vg;
                            float2 wl[NP];
                            operands(fast, r, i, vx, vg);
                            weight(i, wl);
                            out = input_gradient<T>(vx, vg, wl, m2, r2, f1, f2);
                        }
                        out.store(dst, cols.template stored_whole<FAST>(i), cols.at(i), d);
                    }
                }
            });
        }
    }
    if (!ring.arrived && tid == 0)
        ring.drain(min((groups - walk.first + walk.stride - 1) / walk.stride, lost[team] + stages - 1));
    if (!partial) return;
    // The teams' sums are added up in order, in the rings' memory (everything has arrived and been read): value e of a
    // thread's granules at [e][thread], 4 words of padding, so that neither the threads nor the columns' order meets a bank
    // conflict.
    float *const joined = reinterpret_cast<float *>(rows);
    int self, all;  // read anew: what follows from them need not live in registers through the rows' loop
    asm volatile("mov.u32 %0, %%tid.x;\n\tmov.u32 %1, %%ntid.x;" : "=r"(self), "=r"(all));
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                const float2 v = which ? db[i][k] : dw[i][k];
                joined[(i * V + 2 * k) * kNormJoin + self] = v.x;
                joined[(i * V + 2 * k + 1) * kNormJoin + self] = v.y;
            }
        __syncthreads();
        float *dst = partial + ((long long)which * (gridDim.x / parts) + blockIdx.x / parts) * width;
        for (int c0 = self; c0 < d; c0 += 4 * all) {  // four columns at a time, so that their loads overlap
            int from[4];
            float sum[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int at = min(c0 + u * all, d - 1) + (SHIFT ? walk.phase : 0), granule = at / V;
                const int i = granule / team_threads;
                from[u] = (i * V + at % V) * kNormJoin + granule - i * team_threads;
                if (!RSDGC_IN_BOUNDS(i < NV && from[u] >= 0 && from[u] + (all / team_threads - 1) * team_threads < E * kNormJoin)) from[u] = 0;
                sum[u] = joined[from[u]];
            }
            for (int k = 1; k < all / team_threads; ++k)
#pragma unroll
                for (int u = 0; u < 4; ++u) sum[u] += joined[k * team_threads + from[u]];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c0 + u * all < d) dst[c0 + u * all] = sum[u];
        }
    }
}

// A warp per row, a CTA's warps on rows of one phase; the next row is loaded while this one is reduced; the warps' column
// sums are joined in order at the end.  (16384 x 512 bfloat16: 16 us with k_norm_param_gradient, out of L2 in part.)
template <bool SHIFT, typename T, typename P>
__global__ void __launch_bounds__(32 * kBackWarps)
k_norm_backward_warp(const T *__restrict__ dy, long long dys, const T *__restrict__ x, long long xs,
                     const P *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd,
                     T *__restrict__ dx, long long dxs, float *__restrict__ partial, int n, int d, PhaseRows phases,
                     float inv_d)
{
    constexpr int V = Pairs<T>::V, NV = kNormElems / V, NP = Pairs<T>::N;
    __shared__ float joined[kBackWarps][32 * kNormElems];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Walk walk = walk_of<V>(phases, blockIdx.x, gridDim.x, n);  // the CTA's phase, dealt to its warps
    walk.first = walk.first * kBackWarps + warp;
    walk.stride *= kBackWarps;
    const Columns<SHIFT, V, NV> cols(lane, 32, SHIFT ? walk.phase : 0, d, phases.same_out);
    grid_dependency_wait();
    grid_dependency_launch_next();
    Pairs<T> nx[NV], ng[NV];
    float nmu = 0.0f, nr = 0.0f;
    auto fetch = [&](int j) {
        if (j >= walk.count) return;
        const long long row = walk.row0 + walk.period * j;
        const bool edge = near_end<V>(row, n, d);
        by_warp(cols.fast, [&](auto fast) {
            constexpr bool FAST = decltype(fast)::value;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (cols.template any<FAST>(i) &&
                    RSDGC_IN_BOUNDS(row < n && ((edge && !cols.template whole<FAST>(i)) ||
                                                (exist(row * xs + cols.at(i), V, xs, n, d) && exist(row * dys + cols.at(i), V, dys, n, d))))) {
                    take<FAST>(nx[i], cols, i, x + row * xs, edge);
                    take<FAST>(ng[i], cols, i, dy + row * dys, edge);
                }
        });
        nmu = mean[row];
        nr = rstd[row];
    };
    fetch(walk.first);
    float2 dw[NV][NP], db[NV][NP], wv[NV][NP];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load_params<SHIFT, P, NP>(w, cols.at(i), d, 1.0f, wv[i]);
#pragma unroll
        for (int k = 0; k < NP; ++k) dw[i][k] = db[i][k] = make_float2(0.0f, 0.0f);
    }
    for (int j = walk.first; j < walk.count; j += walk.stride) {
        Pairs<T> cx[NV], cg[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) cx[i] = nx[i], cg[i] = ng[i];
        const float mu = nmu, r = nr;
        fetch(j + walk.stride);
        const float2 m2 = make_float2(-mu, -mu), r2 = make_float2(r, r);
        BackSums<T> sums = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
        by_warp(cols.fast, [&](auto fast) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (cols.template any<decltype(fast)::value>(i)) sums.add(cx[i], cg[i], wv[i], m2, r2, dw[i], db[i]);
        });
        const float c1 = -r * (warp_sum(sums.s1.x + sums.s1.y) * inv_d), c2 = -r * (warp_sum(sums.s2.x + sums.s2.y) * inv_d);
        if (dx) {
            T *dst = dx + (long long)(walk.row0 + walk.period * j) * dxs;
            by_warp(cols.fast, [&](auto fast) {
                constexpr bool FAST = decltype(fast)::value;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (cols.template any<FAST>(i))
                        input_gradient<T>(cx[i], cg[i], wv[i], m2, r2, make_float2(c1, c1), make_float2(c2, c2))
                            .store(dst, cols.template stored_whole<FAST>(i), cols.at(i), d);
            });
        }
    }
    if (!partial) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float *dst = partial + ((long long)which * gridDim.x + blockIdx.x) * d;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                const int c = cols.at(i) + 2 * k;
                const float2 v = which ? db[i][k] : dw[i][k];
                if (!RSDGC_IN_BOUNDS(d <= 32 * kNormElems)) continue;
                if ((unsigned)c < (unsigned)d) joined[warp][c] = v.x;
                if ((unsigned)(c + 1) < (unsigned)d) joined[warp][c + 1] = v.y;
            }
        __syncthreads();
        for (int c = threadIdx.x; c < d; c += 32 * kBackWarps) {
            float t = joined[0][c];
#pragma unroll
            for (int k = 1; k < kBackWarps; ++k) t += joined[k][c];
            dst[c] = t;
        }
    }
}

// Any layout and width, a value at a time: two reads of the row; a second kernel walks the columns.  (4096 x 16384
// binary32: 242 and 172 us, where the split rows take 141 for both.)
template <typename T, typename P>
__global__ void __launch_bounds__(kNormLongThreads)
k_norm_backward_any(const T *__restrict__ dy, long long dys, const T *__restrict__ x, long long xs,
                    const P *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd,
                    T *__restrict__ dx, long long dxs, int d, float inv_d)
{
    __shared__ float part[2][32];
    grid_dependency_wait();
    grid_dependency_launch_next();
    const long long row = blockIdx.x;
    const float mu = mean[row], r = rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x; c < d; c += blockDim.x) {
        const float gw = to_f32(dy[row * dys + c]) * (w ? to_f32(w[c]) : 1.0f);
        s1 += gw;
        s2 = fmaf(gw, (to_f32(x[row * xs + c]) - mu) * r, s2);
    }
    const float m1 = row_sum<false>(s1, part[0]) * inv_d, m2 = row_sum<false>(s2, part[1]) * inv_d;
    for (int c = threadIdx.x; c < d; c += blockDim.x) {
        const float gw = to_f32(dy[row * dys + c]) * (w ? to_f32(w[c]) : 1.0f);
        dx[row * dxs + c] = from_f32<T>(r * (gw - m1 - (to_f32(x[row * xs + c]) - mu) * r * m2));
    }
}
// ... a thread per column, a range of rows per CTA row
template <typename T>
__global__ void __launch_bounds__(256)
k_norm_columns_any(const T *__restrict__ dy, long long dys, const T *__restrict__ x, long long xs,
                   const float *__restrict__ mean, const float *__restrict__ rstd, float *__restrict__ partial,
                   long long n, int d)
{
    grid_dependency_wait();
    grid_dependency_launch_next();
    const int c = blockIdx.x * 256 + threadIdx.x;
    const long long per = (n + gridDim.y - 1) / gridDim.y, lo = per * blockIdx.y, hi = min(n, lo + per);
    if (c >= d) return;
    float dw = 0.0f, db = 0.0f;
    for (long long row = lo; row < hi; ++row) {
        const float g = to_f32(dy[row * dys + c]);
        dw = fmaf(g, (to_f32(x[row * xs + c]) - mean[row]) * rstd[row], dw);
        db += g;
    }
    partial[(long long)blockIdx.y * d + c] = dw;
    partial[((long long)gridDim.y + blockIdx.y) * d + c] = db;
}

// dw[c] = sum over the slots of partial[0][slot][c], db likewise: 32 columns x blockDim.x / 32 slot lanes per CTA.
template <typename Q>
__global__ void __launch_bounds__(1024)
k_norm_param_gradient(const float *__restrict__ partial, int slots, int d, Q *__restrict__ dw, Q *__restrict__ db)
{
    __shared__ float sum[32][33];
    const int lane = threadIdx.x & 31, k = threadIdx.x >> 5, lanes = blockDim.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    Q *out = blockIdx.y ? db : dw;
    grid_dependency_wait();
    grid_dependency_launch_next();
    if (!out) return;
    const float *src = partial + (long long)blockIdx.y * slots * d + c;
    float a[4] = {};
    if (c < d) {
        for (int i = k; i < slots; i += 4 * lanes) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u * lanes < slots) a[u] += src[(long long)(i + u * lanes) * d];
        }
    }
    sum[k][lane] = (a[0] + a[1]) + (a[2] + a[3]);
    __syncthreads();
    if (k || c >= d) return;
    float t = sum[0][lane];
    for (int i = 1; i < lanes; ++i) t += sum[i][lane];
    out[c] = from_f32<Q>(t);
}

RSDGC_DEFINE_DEBUG_BOUNDS(layer_norm_debug_bounds)

namespace {

// How the rows of a call can be walked: `packs` granules at most, in PhaseRows, if all inputs' rows have the same
// phases.  The sums' order depends on the inputs' layout alone, the output's decides how it is stored.
struct NormShape {
    bool packed, shift;
    int packs;
    PhaseRows phases;
    int threads(int elems, int v) const { return ((packs * v + elems - 1) / elems + 31) / 32 * 32; }
};
struct Operand {
    const void *p;
    long long stride;
};
NormShape norm_shape(int d, int elem, std::initializer_list<Operand> inputs, Operand output,
                     std::initializer_list<const void *> params, long long n)
{
    const int v = 16 / elem;
    NormShape s{true, d % v != 0, 0, {1, 0, 0, true}};
    auto phase = [&](const Operand &o) { return (int)((reinterpret_cast<uintptr_t>(o.p) & 15) / elem); };
    auto step = [&](const Operand &o) { return n > 1 ? (int)(o.stride & (v - 1)) : 0; };
    s.phases.phase0 = phase(*inputs.begin());
    s.phases.step = step(*inputs.begin());
    for (const Operand &o : inputs)
        if (phase(o) != s.phases.phase0 || step(o) != s.phases.step) s.packed = false;
    if (output.p) s.phases.same_out = phase(output) == s.phases.phase0 && step(output) == s.phases.step;
    while ((s.phases.period * s.phases.step) & (v - 1)) s.phases.period *= 2;
    const bool shifted = s.phases.phase0 || s.phases.step;
    s.packs = (d + (shifted ? v - 1 : 0) + v - 1) / v;
    if (shifted || !s.phases.same_out) s.shift = true;
    for (const void *p : params)
        if (!pointer_aligned(p, 16)) s.shift = true;
    return s;
}

// walkers, a multiple of the period, at most `most` and no more than there are rows for
unsigned walkers(long long rows, long long most, int period)
{
    long long g = rows < most ? rows : most;
    g = (g + period - 1) / period * period;
    return (unsigned)g;
}

// Slots: CTAs whose sums of dw and db are added up at the end; at most one per multiprocessor in the ring, kNormAnySlots in the
// general form, two to three per multiprocessor in the warp's form: what they write and what is read again, 16 bytes per slot
// and column, stays under a tenth of the rows' own traffic, 6 bytes per row and column, unless rows are few.  Multiprocessors
// beyond a B200's 148 get no slots, so that the workspace's size does not depend on the device.
constexpr int kNormSlotSms = 148;
constexpr int kNormAnySlots = 64;
constexpr int kNormMaxPeriod = 8;
int slot_sms()
{
    const int sms = current_device_sms();
    return sms < kNormSlotSms ? sms : kNormSlotSms;
}
int warp_slots(long long n)
{
    const long long few = 2ll * slot_sms(), most = 3ll * slot_sms(), s = n / 27;
    return (int)(s < few ? few : s < most ? s : most);
}
// The most that a gradient of n rows may use, whatever their layout and width: a row per CTA of the ring, a row per warp,
// rounded up to a period; one for none.
int64_t norm_slots(int64_t n)
{
    const int64_t ring = n < kNormSlotSms ? n : kNormSlotSms, rows = (n + kBackWarps - 1) / kBackWarps,
                  warp = rows < 3 * kNormSlotSms ? rows : 3 * kNormSlotSms, most = ring > warp ? ring : warp;
    static_assert(kNormAnySlots <= kNormSlotSms, "the general form has no more than the ring");
    return most ? (most + kNormMaxPeriod - 1) / kNormMaxPeriod * kNormMaxPeriod : 1;
}

int poll_step() { return (int)(kOperatorPolls / operator_polls()); }

// Lets `kernel` have the rings' shared memory, once per device (`ready`: a bit per device).
template <typename K>
cudaError_t allow_ring(K kernel, std::atomic<uint64_t> &ready)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (ready.load() >> (dev & 63) & 1)) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormRingBytes);
    if (e == cudaSuccess) ready.fetch_or(1ull << (dev & 63));
    return e;
}

// CTAs per multiprocessor and stages per ring: as many CTAs as the registers allow and the shared memory holds with three
// stages each (`more` bytes per CTA besides); no stages if there is not room for `least`.
struct RingShape {
    int ctas, stages;
};
RingShape ring_shape(int threads, int registers, long long stage, int least, long long more = 0)
{
    RingShape r{65536 / (registers * threads), 0};
    if (r.ctas > 2048 / threads) r.ctas = 2048 / threads;
    if (r.ctas > 16) r.ctas = 16;
    while (r.ctas > 1 && kNormRingBytes / r.ctas < 3 * stage + more) --r.ctas;
    if (r.ctas < 1) r.ctas = 1;
    r.stages = (int)((kNormRingBytes / r.ctas - more) / stage);
    if (r.stages > kNormMaxStages) r.stages = kNormMaxStages;
    if (r.stages < least) r.stages = 0;
    return r;
}

template <typename T, typename P>
struct ForwardArgs {
    const T *x;
    long long xs;
    const P *w, *b;
    T *y;
    long long ys;
    float *mean, *rstd;
    int n, d;
    float inv, root, eps;
    cudaStream_t s;
};

template <bool SHIFT, typename T, typename P, int E>
bool forward_ring(cudaError_t *e, const ForwardArgs<T, P> &a, const NormShape &sh)
{
    const int threads = sh.threads(E, Pairs<T>::V);
    if (threads > kNormRingThreads) return false;
    const RingShape ring = ring_shape(threads, E <= 16 ? 64 : 128, 16ll * sh.packs, 2);
    if (!ring.stages) return false;
    static std::atomic<uint64_t> ready{0};
    unsigned int *status = nullptr;
    *e = operator_status_ptr(&status);
    if (*e == cudaSuccess) *e = allow_ring(k_norm_forward_ring<SHIFT, T, P, E>, ready);
    if (*e != cudaSuccess) return true;
    *e = launch_chained(k_norm_forward_ring<SHIFT, T, P, E>,
                        walkers(a.n, (long long)ring.ctas * current_device_sms() / sh.phases.period * sh.phases.period,
                                sh.phases.period),
                        threads, (size_t)ring.stages * 16 * sh.packs, a.s, 1, a.x, a.xs, a.w, a.b, a.y, a.ys, a.mean, a.rstd, a.n,
                        a.d, sh.phases, a.inv, a.root, a.eps, ring.stages, 16u * (uint32_t)sh.packs, poll_step(), status);
    return true;
}

template <bool SHIFT, typename T, typename P>
bool norm_forward_packed(cudaError_t *e, const ForwardArgs<T, P> &a, const NormShape &sh)
{
    if (sh.packs <= 32 * kNormElems / Pairs<T>::V) {
        // as many warps as fit the device at a time, a row each at least
        const unsigned g = walkers((a.n + kNormWarps - 1) / kNormWarps, 8ll * current_device_sms(), sh.phases.period);
        *e = launch_chained(k_norm_forward_warp<SHIFT, T, P>, g, 32 * kNormWarps, 0, a.s, 1, a.x, a.xs, a.w, a.b, a.y, a.ys,
                            a.mean, a.rstd, a.n, a.d, sh.phases, a.inv, a.root, a.eps);
        return true;
    }
    return forward_ring<SHIFT, T, P, 16>(e, a, sh) || forward_ring<SHIFT, T, P, 32>(e, a, sh);
}

template <typename T, typename P>
cudaError_t norm_forward(const ForwardArgs<T, P> &a)
{
    const NormShape sh = norm_shape(a.d, (int)sizeof(T), {{a.x, a.xs}}, {a.y, a.ys}, {a.w, a.b}, a.n);
    cudaError_t e = cudaSuccess;
    if (sh.packed && (sh.shift ? norm_forward_packed<true>(&e, a, sh) : norm_forward_packed<false>(&e, a, sh))) return e;
    return launch_chained(k_norm_forward_any<T, P>, (unsigned)a.n, kNormLongThreads, 0, a.s, 1, a.x, a.xs, a.w, a.b, a.y, a.ys,
                          a.mean, a.rstd, a.d, a.inv, a.root, a.eps);
}

template <typename T, typename P>
struct BackwardArgs {
    const T *dy;
    long long dys;
    const T *x;
    long long xs;
    const P *w;
    const float *mean, *rstd;
    T *dx;
    long long dxs;
    float *partial;   // NULL: no dw, no db
    int n, d;
    float inv;
    cudaStream_t s;
};

// Teams of the backward ring: as many as the registers (128 a thread) and the shared memory hold, unless rows are so few
// that they rather spread over the device.
struct TeamShape {
    int threads, teams, stages;
    int warps() const { return threads / 32 * teams; }
};
template <typename T>
TeamShape team_shape(const NormShape &sh, int elems, int rows, long long n)
{
    TeamShape t{sh.threads(elems, Pairs<T>::V), 0, 0};
    if (t.threads > kNormRingThreads) return t;
    const long long stage = 2ll * rows * 16 * sh.packs, weight = elems > 16 ? 4ll * elems * t.threads : 0;
    const long long groups = (n + rows - 1) / rows, share = (groups + current_device_sms() - 1) / current_device_sms();
    t.teams = kNormRingThreads / t.threads;
    if (t.teams > kNormMaxTeams) t.teams = kNormMaxTeams;
    if (t.teams > share) t.teams = (int)share;
    while (t.teams > 1 && (kNormRingBytes - weight) / t.teams < 3 * stage) --t.teams;
    t.stages = (int)((kNormRingBytes - weight) / t.teams / stage);
    if (t.stages > kNormMaxStages) t.stages = kNormMaxStages;
    if (t.stages < (rows > 1 ? 3 : 2)) t.teams = 0;
    return t;
}

// How a row is split over the CTAs of a cluster, two stages each at least; no parts if it cannot be.
struct SplitShape {
    TeamShape team;
    int parts;
    uint32_t row;  // bytes of a part's row
};
template <typename T>
SplitShape split_shape(const NormShape &sh)
{
    SplitShape r{{0, 1, 0}, 0, 0};
    constexpr int V = Pairs<T>::V;
    for (int parts = 2; parts <= kNormMaxParts && !r.parts; ++parts) {
        const int threads = ((sh.packs * V + parts * kNormElems - 1) / (parts * kNormElems) + 31) / 32 * 32;
        if (threads > kNormRingThreads) continue;
        r.row = (uint32_t)(threads * kNormElems * sizeof(T));
        r.team.threads = threads;
        r.team.stages = kNormRingBytes / (2 * (int)r.row);
        if (r.team.stages > kNormMaxStages) r.team.stages = kNormMaxStages;
        // the columns are dealt from the first part on; no part is left without any, whatever the phase: a part less would
        // have to hold kNormRingThreads * kNormElems columns in each of the others
        r.parts = (sh.packs * V + threads * kNormElems - 1) / (threads * kNormElems);
    }
    return r;
}

template <bool SHIFT, typename T, int E, int ROWS, bool SPLIT, typename P>
cudaError_t backward_ring(int *slots, const BackwardArgs<T, P> &a, const NormShape &sh, const TeamShape &t, uint32_t row,
                          int parts)
{
    const long long loop = (long long)t.teams * t.stages * 2 * ROWS * row + (E > 16 ? 4ll * E * t.threads : 0);
    const long long join = 4ll * E * kNormJoin, smem = loop > join ? loop : join;
    static std::atomic<uint64_t> ready{0};
    unsigned int *status = nullptr;
    cudaError_t e = operator_status_ptr(&status);
    if (e == cudaSuccess) e = allow_ring(k_norm_backward_ring<SHIFT, T, E, ROWS, SPLIT, P>, ready);
    if (e != cudaSuccess) return e;
    const int per = ROWS * t.teams, period = sh.phases.period;
    *slots = (int)walkers((a.n + per - 1) / per, slot_sms() / parts / period * period, period);
    return launch_chained(k_norm_backward_ring<SHIFT, T, E, ROWS, SPLIT, P>, (unsigned)(*slots * parts), t.threads * t.teams,
                          (size_t)smem, a.s, parts, a.dy, a.dys, a.x, a.xs, a.w, a.mean, a.rstd, a.dx, a.dxs, a.partial, a.n,
                          a.d, sh.phases, a.inv, t.threads, t.stages, row, poll_step(), status);
}

template <bool SHIFT, typename T, typename P>
bool norm_backward_packed(cudaError_t *e, int *slots, const BackwardArgs<T, P> &a, const NormShape &sh)
{
    if (sh.packs <= 32 * kNormElems / Pairs<T>::V) {
        *slots = (int)walkers((a.n + kBackWarps - 1) / kBackWarps, warp_slots(a.n), sh.phases.period);
        *e = launch_chained(k_norm_backward_warp<SHIFT, T, P>, (unsigned)*slots, 32 * kBackWarps, 0, a.s, 1, a.dy, a.dys, a.x, a.xs,
                            a.w, a.mean, a.rstd, a.dx, a.dxs, a.partial, a.n, a.d, sh.phases, a.inv);
        return true;
    }
    const uint32_t row = 16u * (uint32_t)sh.packs;
    // binary32 rows: a second row per stage does not fit the registers (8192 x 1001 takes 58 us with it, 28 without), and
    // what one CTA cannot hold at 16 columns per thread is better split than held at 32 (4096 x 9000: 103 us against 109, side by
    // side)
    const TeamShape one = team_shape<T>(sh, 16, 1, a.n);
    if constexpr (sizeof(T) < 4) {
        // two rows per stage where they fit; twice the columns per thread where that fills the multiprocessor better (a row
        // of 4100 columns takes 9 of its 16 warps, or three rows 15)
        const TeamShape two = team_shape<T>(sh, 16, 2, a.n), wide = team_shape<T>(sh, 32, 1, a.n);
        const TeamShape &narrow = two.teams ? two : one;
        if (narrow.teams && 3 * wide.warps() < 4 * narrow.warps()) {
            *e = two.teams ? backward_ring<SHIFT, T, 16, 2, false, P>(slots, a, sh, two, row, 1)
                           : backward_ring<SHIFT, T, 16, 1, false, P>(slots, a, sh, one, row, 1);
            return true;
        }
        if (wide.teams) {
            *e = backward_ring<SHIFT, T, 32, 1, false, P>(slots, a, sh, wide, row, 1);
            return true;
        }
    } else if (one.teams) {
        *e = backward_ring<SHIFT, T, 16, 1, false, P>(slots, a, sh, one, row, 1);
        return true;
    }
    const SplitShape split = split_shape<T>(sh);
    if (split.parts) *e = backward_ring<SHIFT, T, 16, 1, true, P>(slots, a, sh, split.team, split.row, split.parts);
    return split.parts > 0;
}

template <typename T, typename P>
cudaError_t norm_backward(const BackwardArgs<T, P> &a, void *dw, void *db, int grad_type)
{
    const NormShape sh = norm_shape(a.d, (int)sizeof(T), {{a.x, a.xs}, {a.dy, a.dys}}, {a.dx, a.dxs}, {a.w}, a.n);
    int slots = 0;
    cudaError_t e = cudaSuccess;
    if (!sh.packed ||
        !(sh.shift ? norm_backward_packed<true>(&e, &slots, a, sh) : norm_backward_packed<false>(&e, &slots, a, sh))) {
        if (a.dx)
            e = launch_chained(k_norm_backward_any<T, P>, (unsigned)a.n, kNormLongThreads, 0, a.s, 1, a.dy, a.dys, a.x, a.xs,
                               a.w, a.mean, a.rstd, a.dx, a.dxs, a.d, a.inv);
        if (e == cudaSuccess && a.partial) {
            slots = a.n < kNormAnySlots ? a.n : kNormAnySlots;
            e = launch_chained(k_norm_columns_any<T>, dim3((unsigned)((a.d + 255) / 256), (unsigned)slots), 256, 0, a.s, 1,
                               a.dy, a.dys, a.x, a.xs, a.mean, a.rstd, a.partial, (long long)a.n, a.d);
        }
    }
    if (e != cudaSuccess || !a.partial) return e;
    const dim3 grid((unsigned)((a.d + 31) / 32), 2);
    const int lanes = slots >= 256 ? 32 : slots >= 128 ? 16 : slots >= 16 ? 8 : 1;
    const float *part = a.partial;
    if (grad_type == RSDGC_F32)
        return launch_chained(k_norm_param_gradient<float>, grid, 32 * lanes, 0, a.s, 1, part, slots, a.d, (float *)dw, (float *)db);
    if (grad_type == RSDGC_BF16)
        return launch_chained(k_norm_param_gradient<__nv_bfloat16>, grid, 32 * lanes, 0, a.s, 1, part, slots, a.d,
                              (__nv_bfloat16 *)dw, (__nv_bfloat16 *)db);
    return launch_chained(k_norm_param_gradient<__half>, grid, 32 * lanes, 0, a.s, 1, part, slots, a.d, (__half *)dw, (__half *)db);
}

// Element and parameter type of a call: the parameters have the rows' type or binary32.
template <typename F>
cudaError_t with_types(int dtype, int param, F f)
{
    if (dtype == RSDGC_F32) return f(float{}, float{});
    if (dtype == RSDGC_BF16)
        return param == RSDGC_F32 ? f(__nv_bfloat16{}, float{}) : f(__nv_bfloat16{}, __nv_bfloat16{});
    return param == RSDGC_F32 ? f(__half{}, float{}) : f(__half{}, __half{});
}

int norm_check(int64_t n, int64_t d, int dtype, int param)
{
    if (n < 0 || d < 1 || !known_dtype(dtype) || !known_dtype(param)) return RSDGC_ERR_INVALID;
    if (param != dtype && param != RSDGC_F32) return RSDGC_ERR_INVALID;
    if (n > (1 << 30) || d > (1 << 24)) return RSDGC_ERR_CAPACITY;
    return RSDGC_OK;
}

}  // namespace
}  // namespace rsdgc

using namespace rsdgc;

extern "C" int64_t rsdgc_layer_norm_workspace_bytes(int64_t n_rows, int64_t width)
{
    if (n_rows < 0 || width < 1) return RSDGC_ERR_INVALID;
    if (n_rows > (1 << 30) || width > (1 << 24)) return RSDGC_ERR_CAPACITY;
    return 2 * 4 * norm_slots(n_rows) * width;
}

extern "C" int rsdgc_layer_norm_forward(const void *x_dev, int64_t x_stride, const void *weight_dev,
                                        const void *bias_dev, void *y_dev, int64_t y_stride, float *mean_dev,
                                        float *rstd_dev, int64_t n_rows, int64_t width, int32_t dtype,
                                        int32_t param_dtype, float eps, void *stream)
{
    int rc = norm_check(n_rows, width, dtype, param_dtype);
    if (rc) return rc;
    if (!(eps >= 0.0f)) return RSDGC_ERR_INVALID;
    if (n_rows == 0) return RSDGC_OK;
    if (!x_dev || !y_dev || x_stride < width || y_stride < width) return RSDGC_ERR_INVALID;
    if (!pointer_aligned(x_dev, dtype_bytes(dtype)) || !pointer_aligned(y_dev, dtype_bytes(dtype)) ||
        !pointer_aligned(weight_dev, dtype_bytes(param_dtype)) || !pointer_aligned(bias_dev, dtype_bytes(param_dtype)) ||
        !pointer_aligned(mean_dev, 4) || !pointer_aligned(rstd_dev, 4))
        return RSDGC_ERR_ALIGNMENT;
    OperatorRange range("rsdgc_layer_norm_forward");
    cudaError_t e = operators_ready();
    if (e != cudaSuccess) return operator_result(e);
    e = with_types(dtype, param_dtype, [&](auto t, auto p) {
        typedef decltype(t) T;
        typedef decltype(p) P;
        return norm_forward<T, P>({(const T *)x_dev, x_stride, (const P *)weight_dev, (const P *)bias_dev, (T *)y_dev, y_stride,
                                   mean_dev, rstd_dev, (int)n_rows, (int)width, 1.0f / (float)width,
                                   1.0f / std::sqrt((float)width), eps, (cudaStream_t)stream});
    });
    return operator_result(e);
}

extern "C" int rsdgc_layer_norm_backward(const void *dy_dev, int64_t dy_stride, const void *x_dev, int64_t x_stride,
                                         const void *weight_dev, const float *mean_dev, const float *rstd_dev,
                                         void *dx_dev, int64_t dx_stride, void *dweight_dev, void *dbias_dev,
                                         int32_t grad_dtype, int64_t n_rows, int64_t width, int32_t dtype,
                                         int32_t param_dtype, void *workspace_dev, void *stream)
{
    int rc = norm_check(n_rows, width, dtype, param_dtype);
    if (rc) return rc;
    if (!known_dtype(grad_dtype)) return RSDGC_ERR_INVALID;
    if (!dx_dev && !dweight_dev && !dbias_dev) return RSDGC_ERR_INVALID;
    if ((dweight_dev || dbias_dev) && !workspace_dev) return RSDGC_ERR_INVALID;
    if (!pointer_aligned(workspace_dev, 16)) return RSDGC_ERR_ALIGNMENT;
    if (n_rows > 0) {
        if (!dy_dev || !x_dev || !mean_dev || !rstd_dev || dy_stride < width || x_stride < width ||
            (dx_dev && dx_stride < width))
            return RSDGC_ERR_INVALID;
        const int b = dtype_bytes(dtype);
        if (!pointer_aligned(dy_dev, b) || !pointer_aligned(x_dev, b) || !pointer_aligned(dx_dev, b) ||
            !pointer_aligned(weight_dev, dtype_bytes(param_dtype)) || !pointer_aligned(mean_dev, 4) ||
            !pointer_aligned(rstd_dev, 4))
            return RSDGC_ERR_ALIGNMENT;
    }
    if (!pointer_aligned(dweight_dev, dtype_bytes(grad_dtype)) || !pointer_aligned(dbias_dev, dtype_bytes(grad_dtype)))
        return RSDGC_ERR_ALIGNMENT;
    OperatorRange range("rsdgc_layer_norm_backward");
    cudaStream_t s = (cudaStream_t)stream;
    if (n_rows == 0) {  // sums over nothing
        cudaError_t e = cudaSuccess;
        const size_t bytes = (size_t)width * dtype_bytes(grad_dtype);
        if (dweight_dev) e = cudaMemsetAsync(dweight_dev, 0, bytes, s);
        if (dbias_dev && e == cudaSuccess) e = cudaMemsetAsync(dbias_dev, 0, bytes, s);
        return operator_result(e);
    }
    cudaError_t e = operators_ready();
    if (e != cudaSuccess) return operator_result(e);
    e = with_types(dtype, param_dtype, [&](auto t, auto p) {
        typedef decltype(t) T;
        typedef decltype(p) P;
        return norm_backward<T, P>({(const T *)dy_dev, dy_stride, (const T *)x_dev, x_stride, (const P *)weight_dev, mean_dev,
                                    rstd_dev, (T *)dx_dev, dx_stride,
                                    dweight_dev || dbias_dev ? (float *)workspace_dev : nullptr, (int)n_rows, (int)width,
                                    1.0f / (float)width, s},
                                   dweight_dev, dbias_dev, grad_dtype);
    });
    return operator_result(e);
}
