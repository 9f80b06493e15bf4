// Layer norm, forward and backward, with the reduction of the weight's and the bias's gradient.
//
//   mean = sum x / D,  rstd = (sum (x - mean)^2 / D + eps)^(-1/2),  xhat = (x - mean) rstd,  y = xhat w + b
//   dx = rstd (g w - mean(g w) - xhat mean(g w xhat)),  dw = sum_n g xhat,  db = sum_n g
//
// Bound: memory (about 2 flop per byte).  A row is read once and stays in registers: the mean, then the
// centred squares (two reductions, no cancellation), then the output.  All statistics and sums are binary32.
#include <atomic>
#include <climits>

#include "device_utils.cuh"
#include "operators_internal.cuh"

namespace rsdgc {

constexpr int kNormVecs = 2;          // 16-byte packs of a row that a lane holds where a warp takes the row
constexpr int kNormScalars = 16;      // elements a thread holds where rows are not 16-byte aligned
constexpr int kNormRingThreads = 512;
constexpr int kNormMaxThreads = 1024;
constexpr int kNormBackThreads = 512; // backward: 128 registers for the columns' sums and the rows' operands
constexpr int kBackWarps = 8;         // warps of a CTA whose rows take one warp each, backward
constexpr int kNormMaxStages = 4;
constexpr int kNormRingBytes = 200 << 10;  // shared memory of a multiprocessor's rings
constexpr unsigned kNormSpin = 1u << 20;   // polls of a wait before it gives up
constexpr int kNormWarps = 4;         // warps of a CTA whose rows take one warp each

// Elements of a row as `VEC` packed values; VEC = 1 where rows do not start on 16-byte boundaries.
template <typename T, int VEC>
struct __align__(sizeof(T) * VEC < 16 ? sizeof(T) * VEC : 16) Pack {
    T v[VEC];
};

template <typename T, int VEC>
__device__ __forceinline__ Pack<T, VEC> load_pack(const T *p)
{
    return *reinterpret_cast<const Pack<T, VEC> *>(p);
}
// parameters may have another type than the rows: the widest load that their own alignment allows
template <typename P, int VEC>
__device__ __forceinline__ void load_param(const P *p, long long i, float *out)
{
    const Pack<P, VEC> k = *reinterpret_cast<const Pack<P, VEC> *>(p + i);
#pragma unroll
    for (int j = 0; j < VEC; ++j) out[j] = to_f32(k.v[j]);
}

// A 16-byte pack as pairs of binary32 values: the arithmetic runs two values per instruction (f32x2), which matters
// because rows of 16-bit values are bound by the issue rate, not by memory, at one instruction per value and step.
template <typename T>
struct Pairs {
    static constexpr int N = 8 / (int)sizeof(T);  // pairs of a pack
    uint32_t w[4];
    __device__ __forceinline__ void load(const T *p)
    {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]); }
    __device__ __forceinline__ float2 get(int i) const;
    __device__ __forceinline__ void set(int i, float2 v);
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
// `count` pairs of a parameter vector, or a constant where there is none
template <typename P, int PAIRS>
__device__ __forceinline__ void load_pairs(const P *p, long long c, bool there, float missing, float2 *out)
{
    if (p && there) {
#pragma unroll
        for (int k = 0; k < PAIRS / Pairs<P>::N; ++k) {
            Pairs<P> v;
            v.load(p + c + k * (16 / (int)sizeof(P)));
#pragma unroll
            for (int i = 0; i < Pairs<P>::N; ++i) out[k * Pairs<P>::N + i] = v.get(i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) out[i] = make_float2(missing, missing);
    }
}

// Sum over the threads of one row.  One warp per row: shuffles only.  Otherwise the whole CTA, one slot of
// `part` per warp; the caller alternates between two buffers, so that one barrier per sum is enough.
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
template <bool WARP>
__device__ __forceinline__ float2 row_sum2(float x, float y, float2 *part)
{
    x = warp_sum(x);
    y = warp_sum(y);
    if (WARP) return make_float2(x, y);
    const int warps = (int)(blockDim.x >> 5), lane = threadIdx.x & 31;
    if (lane == 0) part[threadIdx.x >> 5] = make_float2(x, y);
    __syncthreads();
    const float2 z = lane < warps ? part[lane] : make_float2(0.0f, 0.0f);
    return make_float2(warp_sum(z.x), warp_sum(z.y));
}

// A ring of stages in shared memory, each `operands` rows, filled by bulk copies that run `stages` - 1 (or more) rows
// ahead, so that a CTA has tens of KB on their way whatever its threads wait for.
struct RowRing {
    uint32_t base, full;   // shared-memory addresses: rows, barriers (8 bytes each)
    uint32_t stage_bytes;
    int stages;
    bool arrived;          // false once a wait has given up: the results are void, as the status says
    unsigned int *status;

    __device__ __forceinline__ uint32_t bar(int i) const { return full + 8 * (i % stages); }
    __device__ __forceinline__ uint32_t at(int i) const { return base + (i % stages) * stage_bytes; }
    // bounded; after a failure the others poll once
    __device__ __forceinline__ void wait(int i)
    {
        unsigned left = arrived ? kNormSpin : 1u;
        bool here = false;
        while (left-- && !(here = barrier_try(bar(i), (uint32_t)(i / stages) & 1u))) {}
        if (!here && arrived) {
            arrived = false;
            atomicOr(status, RSDGC_STATUS_TIMEOUT);
        }
    }
    // copies under way after a failure land in this CTA's memory: wait for them (bounded)
    __device__ __forceinline__ void drain(int from, int to) const
    {
        for (int i = from < 0 ? 0 : from; i < to; ++i)
            for (unsigned q = 0; q < kNormSpin && !barrier_try(bar(i), (uint32_t)(i / stages) & 1u); ++q) {}
    }
};
template <typename T>
__device__ __forceinline__ const T *shared_row(uint32_t addr)
{
    return reinterpret_cast<const T *>(__cvta_shared_to_generic(addr));
}

// ---- forward ----------------------------------------------------------------------------------
// Aligned rows: a CTA walks the rows blockIdx.x, blockIdx.x + gridDim.x, ...; its threads keep their columns' weight
// and bias as binary32 pairs.  Two barriers per row (mean, then the centred squares); the next rows arrive meanwhile.
template <typename T, typename P, int E>
__global__ void __launch_bounds__(kNormRingThreads, E <= 16 ? 2 : 1)
k_norm_forward_ring(const T *__restrict__ x, long long xs, const P *__restrict__ w, const P *__restrict__ b,
                    T *__restrict__ y, long long ys, float *__restrict__ mean, float *__restrict__ rstd, int n, int d,
                    float inv_d, float root_inv_d, float eps, int stages, unsigned int *status)
{
    constexpr int VEC = 16 / (int)sizeof(T), NV = E / VEC, NP = Pairs<T>::N;
    extern __shared__ __align__(128) unsigned char rows[];
    __shared__ float part[2][32];
    __shared__ __align__(8) unsigned long long full[kNormMaxStages];
    const int step = blockDim.x;
    const uint32_t row_bytes = (uint32_t)d * sizeof(T);
    RowRing ring = {smem_addr(rows), smem_addr(full), row_bytes, stages, true, status};
    if (threadIdx.x < stages) barrier_init(ring.bar(threadIdx.x), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    grid_dependency_wait();
    grid_dependency_launch_next();
    auto load = [&](int i) {
        const long long row = blockIdx.x + (long long)i * gridDim.x;
        if (row >= n) return;
        barrier_expect(ring.bar(i), row_bytes);
        bulk_copy(ring.at(i), x + row * xs, row_bytes, ring.bar(i));
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < stages; ++i) load(i);
    float2 wv[NV][NP], bv[NV][NP];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (threadIdx.x + i * step) * VEC;
        load_pairs<P, NP>(w, c, c < d, 1.0f, wv[i]);
        load_pairs<P, NP>(b, c, c < d, 0.0f, bv[i]);
    }
    int it = 0;
    for (int row = blockIdx.x; row < n; row += gridDim.x, ++it) {
        ring.wait(it);
        const T *src = shared_row<T>(ring.at(it));
        Pairs<T> in[NV];
        float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (threadIdx.x + i * step) * VEC;
            if (c < d) {
                in[i].load(src + c);
#pragma unroll
                for (int k = 0; k < NP; ++k) sum = add2(sum, in[i].get(k));
            }
        }
        const float mu = row_sum<false>(sum.x + sum.y, part[0]) * inv_d;
        if (threadIdx.x == 0) load(it + stages);  // every thread has read the stage
        // the squares are scaled term by term: their sum may leave the range where their mean does not
        const float2 rr = make_float2(root_inv_d, root_inv_d), m2 = make_float2(-mu, -mu);
        float2 sq = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (threadIdx.x + i * step) * VEC;
            if (c < d) {
#pragma unroll
                for (int k = 0; k < NP; ++k) {
                    const float2 e = mul2(add2(in[i].get(k), m2), rr);
                    sq = fma2(e, e, sq);
                }
            }
        }
        const float r = rsqrtf(row_sum<false>(sq.x + sq.y, part[1]) + eps);
        if (threadIdx.x == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
        const float2 r2 = make_float2(r, r);
        T *dst = y + row * ys;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (threadIdx.x + i * step) * VEC;
            if (c < d) {
                Pairs<T> out;
#pragma unroll
                for (int k = 0; k < NP; ++k)
                    out.set(k, fma2(mul2(add2(in[i].get(k), m2), r2), wv[i][k], bv[i][k]));
                out.store(dst + c);
            }
        }
    }
    if (!ring.arrived && threadIdx.x == 0) {
        const long long mine = (n - (long long)blockIdx.x + gridDim.x - 1) / gridDim.x;
        ring.drain(it - 1, (int)min(mine, (long long)it + stages));
    }
}

// Rows in registers: a warp per row (aligned rows of at most 32 * kNormVecs packs, others of at most 32 * kNormScalars
// values), or, where rows are not aligned and longer, a CTA per row.
template <typename T, typename P, int VEC, int NV, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kNormWarps : kNormMaxThreads)
k_norm_forward(const T *__restrict__ x, long long xs, const P *__restrict__ w, const P *__restrict__ b,
               T *__restrict__ y, long long ys, float *__restrict__ mean, float *__restrict__ rstd, long long n,
               int d, float inv_d, float root_inv_d, float eps)
{
    __shared__ float part[2][32];
    const int tid = WARP ? (threadIdx.x & 31) : threadIdx.x;
    const int step = WARP ? 32 : blockDim.x;
    const long long row = WARP ? (long long)blockIdx.x * kNormWarps + (threadIdx.x >> 5) : (long long)blockIdx.x;
    grid_dependency_wait();
    grid_dependency_launch_next();
    if (row >= n) return;
    const T *xr = x + row * xs;
    Pack<T, VEC> in[NV];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (tid + i * step) * VEC;
        if (c < d) in[i] = load_pack<T, VEC>(xr + c);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (tid + i * step) * VEC;
        if (c < d) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) sum += to_f32(in[i].v[j]);
        }
    }
    const float mu = row_sum<WARP>(sum, part[0]) * inv_d;
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (tid + i * step) * VEC;
        if (c < d) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float e = (to_f32(in[i].v[j]) - mu) * root_inv_d;
                sq = fmaf(e, e, sq);
            }
        }
    }
    const float r = rsqrtf(row_sum<WARP>(sq, part[1]) + eps);
    if (tid == 0) {
        if (mean) mean[row] = mu;
        if (rstd) rstd[row] = r;
    }
    T *yr = y + row * ys;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (tid + i * step) * VEC;
        if (c < d) {
            float wv[VEC], bv[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) wv[j] = 1.0f, bv[j] = 0.0f;
            if (w) load_param<P, VEC>(w, c, wv);
            if (b) load_param<P, VEC>(b, c, bv);
            Pack<T, VEC> out;
#pragma unroll
            for (int j = 0; j < VEC; ++j) out.v[j] = from_f32<T>(fmaf((to_f32(in[i].v[j]) - mu) * r, wv[j], bv[j]));
            *reinterpret_cast<Pack<T, VEC> *>(yr + c) = out;
        }
    }
}

// Rows longer than a CTA's registers hold: the row is read three times, the last two out of L2.
template <typename T, typename P>
__global__ void __launch_bounds__(kNormMaxThreads)
k_norm_forward_long(const T *__restrict__ x, long long xs, const P *__restrict__ w, const P *__restrict__ b,
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
// Sums of dw and db: every thread keeps those of its columns over all rows its CTA takes, and writes them to
// `partial` ([2][CTAs][d]) at the end; k_norm_param_gradient adds them up in a fixed order.  No atomics: the same
// bits from run to run.
constexpr int kBackElems = 16;  // columns of a thread

// Aligned rows: ROWS rows of x and dy per stage of the ring.  One barrier per stage: it ends the sums of this stage
// and, with it, all reads of the one before, which is refilled behind it.
template <typename T, int E, int ROWS, typename P>
__global__ void __launch_bounds__(kNormBackThreads)
k_norm_backward_ring(const T *__restrict__ dy, long long dys, const T *__restrict__ x, long long xs,
                     const P *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd,
                     T *__restrict__ dx, long long dxs, float *__restrict__ partial, int n, int d, float inv_d, int stages,
                     unsigned int *status)
{
    constexpr int VEC = 16 / (int)sizeof(T), NV = E / VEC, NP = Pairs<T>::N;
    constexpr bool KEEP = E <= 16;  // weight, x and dy stay in registers between the two passes over a row
    extern __shared__ __align__(128) unsigned char rows[];
    __shared__ float2 part[2][ROWS][32];
    __shared__ __align__(8) unsigned long long full[kNormMaxStages];
    const int step = blockDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t row_bytes = (uint32_t)d * sizeof(T);
    const int groups = (n + ROWS - 1) / ROWS;
    RowRing ring = {smem_addr(rows), smem_addr(full), ROWS * 2 * row_bytes, stages, true, status};
    if (threadIdx.x < stages) barrier_init(ring.bar(threadIdx.x), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    grid_dependency_wait();
    grid_dependency_launch_next();
    auto load = [&](int i) {  // by one thread
        const long long g = blockIdx.x + (long long)i * gridDim.x;
        if (g >= groups) return;
        const int count = min(ROWS, n - (int)g * ROWS);
        barrier_expect(ring.bar(i), 2 * count * row_bytes);
        for (int r = 0; r < count; ++r) {
            bulk_copy(ring.at(i) + 2 * r * row_bytes, x + (g * ROWS + r) * xs, row_bytes, ring.bar(i));
            bulk_copy(ring.at(i) + (2 * r + 1) * row_bytes, dy + (g * ROWS + r) * dys, row_bytes, ring.bar(i));
        }
    };
    if (threadIdx.x == 0)
        for (int i = 0; i + 1 < stages; ++i) load(i);

    float2 dw[NV][NP], db[NV][NP], wv[KEEP ? NV : 1][NP];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (threadIdx.x + i * step) * VEC;
        if constexpr (KEEP) load_pairs<P, NP>(w, c, c < d, 1.0f, wv[i]);
#pragma unroll
        for (int k = 0; k < NP; ++k) dw[i][k] = db[i][k] = make_float2(0.0f, 0.0f);
    }
    float nmu[ROWS], nr[ROWS];  // the next stage's statistics
    auto statistics = [&](long long g) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const long long row = g * ROWS + r;
            nmu[r] = row < n ? mean[row] : 0.0f;
            nr[r] = row < n ? rstd[row] : 0.0f;
        }
    };
    statistics(blockIdx.x);
    int it = 0;
    for (int g = blockIdx.x; g < groups; g += gridDim.x, ++it) {
        const int turn = it & 1;
        float mu[ROWS], rs[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) mu[r] = nmu[r], rs[r] = nr[r];
        statistics((long long)g + gridDim.x);
        ring.wait(it);
        Pairs<T> px[KEEP ? ROWS : 1][KEEP ? NV : 1], pg[KEEP ? ROWS : 1][KEEP ? NV : 1];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const T *sx = shared_row<T>(ring.at(it) + 2 * r * row_bytes), *sg = shared_row<T>(ring.at(it) + (2 * r + 1) * row_bytes);
            const float2 m2 = make_float2(-mu[r], -mu[r]), r2 = make_float2(rs[r], rs[r]);
            float2 s1 = make_float2(0.0f, 0.0f), s2 = s1;
            if (g * ROWS + r < n) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = (threadIdx.x + i * step) * VEC;
                    if (c < d) {
                        Pairs<T> vx, vg;
                        vx.load(sx + c);
                        vg.load(sg + c);
                        if constexpr (KEEP) px[r][i] = vx, pg[r][i] = vg;
                        float2 wl[NP];
                        if constexpr (!KEEP) load_pairs<P, NP>(w, c, true, 1.0f, wl);
#pragma unroll
                        for (int k = 0; k < NP; ++k) {
                            const float2 gv = vg.get(k), xhat = mul2(add2(vx.get(k), m2), r2);
                            const float2 gw = mul2(gv, KEEP ? wv[KEEP ? i : 0][k] : wl[k]);
                            s1 = add2(s1, gw);
                            s2 = fma2(gw, xhat, s2);
                            dw[i][k] = fma2(gv, xhat, dw[i][k]);
                            db[i][k] = add2(db[i][k], gv);
                        }
                    }
                }
            }
            const float a = warp_sum(s1.x + s1.y), b = warp_sum(s2.x + s2.y);
            if (lane == 0) part[turn][r][warp] = make_float2(a, b);
        }
        __syncthreads();
        if (threadIdx.x == 0) load(it + stages - 1);
        if (!dx) continue;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int row = g * ROWS + r;
            if (row >= n) break;
            const float2 t = lane < (step >> 5) ? part[turn][r][lane] : make_float2(0.0f, 0.0f);
            // dx = rstd g w - rstd mean(g w) - xhat rstd mean(g w xhat)
            const float c1 = -rs[r] * (warp_sum(t.x) * inv_d), c2 = -rs[r] * (warp_sum(t.y) * inv_d);
            const float2 m2 = make_float2(-mu[r], -mu[r]), r2 = make_float2(rs[r], rs[r]), f1 = make_float2(c1, c1),
                         f2 = make_float2(c2, c2);
            const T *sx = shared_row<T>(ring.at(it) + 2 * r * row_bytes), *sg = shared_row<T>(ring.at(it) + (2 * r + 1) * row_bytes);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (threadIdx.x + i * step) * VEC;
                if (c < d) {
                    Pairs<T> vx, vg, out;
                    if constexpr (KEEP) {
                        vx = px[r][i], vg = pg[r][i];
                    } else {
                        vx.load(sx + c);
                        vg.load(sg + c);
                    }
                    float2 wl[NP];
                    if constexpr (!KEEP) load_pairs<P, NP>(w, c, true, 1.0f, wl);
#pragma unroll
                    for (int k = 0; k < NP; ++k) {
                        const float2 xhat = mul2(add2(vx.get(k), m2), r2);
                        const float2 gw = mul2(vg.get(k), KEEP ? wv[KEEP ? i : 0][k] : wl[k]);
                        out.set(k, fma2(xhat, f2, fma2(gw, r2, f1)));
                    }
                    out.store(dx + (long long)row * dxs + c);
                }
            }
        }
    }
    if (!ring.arrived && threadIdx.x == 0) {
        const long long mine = ((long long)groups - blockIdx.x + gridDim.x - 1) / gridDim.x;
        ring.drain(it - 1, (int)min(mine, (long long)it + stages - 1));
    }
    if (!partial) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (threadIdx.x + i * step) * VEC;
        if (c < d) {
            float *a = partial + (long long)blockIdx.x * d + c, *b = a + (long long)gridDim.x * d;
#pragma unroll
            for (int k = 0; k < NP; k += 2) {
                *reinterpret_cast<float4 *>(a + 2 * k) = make_float4(dw[i][k].x, dw[i][k].y, dw[i][k + 1].x, dw[i][k + 1].y);
                *reinterpret_cast<float4 *>(b + 2 * k) = make_float4(db[i][k].x, db[i][k].y, db[i][k + 1].x, db[i][k + 1].y);
            }
        }
    }
}

// Rows in registers: a warp per row (rows of at most 32 * kBackElems columns), or, where rows are not 16-byte aligned
// and longer, a CTA per row.  The next row is loaded while this one is reduced.
template <typename T, typename P, int VEC, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kBackWarps : kNormBackThreads)
k_norm_backward(const T *__restrict__ dy, long long dys, const T *__restrict__ x, long long xs,
                const P *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd,
                T *__restrict__ dx, long long dxs, float *__restrict__ partial, long long n, int d, float inv_d)
{
    constexpr int NV = kBackElems / VEC;
    __shared__ float2 part[2][32];
    __shared__ float joined[WARP ? kBackWarps : 1][WARP ? 32 * kBackElems : 1];
    const int tid = WARP ? (threadIdx.x & 31) : threadIdx.x;
    const int step = WARP ? 32 : blockDim.x;
    const long long first = WARP ? (long long)blockIdx.x * kBackWarps + (threadIdx.x >> 5) : (long long)blockIdx.x;
    const long long stride = WARP ? (long long)gridDim.x * kBackWarps : (long long)gridDim.x;
    grid_dependency_wait();
    grid_dependency_launch_next();
    float dw[NV][VEC] = {}, db[NV][VEC] = {};
    Pack<T, VEC> nx[NV], ng[NV];
    float nmu = 0.0f, nr = 0.0f;
    auto fetch = [&](long long row) {
        if (row >= n) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (tid + i * step) * VEC;
            if (c < d) {
                nx[i] = load_pack<T, VEC>(x + row * xs + c);
                ng[i] = load_pack<T, VEC>(dy + row * dys + c);
            }
        }
        nmu = mean[row];
        nr = rstd[row];
    };
    fetch(first);
    int turn = 0;
    for (long long row = first; row < n; row += stride, turn ^= 1) {
        Pack<T, VEC> cx[NV], cg[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) cx[i] = nx[i], cg[i] = ng[i];
        const float mu = nmu, r = nr;
        fetch(row + stride);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (tid + i * step) * VEC;
            if (c < d) {
                float wv[VEC];
                if (w) load_param<P, VEC>(w, c, wv);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float g = to_f32(cg[i].v[j]), xhat = (to_f32(cx[i].v[j]) - mu) * r;
                    const float gw = w ? g * wv[j] : g;
                    s1 += gw;
                    s2 = fmaf(gw, xhat, s2);
                    dw[i][j] = fmaf(g, xhat, dw[i][j]);
                    db[i][j] += g;
                }
            }
        }
        const float2 s = row_sum2<WARP>(s1, s2, part[turn]);
        const float m1 = s.x * inv_d, m2 = s.y * inv_d;
        if (dx) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (tid + i * step) * VEC;
                if (c < d) {
                    float wv[VEC];
                    if (w) load_param<P, VEC>(w, c, wv);
                    Pack<T, VEC> out;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float g = to_f32(cg[i].v[j]), xhat = (to_f32(cx[i].v[j]) - mu) * r;
                        const float gw = w ? g * wv[j] : g;
                        out.v[j] = from_f32<T>(r * (gw - m1 - xhat * m2));
                    }
                    *reinterpret_cast<Pack<T, VEC> *>(dx + row * dxs + c) = out;
                }
            }
        }
    }
    if (!partial) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float *dst = partial + ((long long)which * gridDim.x + blockIdx.x) * d;
        if constexpr (WARP) {  // the CTA's warps first, in order
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    joined[threadIdx.x >> 5][(tid + i * 32) * VEC + j] = which ? db[i][j] : dw[i][j];
            __syncthreads();
            for (int c = threadIdx.x; c < d; c += 32 * kBackWarps) {
                float t = joined[0][c];
#pragma unroll
                for (int k = 1; k < kBackWarps; ++k) t += joined[k][c];
                dst[c] = t;
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (tid + i * step) * VEC;
                if (c < d) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) dst[c + j] = which ? db[i][j] : dw[i][j];
                }
            }
        }
    }
}

// Rows longer than a CTA's registers hold: two reads of the row; a second kernel walks the columns.
template <typename T, typename P>
__global__ void __launch_bounds__(kNormMaxThreads)
k_norm_backward_long(const T *__restrict__ dy, long long dys, const T *__restrict__ x, long long xs,
                     const P *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd,
                     T *__restrict__ dx, long long dxs, int d, float inv_d)
{
    __shared__ float2 part[32];
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
    const float2 s = row_sum2<false>(s1, s2, part);
    const float m1 = s.x * inv_d, m2 = s.y * inv_d;
    for (int c = threadIdx.x; c < d; c += blockDim.x) {
        const float gw = to_f32(dy[row * dys + c]) * (w ? to_f32(w[c]) : 1.0f);
        dx[row * dxs + c] = from_f32<T>(r * (gw - m1 - (to_f32(x[row * xs + c]) - mu) * r * m2));
    }
}

// Column sums of long rows: a thread per column, a range of rows per CTA row.
template <typename T>
__global__ void __launch_bounds__(256)
k_norm_columns_long(const T *__restrict__ dy, long long dys, const T *__restrict__ x, long long xs,
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

// dw[c] = sum over the slots of partial[0][slot][c], db likewise: 32 columns x 8 slot lanes per CTA.
template <typename Q>
__global__ void __launch_bounds__(256)
k_norm_param_gradient(const float *__restrict__ partial, int slots, int d, Q *__restrict__ dw, Q *__restrict__ db)
{
    __shared__ float sum[8][33];
    const int lane = threadIdx.x & 31, k = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    Q *out = blockIdx.y ? db : dw;
    grid_dependency_wait();
    grid_dependency_launch_next();
    if (!out) return;
    const float *src = partial + (long long)blockIdx.y * slots * d + c;
    float a[4] = {};
    if (c < d) {
        int i = k;
        for (; i + 24 < slots; i += 32) {
#pragma unroll
            for (int u = 0; u < 4; ++u) a[u] += src[(long long)(i + 8 * u) * d];
        }
        for (; i < slots; i += 8) a[0] += src[(long long)i * d];
    }
    sum[k][lane] = (a[0] + a[1]) + (a[2] + a[3]);
    __syncthreads();
    if (k == 0 && c < d) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t += sum[i][lane];
        out[c] = from_f32<Q>(t);
    }
}

namespace {

// 16-byte accesses where every row of every operand starts on such a boundary and the width is a whole number of
// packs.
struct NormShape {
    bool vec;
    int units, threads;   // packs (or elements) of a row; threads of a CTA that takes one row
};
NormShape norm_shape(int d, int elem, bool aligned, int per_vec, int per_scalar)
{
    NormShape s{};
    const int vec = 16 / elem;
    s.vec = aligned && d % vec == 0;
    s.units = s.vec ? d / vec : d;
    const int per = s.vec ? per_vec : per_scalar;
    s.threads = ((s.units + per - 1) / per + 31) / 32 * 32;
    return s;
}

bool rows_aligned(const void *p, long long stride, int elem) { return pointer_aligned(p, 16) && (stride * elem) % 16 == 0; }

// CTAs whose sums of dw and db are added up at the end: what they write and what is read again stays under a tenth of
// the rows' own traffic (16 bytes per slot and column against 6 per row and column), unless rows are few.
int norm_slots(long long n) { return (int)(n / 27 > 2 * current_device_sms() ? n / 27 : 2 * current_device_sms()); }
int norm_slots_max() { return 6 * current_device_sms(); }

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
// stages each.
struct RingShape {
    int ctas, stages;
};
RingShape ring_shape(int threads, int registers, int stage, int least)
{
    RingShape r{65536 / (registers * threads), 0};
    if (r.ctas > 2048 / threads) r.ctas = 2048 / threads;
    if (r.ctas > 16) r.ctas = 16;
    while (r.ctas > 1 && kNormRingBytes / r.ctas < 3 * stage) --r.ctas;
    if (r.ctas < 1) r.ctas = 1;
    r.stages = kNormRingBytes / r.ctas / stage;
    if (r.stages > kNormMaxStages) r.stages = kNormMaxStages;
    if (r.stages < least) r.stages = 0;
    return r;
}

template <typename T, typename P, int E>
cudaError_t forward_ring(RingShape ring, int threads, const T *xp, long long xs, const P *wp, const P *bp, T *yp, long long ys,
                         float *mean, float *rstd, long long n, int d, float eps, cudaStream_t s)
{
    static std::atomic<uint64_t> ready{0};
    unsigned int *status = nullptr;
    cudaError_t e = operator_status_ptr(&status);
    if (e == cudaSuccess) e = allow_ring(k_norm_forward_ring<T, P, E>, ready);
    if (e != cudaSuccess) return e;
    const long long most = (long long)ring.ctas * current_device_sms();
    return launch_chained(k_norm_forward_ring<T, P, E>, (unsigned)(n < most ? n : most), threads,
                          (size_t)ring.stages * d * sizeof(T), s, 1, xp, xs, wp, bp, yp, ys, mean, rstd, (int)n, d,
                          1.0f / (float)d, 1.0f / sqrtf((float)d), eps, ring.stages, status);
}

template <typename T, typename P>
cudaError_t norm_forward(const void *x, long long xs, const void *w, const void *b, void *y, long long ys, float *mean,
                         float *rstd, long long n, int d, float eps, cudaStream_t s)
{
    constexpr int V = 16 / (int)sizeof(T), E = (int)sizeof(T);
    const NormShape sh = norm_shape(d, E, rows_aligned(x, xs, E) && rows_aligned(y, ys, E) && pointer_aligned(w, 16) &&
                                              pointer_aligned(b, 16), 16 / V, kNormScalars);
    const float inv = 1.0f / (float)d, root = 1.0f / sqrtf((float)d);
    const T *xp = (const T *)x;
    const P *wp = (const P *)w, *bp = (const P *)b;
    T *yp = (T *)y;
    const unsigned rows = (unsigned)n, groups = (unsigned)((n + kNormWarps - 1) / kNormWarps);
    if (sh.vec && sh.units <= 32 * kNormVecs)
        return launch_chained(k_norm_forward<T, P, V, kNormVecs, true>, groups, 32 * kNormWarps, 0, s, 1, xp, xs, wp,
                              bp, yp, ys, mean, rstd, n, d, inv, root, eps);
    if (sh.vec) {
        const int wide = (sh.threads / 2 + 31) / 32 * 32;  // threads that hold twice as many columns
        if (sh.threads <= kNormRingThreads) {
            const RingShape ring = ring_shape(sh.threads, 64, d * E, 2);
            if (ring.stages)
                return forward_ring<T, P, 16>(ring, sh.threads, xp, xs, wp, bp, yp, ys, mean, rstd, n, d, eps, s);
        } else if (wide <= kNormRingThreads) {
            const RingShape ring = ring_shape(wide, 128, d * E, 2);
            if (ring.stages) return forward_ring<T, P, 32>(ring, wide, xp, xs, wp, bp, yp, ys, mean, rstd, n, d, eps, s);
        }
    }
    if (!sh.vec && sh.units <= 32 * kNormScalars)
        return launch_chained(k_norm_forward<T, P, 1, kNormScalars, true>, groups, 32 * kNormWarps, 0, s, 1, xp, xs,
                              wp, bp, yp, ys, mean, rstd, n, d, inv, root, eps);
    if (!sh.vec && sh.threads <= kNormMaxThreads)
        return launch_chained(k_norm_forward<T, P, 1, kNormScalars, false>, rows, sh.threads, 0, s, 1, xp, xs, wp, bp, yp,
                              ys, mean, rstd, n, d, inv, root, eps);
    return launch_chained(k_norm_forward_long<T, P>, rows, kNormMaxThreads, 0, s, 1, xp, xs, wp, bp, yp, ys, mean, rstd, d,
                          inv, root, eps);
}

// Launches the ring kernel with `rows` rows per stage if its shared memory holds two stages at least.
template <typename T, int E, int ROWS, typename P>
bool launch_ring(cudaError_t *e, int *slots, int threads, const T *gp, long long dys, const T *xp, long long xs, const P *wp,
                 const float *mean, const float *rstd, T *dxp, long long dxs, float *part, long long n, int d, float inv,
                 cudaStream_t s)
{
    const int stage = ROWS * 2 * d * (int)sizeof(T);
    const RingShape ring = ring_shape(threads, 128, stage, ROWS > 1 ? 3 : 2);
    if (!ring.stages) return false;
    static std::atomic<uint64_t> ready{0};
    unsigned int *status = nullptr;
    *e = operator_status_ptr(&status);
    if (*e == cudaSuccess) *e = allow_ring(k_norm_backward_ring<T, E, ROWS, P>, ready);
    if (*e != cudaSuccess) return true;
    long long grid = (n + ROWS - 1) / ROWS, most = (long long)ring.ctas * current_device_sms();
    if (most > norm_slots(n)) most = norm_slots(n);
    if (most > norm_slots_max()) most = norm_slots_max();
    if (grid > most) grid = most;
    *slots = (int)grid;
    *e = launch_chained(k_norm_backward_ring<T, E, ROWS, P>, (unsigned)grid, threads, (size_t)ring.stages * stage, s, 1, gp, dys, xp,
                        xs, wp, mean, rstd, dxp, dxs, part, (int)n, d, inv, ring.stages, status);
    return true;
}

template <typename T, typename P>
cudaError_t norm_backward(const void *dy, long long dys, const void *x, long long xs, const void *w, const float *mean,
                          const float *rstd, void *dx, long long dxs, void *dw, void *db, int grad_type, long long n,
                          int d, float *partial, cudaStream_t s)
{
    constexpr int V = 16 / (int)sizeof(T), E = (int)sizeof(T);
    const NormShape sh = norm_shape(d, E, rows_aligned(x, xs, E) && rows_aligned(dy, dys, E) &&
                                              (!dx || rows_aligned(dx, dxs, E)) && pointer_aligned(w, 16),
                                    kBackElems / V, kBackElems);
    const float inv = 1.0f / (float)d;
    const T *xp = (const T *)x, *gp = (const T *)dy;
    const P *wp = (const P *)w;
    T *dxp = (T *)dx;
    float *part = dw || db ? partial : nullptr;
    int slots = 0;
    cudaError_t e = cudaSuccess;
    const int wide = (sh.threads / 2 + 31) / 32 * 32;  // threads that hold twice as many columns
    if (d <= 32 * kBackElems) {
        const long long groups = (n + kBackWarps - 1) / kBackWarps, most = 3ll * current_device_sms();
        long long g = groups < most ? groups : most;
        if (g > norm_slots(n)) g = norm_slots(n);
        slots = (int)g;
        e = sh.vec ? launch_chained(k_norm_backward<T, P, V, true>, (unsigned)g, 32 * kBackWarps, 0, s, 1, gp, dys, xp, xs, wp,
                                    mean, rstd, dxp, dxs, part, n, d, inv)
                   : launch_chained(k_norm_backward<T, P, 1, true>, (unsigned)g, 32 * kBackWarps, 0, s, 1, gp, dys, xp, xs, wp,
                                    mean, rstd, dxp, dxs, part, n, d, inv);
    } else if (sh.vec && sh.threads <= kNormBackThreads &&
               launch_ring<T, 16, 2, P>(&e, &slots, sh.threads, gp, dys, xp, xs, wp, mean, rstd, dxp, dxs, part, n, d, inv, s)) {
    } else if (sh.vec && sh.threads <= kNormBackThreads &&
               launch_ring<T, 16, 1, P>(&e, &slots, sh.threads, gp, dys, xp, xs, wp, mean, rstd, dxp, dxs, part, n, d, inv, s)) {
    } else if (sh.vec && wide <= kNormBackThreads &&
               launch_ring<T, 32, 1, P>(&e, &slots, wide, gp, dys, xp, xs, wp, mean, rstd, dxp, dxs, part, n, d, inv, s)) {
    } else if (!sh.vec && sh.threads <= kNormBackThreads) {
        long long most = (long long)(65536 / (128 * sh.threads)) * current_device_sms();
        if (most > norm_slots(n)) most = norm_slots(n);
        if (most > norm_slots_max()) most = norm_slots_max();
        slots = (int)(n < most ? n : most);
        e = launch_chained(k_norm_backward<T, P, 1, false>, (unsigned)slots, sh.threads, 0, s, 1, gp, dys, xp, xs, wp, mean,
                           rstd, dxp, dxs, part, n, d, inv);
    } else {
        if (dx)
            e = launch_chained(k_norm_backward_long<T, P>, (unsigned)n, kNormMaxThreads, 0, s, 1, gp, dys, xp, xs, wp,
                               mean, rstd, dxp, dxs, d, inv);
        if (e == cudaSuccess && part) {
            slots = (int)(n < 64 ? n : 64);
            e = launch_chained(k_norm_columns_long<T>, dim3((unsigned)((d + 255) / 256), (unsigned)slots), 256, 0, s, 1,
                               gp, dys, xp, xs, mean, rstd, part, n, d);
        }
    }
    if (e != cudaSuccess || !part) return e;
    const dim3 grid((unsigned)((d + 31) / 32), 2);
    if (grad_type == RSDGC_F32)
        return launch_chained(k_norm_param_gradient<float>, grid, 256, 0, s, 1, part, slots, d, (float *)dw, (float *)db);
    if (grad_type == RSDGC_BF16)
        return launch_chained(k_norm_param_gradient<__nv_bfloat16>, grid, 256, 0, s, 1, part, slots, d,
                              (__nv_bfloat16 *)dw, (__nv_bfloat16 *)db);
    return launch_chained(k_norm_param_gradient<__half>, grid, 256, 0, s, 1, part, slots, d, (__half *)dw, (__half *)db);
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
    if (n > INT_MAX || d > (1 << 24)) return RSDGC_ERR_CAPACITY;
    return RSDGC_OK;
}

}  // namespace
}  // namespace rsdgc

using namespace rsdgc;

extern "C" int64_t rsdgc_layer_norm_workspace_bytes(int64_t n_rows, int64_t width)
{
    if (n_rows < 0 || width < 1) return RSDGC_ERR_INVALID;
    const int64_t slots = norm_slots_max();
    return 2 * 4 * slots * width;
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
    const cudaError_t e = with_types(dtype, param_dtype, [&](auto t, auto p) {
        return norm_forward<decltype(t), decltype(p)>(x_dev, x_stride, weight_dev, bias_dev, y_dev, y_stride, mean_dev,
                                                      rstd_dev, n_rows, (int)width, eps, (cudaStream_t)stream);
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
    const cudaError_t e = with_types(dtype, param_dtype, [&](auto t, auto p) {
        return norm_backward<decltype(t), decltype(p)>(dy_dev, dy_stride, x_dev, x_stride, weight_dev, mean_dev, rstd_dev,
                                                       dx_dev, dx_stride, dweight_dev, dbias_dev, grad_dtype, n_rows,
                                                       (int)width, (float *)workspace_dev, s);
    });
    return operator_result(e);
}
