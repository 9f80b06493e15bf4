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

constexpr int kNormVecs = 4;          // 16-byte vectors of a row that a thread holds
constexpr int kNormVecsWarp = 16;     // ... where rows are many and a warp takes one
constexpr int kNormScalars = 16;      // elements it holds where rows are not 16-byte aligned
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

// ---- forward ----------------------------------------------------------------------------------
// WARP: a warp per row (rows of at most 32 * NV packs), kNormWarps rows per CTA; else a CTA per row.
template <typename T, typename P, int VEC, int NV, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kNormWarps : kNormMaxThreads)
k_norm_forward(const T *__restrict__ x, long long xs, const P *__restrict__ w, const P *__restrict__ b,
               T *__restrict__ y, long long ys, float *__restrict__ mean, float *__restrict__ rstd, long long n,
               int d, float inv_d, float eps)
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
                const float e = to_f32(in[i].v[j]) - mu;
                sq = fmaf(e * inv_d, e, sq);  // the mean, term by term: the sum itself may leave the range
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
            if (w) load_param<P, VEC>(w, c, wv);
            if (b) load_param<P, VEC>(b, c, bv);
            Pack<T, VEC> out;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float xhat = (to_f32(in[i].v[j]) - mu) * r;
                out.v[j] = from_f32<T>(fmaf(xhat, w ? wv[j] : 1.0f, b ? bv[j] : 0.0f));
            }
            *reinterpret_cast<Pack<T, VEC> *>(yr + c) = out;
        }
    }
}

// Rows longer than a CTA's registers hold: the row is read three times, the last two out of L2.
template <typename T, typename P>
__global__ void __launch_bounds__(kNormMaxThreads)
k_norm_forward_long(const T *__restrict__ x, long long xs, const P *__restrict__ w, const P *__restrict__ b,
                    T *__restrict__ y, long long ys, float *__restrict__ mean, float *__restrict__ rstd,
                    int d, float inv_d, float eps)
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
        const float e = to_f32(xr[c]) - mu;
        sq = fmaf(e * inv_d, e, sq);  // the mean, term by term: the sum itself may leave the range
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

// Rows in shared memory: a ring of stages, each ROWS rows of x and dy, filled by bulk copies that run kStages - 1
// stages ahead, so that a CTA has tens of KB on their way whatever its threads wait for.  One barrier per stage: it
// ends the sums of this stage and, with it, all reads of the one before, which is refilled behind it.
template <typename T, int E, int ROWS, typename P>
__global__ void __launch_bounds__(kNormBackThreads)
k_norm_backward_ring(const T *__restrict__ dy, long long dys, const T *__restrict__ x, long long xs,
                     const P *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd,
                     T *__restrict__ dx, long long dxs, float *__restrict__ partial, int n, int d, float inv_d, int stages,
                     unsigned int *status)
{
    constexpr int VEC = 16 / (int)sizeof(T), NV = E / VEC;
    constexpr bool KEEP = E <= 16;  // x and dy stay in registers between the two passes over a row
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ float2 part[2][ROWS][32];
    __shared__ __align__(8) unsigned long long full[kNormMaxStages];
    const int step = blockDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t row_bytes = (uint32_t)d * sizeof(T), stage_bytes = ROWS * 2 * row_bytes;
    const int groups = (n + ROWS - 1) / ROWS;
    if (threadIdx.x < stages) barrier_init(smem_addr(&full[threadIdx.x]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    grid_dependency_wait();
    grid_dependency_launch_next();

    auto load = [&](int i) {  // stage i of this CTA, by one thread
        const int g = blockIdx.x + i * (int)gridDim.x;
        if (g >= groups) return;
        const int s = i % stages, rows = min(ROWS, n - g * ROWS);
        const uint32_t bar = smem_addr(&full[s]), dst = smem_addr(ring) + s * stage_bytes;
        barrier_expect(bar, 2 * rows * row_bytes);
        for (int r = 0; r < rows; ++r) {
            bulk_copy(dst + 2 * r * row_bytes, x + (long long)(g * ROWS + r) * xs, row_bytes, bar);
            bulk_copy(dst + (2 * r + 1) * row_bytes, dy + (long long)(g * ROWS + r) * dys, row_bytes, bar);
        }
    };
    if (threadIdx.x == 0)
        for (int i = 0; i + 1 < stages; ++i) load(i);

    float dw[NV][VEC] = {}, db[NV][VEC] = {}, wv[KEEP ? NV : 1][VEC];
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (threadIdx.x + i * step) * VEC;
#pragma unroll
            for (int j = 0; j < VEC; ++j) wv[i][j] = 1.0f;
            if (w && c < d) load_param<P, VEC>(w, c, wv[i]);
        }
    }
    float nmu[ROWS], nr[ROWS];  // the next stage's statistics
    auto statistics = [&](int g) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int row = g * ROWS + r;
            nmu[r] = row < n ? mean[row] : 0.0f;
            nr[r] = row < n ? rstd[row] : 0.0f;
        }
    };
    statistics(blockIdx.x);
    bool arrived = true;
    int it = 0;
    for (int g = blockIdx.x; g < groups; g += gridDim.x, ++it) {
        const int s = it % stages, turn = it & 1;
        const unsigned char *stage = ring + s * stage_bytes;
        float mu[ROWS], rs[ROWS], s1[ROWS], s2[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) mu[r] = nmu[r], rs[r] = nr[r], s1[r] = s2[r] = 0.0f;
        statistics(g + gridDim.x);
        // bounded; once a wait has given up the results are void (the status says so) and the others poll once
        unsigned left = arrived ? kNormSpin : 1u;
        bool here = false;
        while (left-- && !(here = barrier_try(smem_addr(&full[s]), (uint32_t)(it / stages) & 1u))) {}
        if (!here && arrived) {
            arrived = false;
            atomicOr(status, RSDGC_STATUS_TIMEOUT);
        }
        Pack<T, VEC> px[KEEP ? ROWS : 1][KEEP ? NV : 1], pg[KEEP ? ROWS : 1][KEEP ? NV : 1];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const T *sx = reinterpret_cast<const T *>(stage + 2 * r * row_bytes);
            const T *sg = reinterpret_cast<const T *>(stage + (2 * r + 1) * row_bytes);
            if (g * ROWS + r < n) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = (threadIdx.x + i * step) * VEC;
                    if (c < d) {
                        const Pack<T, VEC> vx = load_pack<T, VEC>(sx + c), vg = load_pack<T, VEC>(sg + c);
                        if constexpr (KEEP) px[r][i] = vx, pg[r][i] = vg;
                        float wl[VEC];
                        if constexpr (!KEEP)
                            if (w) load_param<P, VEC>(w, c, wl);
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            const float gv = to_f32(vg.v[j]), xhat = (to_f32(vx.v[j]) - mu[r]) * rs[r];
                            const float gw = KEEP ? gv * wv[KEEP ? i : 0][j] : w ? gv * wl[j] : gv;
                            s1[r] += gw;
                            s2[r] = fmaf(gw, xhat, s2[r]);
                            dw[i][j] = fmaf(gv, xhat, dw[i][j]);
                            db[i][j] += gv;
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            s1[r] = warp_sum(s1[r]);
            s2[r] = warp_sum(s2[r]);
            if (lane == 0) part[turn][r][warp] = make_float2(s1[r], s2[r]);
        }
        __syncthreads();
        if (threadIdx.x == 0) load(it + stages - 1);
        if (!dx) continue;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int row = g * ROWS + r;
            if (row >= n) break;
            const float2 t = lane < (step >> 5) ? part[turn][r][lane] : make_float2(0.0f, 0.0f);
            const float m1 = warp_sum(t.x) * inv_d, m2 = warp_sum(t.y) * inv_d;
            const T *sx = reinterpret_cast<const T *>(stage + 2 * r * row_bytes);
            const T *sg = reinterpret_cast<const T *>(stage + (2 * r + 1) * row_bytes);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (threadIdx.x + i * step) * VEC;
                if (c < d) {
                    Pack<T, VEC> vx, vg;
                    if constexpr (KEEP)
                        vx = px[r][i], vg = pg[r][i];
                    else
                        vx = load_pack<T, VEC>(sx + c), vg = load_pack<T, VEC>(sg + c);
                    float wl[VEC];
                    if constexpr (!KEEP)
                        if (w) load_param<P, VEC>(w, c, wl);
                    Pack<T, VEC> out;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float gv = to_f32(vg.v[j]), xhat = (to_f32(vx.v[j]) - mu[r]) * rs[r];
                        const float gw = KEEP ? gv * wv[KEEP ? i : 0][j] : w ? gv * wl[j] : gv;
                        out.v[j] = from_f32<T>(rs[r] * (gw - m1 - xhat * m2));
                    }
                    *reinterpret_cast<Pack<T, VEC> *>(dx + (long long)row * dxs + c) = out;
                }
            }
        }
    }
    if (!arrived && threadIdx.x == 0)  // copies still under way land in this CTA's memory: wait for them (bounded)
        for (int i = it > stages ? it - stages : 0; i < it + stages - 1; ++i)
            if (blockIdx.x + (long long)i * gridDim.x < groups)
                for (unsigned q = 0; q < kNormSpin && !barrier_try(smem_addr(&full[i % stages]), (uint32_t)(i / stages) & 1u); ++q) {}
    if (!partial) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (threadIdx.x + i * step) * VEC;
        if (c < d) {
            float *a = partial + (long long)blockIdx.x * d + c, *b = a + (long long)gridDim.x * d;
#pragma unroll
            for (int j = 0; j < VEC; j += 4) {
                *reinterpret_cast<float4 *>(a + j) = make_float4(dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]);
                *reinterpret_cast<float4 *>(b + j) = make_float4(db[i][j], db[i][j + 1], db[i][j + 2], db[i][j + 3]);
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
    float a = 0.0f, b = 0.0f;
    if (c < d) {
        int i = k;
        for (; i + 8 < slots; i += 16) {
            a += src[(long long)i * d];
            b += src[(long long)(i + 8) * d];
        }
        if (i < slots) a += src[(long long)i * d];
    }
    sum[k][lane] = a + b;
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
int norm_slots(long long n) { return (int)(n / 27 > current_device_sms() ? n / 27 : current_device_sms()); }
int norm_slots_max() { return 6 * current_device_sms(); }

template <typename T, typename P>
cudaError_t norm_forward(const void *x, long long xs, const void *w, const void *b, void *y, long long ys, float *mean,
                         float *rstd, long long n, int d, float eps, cudaStream_t s)
{
    constexpr int V = 16 / (int)sizeof(T), E = (int)sizeof(T);
    const NormShape sh = norm_shape(d, E, rows_aligned(x, xs, E) && rows_aligned(y, ys, E) && pointer_aligned(w, 16) &&
                                              pointer_aligned(b, 16), kNormVecs, kNormScalars);
    const float inv = 1.0f / (float)d;
    const T *xp = (const T *)x;
    const P *wp = (const P *)w, *bp = (const P *)b;
    T *yp = (T *)y;
    const unsigned rows = (unsigned)n, groups = (unsigned)((n + kNormWarps - 1) / kNormWarps);
    if (sh.threads > kNormMaxThreads)
        return launch_chained(k_norm_forward_long<T, P>, rows, kNormMaxThreads, 0, s, 1, xp, xs, wp, bp, yp, ys, mean,
                              rstd, d, inv, eps);
    // a warp per row: always for short rows, for long ones where rows are enough to fill the device with such warps
    const bool many = groups >= 2u * (unsigned)current_device_sms();
    if (sh.vec && sh.units <= 32 * kNormVecs)
        return launch_chained(k_norm_forward<T, P, V, kNormVecs, true>, groups, 32 * kNormWarps, 0, s, 1, xp, xs, wp,
                              bp, yp, ys, mean, rstd, n, d, inv, eps);
    if (sh.vec && sh.units <= 32 * kNormVecsWarp && many)
        return launch_chained(k_norm_forward<T, P, V, kNormVecsWarp, true>, groups, 32 * kNormWarps, 0, s, 1, xp, xs, wp,
                              bp, yp, ys, mean, rstd, n, d, inv, eps);
    if (sh.vec)
        return launch_chained(k_norm_forward<T, P, V, kNormVecs, false>, rows, sh.threads, 0, s, 1, xp, xs, wp, bp, yp,
                              ys, mean, rstd, n, d, inv, eps);
    if (sh.units <= 32 * kNormScalars)
        return launch_chained(k_norm_forward<T, P, 1, kNormScalars, true>, groups, 32 * kNormWarps, 0, s, 1, xp, xs,
                              wp, bp, yp, ys, mean, rstd, n, d, inv, eps);
    return launch_chained(k_norm_forward<T, P, 1, kNormScalars, false>, rows, sh.threads, 0, s, 1, xp, xs, wp, bp, yp,
                          ys, mean, rstd, n, d, inv, eps);
}

// Launches the ring kernel with `rows` rows per stage if its shared memory holds two stages at least.
template <typename T, int E, int ROWS, typename P>
bool launch_ring(cudaError_t *e, int *slots, int threads, const T *gp, long long dys, const T *xp, long long xs, const P *wp,
                 const float *mean, const float *rstd, T *dxp, long long dxs, float *part, long long n, int d, float inv,
                 cudaStream_t s)
{
    const int stage = ROWS * 2 * d * (int)sizeof(T);
    int ctas = 65536 / (128 * threads);                     // registers
    if (ctas > 2048 / threads) ctas = 2048 / threads;
    while (ctas > 1 && kNormRingBytes / ctas < 3 * stage) --ctas;  // rather fewer CTAs with three stages
    if (ctas < 1) ctas = 1;
    int stages = kNormRingBytes / ctas / stage;
    if (stages > kNormMaxStages) stages = kNormMaxStages;
    if (stages < (ROWS > 1 ? 3 : 2)) return false;
    unsigned int *status = nullptr;
    *e = operator_status_ptr(&status);
    static std::atomic<uint64_t> ready{0};  // devices on which the kernel may have that much shared memory
    int dev = 0;
    if (*e == cudaSuccess) *e = cudaGetDevice(&dev);
    if (*e == cudaSuccess && !(ready.load() >> (dev & 63) & 1)) {
        *e = cudaFuncSetAttribute(k_norm_backward_ring<T, E, ROWS, P>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                  kNormRingBytes);
        if (*e == cudaSuccess) ready.fetch_or(1ull << (dev & 63));
    }
    if (*e != cudaSuccess) return true;
    long long grid = (n + ROWS - 1) / ROWS, most = (long long)ctas * current_device_sms();
    if (most > norm_slots(n)) most = norm_slots(n);
    if (most > norm_slots_max()) most = norm_slots_max();
    if (grid > most) grid = most;
    *slots = (int)grid;
    *e = launch_chained(k_norm_backward_ring<T, E, ROWS, P>, (unsigned)grid, threads, (size_t)stages * stage, s, 1, gp, dys, xp,
                        xs, wp, mean, rstd, dxp, dxs, part, (int)n, d, inv, stages, status);
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
        const long long most = current_device_sms();
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
