// Layer norm, forward and backward, with the reduction of the weight's and the bias's gradient.
//
//   mean = sum x / D,  rstd = (sum (x - mean)^2 / D + eps)^(-1/2),  xhat = (x - mean) rstd,  y = xhat w + b
//   dx = rstd (g w - mean(g w) - xhat mean(g w xhat)),  dw = sum_n g xhat,  db = sum_n g
//
// Bound: memory (about 2 flop per byte).  A row is read once and stays in registers: the mean, then the
// centred squares (two reductions, no cancellation), then the output.  All statistics and sums are binary32.
#include <climits>

#include "device_utils.cuh"
#include "operators_internal.cuh"

namespace rsdgc {

constexpr int kNormVecs = 4;          // 16-byte vectors of a row that a thread holds
constexpr int kNormScalars = 16;      // elements it holds where rows are not 16-byte aligned
constexpr int kNormMaxThreads = 1024;
constexpr int kNormBackThreads = 512; // backward: 128 registers for the columns' sums and two rows of operands
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
// A CTA (or warp) walks the rows blockIdx.x, blockIdx.x + gridDim.x, ... and keeps the sums of the columns it
// owns for dw and db in registers; they go to `partial` ([2][CTAs][d]) at the end and are added up in a fixed
// order by k_norm_param_gradient: no atomics, the same bits from run to run.  The next row is loaded while
// this one is reduced.
template <typename T, typename P, int VEC, int NV, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kNormWarps : kNormBackThreads)
k_norm_backward(const T *__restrict__ dy, long long dys, const T *__restrict__ x, long long xs,
                const P *__restrict__ w, const float *__restrict__ mean, const float *__restrict__ rstd,
                T *__restrict__ dx, long long dxs, float *__restrict__ partial, long long n, int d, float inv_d)
{
    __shared__ float2 part[2][32];
    const int tid = WARP ? (threadIdx.x & 31) : threadIdx.x;
    const int step = WARP ? 32 : blockDim.x;
    const long long first = WARP ? (long long)blockIdx.x * kNormWarps + (threadIdx.x >> 5) : (long long)blockIdx.x;
    const long long stride = WARP ? (long long)gridDim.x * kNormWarps : (long long)gridDim.x;
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
    const long long slot = WARP ? (long long)blockIdx.x * kNormWarps + (threadIdx.x >> 5) : (long long)blockIdx.x;
    const long long slots = WARP ? (long long)gridDim.x * kNormWarps : (long long)gridDim.x;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (tid + i * step) * VEC;
        if (c < d) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                partial[slot * d + c + j] = dw[i][j];
                partial[(slots + slot) * d + c + j] = db[i][j];
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

struct NormShape {
    bool vec, warp, lng;
    int threads;
};

// 16-byte accesses where every row of every operand starts on such a boundary and the width is a whole number
// of packs; a warp per row while a row fits a warp's registers.
NormShape norm_shape(int d, int elem, bool aligned, int most = kNormMaxThreads)
{
    NormShape s{};
    const int vec = 16 / elem;
    s.vec = aligned && d % vec == 0;
    const int units = s.vec ? d / vec : d, per = s.vec ? kNormVecs : kNormScalars;
    s.warp = units <= 32 * per;
    s.threads = ((units + per - 1) / per + 31) / 32 * 32;
    s.lng = s.threads > most;
    return s;
}

int norm_slots_max() { return 4 * current_device_sms(); }

template <typename T, typename P>
cudaError_t norm_forward(const void *x, long long xs, const void *w, const void *b, void *y, long long ys, float *mean,
                         float *rstd, long long n, int d, float eps, cudaStream_t s)
{
    constexpr int V = 16 / (int)sizeof(T);
    const bool aligned = pointer_aligned(x, 16) && pointer_aligned(y, 16) && (xs * (long long)sizeof(T)) % 16 == 0 &&
                         (ys * (long long)sizeof(T)) % 16 == 0 && pointer_aligned(w, 16) &&
                         pointer_aligned(b, 16);
    const NormShape sh = norm_shape(d, (int)sizeof(T), aligned);
    const float inv = 1.0f / (float)d;
    const T *xp = (const T *)x;
    const P *wp = (const P *)w, *bp = (const P *)b;
    T *yp = (T *)y;
    const unsigned rows = (unsigned)n, groups = (unsigned)((n + kNormWarps - 1) / kNormWarps);
    if (sh.lng)
        return launch_chained(k_norm_forward_long<T, P>, rows, kNormMaxThreads, 0, s, 1, xp, xs, wp, bp, yp, ys, mean,
                              rstd, d, inv, eps);
    if (sh.vec && sh.warp)
        return launch_chained(k_norm_forward<T, P, V, kNormVecs, true>, groups, 32 * kNormWarps, 0, s, 1, xp, xs, wp,
                              bp, yp, ys, mean, rstd, n, d, inv, eps);
    if (sh.vec)
        return launch_chained(k_norm_forward<T, P, V, kNormVecs, false>, rows, sh.threads, 0, s, 1, xp, xs, wp, bp, yp,
                              ys, mean, rstd, n, d, inv, eps);
    if (sh.warp)
        return launch_chained(k_norm_forward<T, P, 1, kNormScalars, true>, groups, 32 * kNormWarps, 0, s, 1, xp, xs,
                              wp, bp, yp, ys, mean, rstd, n, d, inv, eps);
    return launch_chained(k_norm_forward<T, P, 1, kNormScalars, false>, rows, sh.threads, 0, s, 1, xp, xs, wp, bp, yp,
                          ys, mean, rstd, n, d, inv, eps);
}

template <typename T, typename P>
cudaError_t norm_backward(const void *dy, long long dys, const void *x, long long xs, const void *w, const float *mean,
                          const float *rstd, void *dx, long long dxs, void *dw, void *db, int grad_type, long long n,
                          int d, float *partial, cudaStream_t s)
{
    constexpr int V = 16 / (int)sizeof(T);
    const bool aligned = pointer_aligned(x, 16) && pointer_aligned(dy, 16) && pointer_aligned(dx, 16) &&
                         (xs * (long long)sizeof(T)) % 16 == 0 && (dys * (long long)sizeof(T)) % 16 == 0 && (dxs * (long long)sizeof(T)) % 16 == 0 &&
                         pointer_aligned(w, 16);
    const NormShape sh = norm_shape(d, (int)sizeof(T), aligned, kNormBackThreads);
    const float inv = 1.0f / (float)d;
    const T *xp = (const T *)x, *gp = (const T *)dy;
    const P *wp = (const P *)w;
    T *dxp = (T *)dx;
    float *part = dw || db ? partial : nullptr;
    int slots = 0;
    cudaError_t e = cudaSuccess;
    if (sh.lng) {
        if (dx)
            e = launch_chained(k_norm_backward_long<T, P>, (unsigned)n, kNormMaxThreads, 0, s, 1, gp, dys, xp, xs, wp,
                               mean, rstd, dxp, dxs, d, inv);
        if (e == cudaSuccess && part) {
            slots = (int)(n < 64 ? n : 64);
            e = launch_chained(k_norm_columns_long<T>, dim3((unsigned)((d + 255) / 256), (unsigned)slots), 256, 0, s, 1,
                               gp, dys, xp, xs, mean, rstd, part, n, d);
        }
    } else if (sh.warp) {
        const long long groups = (n + kNormWarps - 1) / kNormWarps, most = norm_slots_max() / kNormWarps;
        const unsigned g = (unsigned)(groups < most ? groups : most);
        slots = (int)g * kNormWarps;
        if (sh.vec)
            e = launch_chained(k_norm_backward<T, P, V, kNormVecs, true>, g, 32 * kNormWarps, 0, s, 1, gp, dys, xp, xs, wp,
                               mean, rstd, dxp, dxs, part, n, d, inv);
        else
            e = launch_chained(k_norm_backward<T, P, 1, kNormScalars, true>, g, 32 * kNormWarps, 0, s, 1, gp, dys, xp, xs,
                               wp, mean, rstd, dxp, dxs, part, n, d, inv);
    } else {
        const long long most = current_device_sms();
        slots = (int)(n < most ? n : most);
        if (sh.vec)
            e = launch_chained(k_norm_backward<T, P, V, kNormVecs, false>, (unsigned)slots, sh.threads, 0, s, 1, gp, dys,
                               xp, xs, wp, mean, rstd, dxp, dxs, part, n, d, inv);
        else
            e = launch_chained(k_norm_backward<T, P, 1, kNormScalars, false>, (unsigned)slots, sh.threads, 0, s, 1, gp,
                               dys, xp, xs, wp, mean, rstd, dxp, dxs, part, n, d, inv);
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
