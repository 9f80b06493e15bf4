// Gated scan: a recurrence over a sequence's steps, channel by channel, forward and backward.
//
//   a_t = 1 / (1 + exp(-(gate_t + bias))),  b_t = 1 - a_t,  h_t = a_t h_{t-1} + b_t x_t,  y_t = h_t
//   delta_t = dy_t + a_{t+1} delta_{t+1},  dx_t = b_t delta_t,  dgate_t = delta_t a_t b_t (h_{t-1} - x_t)
//
// The step is affine in the state, and so is a run of steps: h -> h + (L - Q h) with Q = 1 - (product of a), which is how runs are
// computed side by side and joined.  b is formed as a value of its own and the state as h + b (x - h), so that a slow
// channel (b of 1e-5) keeps its digits, which a, next to 1, would round away.
//
// A warp takes 64 channels (two a lane, one 4-byte or 8-byte access per row) and runs of S steps, straight from memory to
// registers; the next run's rows are on their way while a run is computed.  Where there are sequences enough for every warp
// to have one, it walks alone.  Otherwise W warps of a CTA take W runs side by side, say what their runs do to a state (L, Q)
// in shared memory and start again from the state that follows; and the CTAs of a cluster do the same with W runs each,
// through one another's shared memory.  Runs are joined in the order of time, whoever is first: results are the same bits from
// call to call.
//
// What bounds it: memory.
#include <atomic>
#include <climits>
#include <mutex>

#include "device_utils.cuh"
#include "operators_internal.cuh"
#include "tensor_core.cuh"

namespace rsdgc {

constexpr int kScanGroup = 64;      // channels of a warp
constexpr int kScanBlock = RSDGC_SCAN_STATE_STEPS;  // steps between the states that the backward pass starts from
constexpr int kScanCluster = 8;     // most CTAs that share a sequence's group
constexpr int kScanLoneWarps = 4;   // of a CTA whose warps walk alone

struct ScanView {                   // a [sequences][steps][width] operand
    const void *p;
    long long seq, step;
};

struct ScanParams {
    ScanView x, gate, y;            // y: dy in the backward pass
    ScanView dx, dgate;             // written
    const void *bias;
    int bias_type;
    const float *first;             // [sequences][width]: the state before the first step; backward: the last state's gradient
    float *last;                    // the state behind the last step; backward: the first state's gradient
    const unsigned char *restart;
    long long restart_stride;
    const long long *lengths;
    float *states;                  // [sequences][blocks of kScanBlock steps][width]
    float *partial;                 // backward: [sequence parts x cluster][width], or NULL
    int n_seq, n_steps, width, groups, blocks;
    int cluster, seq_parts;
    int vec;                        // pairs of channels may be accessed at once
};

__device__ __forceinline__ void scan_store_in(uint32_t addr, uint32_t rank, float4 v)  // to a CTA of the cluster
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr_in(addr, rank)), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// Two neighbouring channels as they lie in memory.  `pair`: one access; otherwise `n` of the two values are there.
template <typename T>
struct Channels {
    typedef uint32_t Raw;
    static __device__ __forceinline__ Raw load(const T *p, bool pair, int n)
    {
        if (pair) return __ldg(reinterpret_cast<const uint32_t *>(p));
        const unsigned short *q = reinterpret_cast<const unsigned short *>(p);
        return (n > 0 ? (uint32_t)__ldg(q) : 0u) | (n > 1 ? (uint32_t)__ldg(q + 1) << 16 : 0u);
    }
    static __device__ __forceinline__ Raw none() { return 0u; }
    static __device__ __forceinline__ float2 widen(Raw r)
    {
        T v[2];
        *reinterpret_cast<uint32_t *>(v) = r;
        return make_float2(to_f32(v[0]), to_f32(v[1]));
    }
    static __device__ __forceinline__ void store(T *p, bool pair, int n, float2 v)
    {
        const uint32_t r = pack2<T>(v.x, v.y);
        if (pair) {
            *reinterpret_cast<uint32_t *>(p) = r;
        } else {
            unsigned short *q = reinterpret_cast<unsigned short *>(p);
            if (n > 0) q[0] = (unsigned short)r;
            if (n > 1) q[1] = (unsigned short)(r >> 16);
        }
    }
};
template <>
struct Channels<float> {
    typedef float2 Raw;
    static __device__ __forceinline__ Raw load(const float *p, bool pair, int n)
    {
        if (pair) return __ldg(reinterpret_cast<const float2 *>(p));
        return make_float2(n > 0 ? __ldg(p) : 0.0f, n > 1 ? __ldg(p + 1) : 0.0f);
    }
    static __device__ __forceinline__ Raw none() { return make_float2(0.0f, 0.0f); }
    static __device__ __forceinline__ float2 widen(Raw r) { return r; }
    static __device__ __forceinline__ void store(float *p, bool pair, int n, float2 v)
    {
        if (pair) {
            *reinterpret_cast<float2 *>(p) = v;
        } else {
            if (n > 0) p[0] = v.x;
            if (n > 1) p[1] = v.y;
        }
    }
};

__device__ __forceinline__ float2 scan_load2(const float *p, int n)
{
    return make_float2(n > 0 ? p[0] : 0.0f, n > 1 ? p[1] : 0.0f);
}
__device__ __forceinline__ void scan_store2(float *p, int n, float2 v)
{
    if (n > 0) p[0] = v.x;
    if (n > 1) p[1] = v.y;
}

// e = exp(-z) from z in units of -log2(e), at most 2^115 so that e * a stays a number (a is 0 there in any case); NaN stays NaN.
__device__ __forceinline__ void scan_gate(float u, float &a, float &b)
{
    float e;
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(u) : "f"(115.0f));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(u));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(1.0f + e));
    b = e * a;
}

// What a run does to a state that comes into it: h -> h + (L - Q h).  Q = kScanCut: the state does not come through.
constexpr float kScanCut = 2.0f;
__device__ __forceinline__ float scan_apply(float l, float q, float h) { return q == kScanCut ? l : h + (l - q * h); }
__device__ __forceinline__ float2 scan_apply(float4 r, float2 h)
{
    return make_float2(scan_apply(r.x, r.z, h.x), scan_apply(r.y, r.w, h.y));
}
// ... and two runs, the second one behind the first
__device__ __forceinline__ void scan_join(float &l, float &q, float l2, float q2)
{
    const bool cut = q == kScanCut || q2 == kScanCut;
    l = scan_apply(l2, q2, l);
    q = cut ? kScanCut : q + q2 * (1.0f - q);
}

constexpr float kScanLog2e = 1.4426950408889634f;

__device__ __forceinline__ float scan_param(const void *p, int type, int i)
{
    return type == RSDGC_F32 ? ((const float *)p)[i]
           : type == RSDGC_BF16 ? to_f32(((const __nv_bfloat16 *)p)[i])
                                : to_f32(((const __half *)p)[i]);
}

// Where a lane stands: its channels.
struct ScanPlace {
    int c, n;        // first channel, channels of this lane (0 to 2)
    bool pair;
    __device__ __forceinline__ ScanPlace(const ScanParams &p, int group, int lane)
    {
        c = group * kScanGroup + 2 * lane;
        n = min(max(p.width - c, 0), 2);
        pair = p.vec && group * kScanGroup + kScanGroup <= p.width;
    }
    __device__ __forceinline__ float2 bias(const ScanParams &p) const  // in the gate's units
    {
        float2 v = make_float2(0.0f, 0.0f);
        if (p.bias) {
            if (n > 0) v.x = -kScanLog2e * scan_param(p.bias, p.bias_type, c);
            if (n > 1) v.y = -kScanLog2e * scan_param(p.bias, p.bias_type, c + 1);
        }
        return v;
    }
};
__device__ __forceinline__ int scan_length(const ScanParams &p, int seq)
{
    if (!p.lengths) return p.n_steps;
    const long long l = p.lengths[seq];
    return l < 0 ? 0 : l > p.n_steps ? p.n_steps : (int)l;
}

// S rows of an operand from step t on; rows outside [0, len) are not read
template <typename T, int S>
__device__ __forceinline__ void scan_rows(typename Channels<T>::Raw (&r)[S], const ScanParams &p, const ScanView &v, int seq,
                                          const ScanPlace &at, int t, int len)
{
    const T *src = (const T *)v.p + seq * v.seq + t * v.step + at.c;
    if (at.pair && t >= 0 && t + S <= len && RSDGC_IN_BOUNDS(seq < p.n_seq && len <= p.n_steps && at.c + 2 <= p.width)) {
#pragma unroll
        for (int i = 0; i < S; ++i, src += v.step) r[i] = Channels<T>::load(src, true, 2);
    } else {
#pragma unroll
        for (int i = 0; i < S; ++i, src += v.step) {
            r[i] = Channels<T>::none();
            if (t + i >= 0 && t + i < len && RSDGC_IN_BOUNDS(seq < p.n_seq && len <= p.n_steps && at.c + at.n <= max(at.c, p.width)))
                r[i] = Channels<T>::load(src, at.pair, at.n);
        }
    }
}

// One byte per lane: whether step t + lane starts a text
template <int S>
__device__ __forceinline__ bool scan_restarts(const ScanParams &p, int seq, int t, int len, int lane)
{
    return p.restart && lane < S && t + lane >= 0 && t + lane < len && p.restart[seq * p.restart_stride + t + lane] != 0;
}

// ---- forward --------------------------------------------------------------------------------------
// W warps of a CTA, p.cluster CTAs share a sequence's group; W = 1: kScanLoneWarps warps with one each.
template <typename T, int S, int W>
__global__ void __launch_bounds__(W == 1 ? 32 * kScanLoneWarps : 32 * W) k_scan_forward(const ScanParams p)
{
    __shared__ float4 runs[W == 1 ? 1 : 2][W][32];                            // by round: what each warp's run does
    __shared__ float4 parts[W == 1 ? 1 : 2][W == 1 ? 1 : kScanCluster][32];   // ... and each CTA's W runs
    typedef typename Channels<T>::Raw Raw;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cluster = W == 1 ? 1 : p.cluster, rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int unit = W == 1 ? blockIdx.x * kScanLoneWarps + warp : (int)blockIdx.x / cluster;
    grid_dependency_wait();
    grid_dependency_launch_next();
    const int seq = unit / p.groups, group = unit - seq * p.groups;
    if (seq >= p.n_seq) return;  // W = 1 only: a warp too many
    if (cluster > 1) cluster_sync_all();  // nothing is written to a CTA that has not begun
    const ScanPlace at(p, group, lane);
    const float2 bias = at.bias(p), scale = make_float2(-kScanLog2e, -kScanLog2e);
    const int len = scan_length(p, seq);
    const int run = W == 1 ? 0 : warp, tile = S * W, stride = tile * cluster;
    float2 h = make_float2(0.0f, 0.0f);  // the state that comes into the round
    if (p.first) h = scan_load2(p.first + (long long)seq * p.width + at.c, at.n);

    int t = rank * tile + run * S, parity = 0;
    Raw xr[S], gr[S];
    scan_rows<T, S>(xr, p, p.x, seq, at, t, len);
    scan_rows<T, S>(gr, p, p.gate, seq, at, t, len);
    bool starts = scan_restarts<S>(p, seq, t, len, lane);
    for (int t0 = 0; t0 < len; t0 += stride, t += stride, parity ^= 1) {
        float2 x[S], b[S];
        const uint32_t restart = __ballot_sync(0xFFFFFFFFu, starts);
#pragma unroll
        for (int i = 0; i < S; ++i) {
            float a;
            const float2 u = fma2(Channels<T>::widen(gr[i]), scale, bias);
            x[i] = Channels<T>::widen(xr[i]);
            scan_gate(u.x, a, b[i].x);
            scan_gate(u.y, a, b[i].y);
        }
        if (t + S > len) {  // steps that do not exist leave the state as it is
#pragma unroll
            for (int i = 0; i < S; ++i)
                if (t + i >= len) b[i] = make_float2(0.0f, 0.0f);
        }
        if (t0 + stride < len) {
            scan_rows<T, S>(xr, p, p.x, seq, at, t + stride, len);
            scan_rows<T, S>(gr, p, p.gate, seq, at, t + stride, len);
            starts = scan_restarts<S>(p, seq, t + stride, len, lane);
        }
        if (W > 1) {
            float2 l = make_float2(0.0f, 0.0f), q = l, r = make_float2(1.0f, 1.0f);  // r = 1 - q, of its own digits
            if (!restart) {
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    const float2 m = make_float2(-l.x, -l.y), s = mul2(b[i], r);
                    l = fma2(b[i], add2(x[i], m), l);
                    q = add2(q, s);
                    r = add2(r, make_float2(-s.x, -s.y));
                }
            } else {
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    if (restart >> i & 1) l = make_float2(0.0f, 0.0f);
                    l = fma2(b[i], make_float2(x[i].x - l.x, x[i].y - l.y), l);
                }
                q = make_float2(kScanCut, kScanCut);
            }
            runs[parity][warp][lane] = make_float4(l.x, l.y, q.x, q.y);
            __syncthreads();
            float2 in = h;
            if (cluster > 1) {
                // warp k tells CTA k what this CTA's runs do
                if (warp < cluster) {
                    float4 all = runs[parity][0][lane];
                    for (int w = 1; w < W; ++w) {
                        const float4 o = runs[parity][w][lane];
                        scan_join(all.x, all.z, o.x, o.z);
                        scan_join(all.y, all.w, o.y, o.w);
                    }
                    for (int k = warp; k < cluster; k += W) scan_store_in(smem_addr(&parts[parity][rank][lane]), (uint32_t)k, all);
                }
                cluster_sync_all();
                for (int k = 0; k < cluster; ++k) {
                    if (k == rank) in = h;
                    h = scan_apply(parts[parity][k][lane], h);
                }
                for (int w = 0; w < warp; ++w) in = scan_apply(runs[parity][w][lane], in);
            } else {
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    if (w == warp) in = h;
                    h = scan_apply(runs[parity][w][lane], h);
                }
            }
            if (t >= len) continue;
            if (p.states && t % kScanBlock == 0 && RSDGC_IN_BOUNDS(t / kScanBlock < p.blocks))
                scan_store2(p.states + ((long long)seq * p.blocks + t / kScanBlock) * p.width + at.c, at.n, in);
            T *dst = (T *)p.y.p + seq * p.y.seq + t * p.y.step + at.c;
#pragma unroll
            for (int i = 0; i < S; ++i, dst += p.y.step) {
                if (restart >> i & 1) in = make_float2(0.0f, 0.0f);
                in = fma2(b[i], add2(x[i], make_float2(-in.x, -in.y)), in);
                if (t + i < len && RSDGC_IN_BOUNDS(t + i < p.n_steps)) Channels<T>::store(dst, at.pair, at.n, in);
            }
        } else {
            if (p.states && t % kScanBlock == 0 && RSDGC_IN_BOUNDS(t / kScanBlock < p.blocks))
                scan_store2(p.states + ((long long)seq * p.blocks + t / kScanBlock) * p.width + at.c, at.n, h);
            T *dst = (T *)p.y.p + seq * p.y.seq + t * p.y.step + at.c;
#pragma unroll
            for (int i = 0; i < S; ++i, dst += p.y.step) {
                if (restart >> i & 1) h = make_float2(0.0f, 0.0f);
                h = fma2(b[i], add2(x[i], make_float2(-h.x, -h.y)), h);
                if (t + i < len && RSDGC_IN_BOUNDS(t + i < p.n_steps)) Channels<T>::store(dst, at.pair, at.n, h);
            }
        }
    }
    if (p.last && rank == 0 && run == 0) scan_store2(p.last + (long long)seq * p.width + at.c, at.n, h);
}

// ---- backward -------------------------------------------------------------------------------------
// The same runs, the last one first.  A run's states are computed again from the state saved at the head of its block of
// kScanBlock steps; what a run does to the gradient that comes into it from behind is e -> R + P e, P the product of its a.
template <typename T, int S, int W>
__global__ void __launch_bounds__(32 * W) k_scan_backward(const ScanParams p)
{
    static_assert(S * W % kScanBlock == 0 && kScanBlock % S == 0, "a CTA's runs are whole blocks");
    constexpr int kPer = kScanBlock / S;  // runs of a block
    __shared__ float4 runs[2][W][32];     // (L, R) of the two channels
    __shared__ float2 through[2][W][32];  // P; 0: nothing comes through
    __shared__ float4 parts[2][kScanCluster][32];  // of a CTA's W runs: (R, P)
    typedef typename Channels<T>::Raw Raw;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cluster = p.cluster, rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int unit = (int)blockIdx.x / cluster;
    grid_dependency_wait();
    grid_dependency_launch_next();
    const int part = unit / p.groups, group = unit - part * p.groups;
    if (cluster > 1) cluster_sync_all();  // nothing is written to a CTA that has not begun
    const ScanPlace at(p, group, lane);
    const float2 bias = at.bias(p), scale = make_float2(-kScanLog2e, -kScanLog2e);
    constexpr int tile = S * W;
    float2 sum = make_float2(0.0f, 0.0f), rest = sum;  // of dgate, with what the sum's rounding left out
    int parity = 0;
    for (int seq = part; seq < p.n_seq; seq += p.seq_parts) {
        const int len = scan_length(p, seq);
        float2 e = make_float2(0.0f, 0.0f);  // the gradient that comes into the round from behind
        if (p.first) e = scan_load2(p.first + (long long)seq * p.width + at.c, at.n);
        const int tiles = (len + tile - 1) / tile;
        int t = (tiles - 1 - rank) * tile + warp * S;
        Raw xr[S], gr[S], yr[S];
        float2 from;
        bool starts;
        auto load = [&]() {
            scan_rows<T, S>(xr, p, p.x, seq, at, t, len);
            scan_rows<T, S>(gr, p, p.gate, seq, at, t, len);
            scan_rows<T, S>(yr, p, p.y, seq, at, t, len);
            starts = scan_restarts<S>(p, seq, t, len, lane);
            from = make_float2(0.0f, 0.0f);
            if (t >= 0 && t < len && RSDGC_IN_BOUNDS(t / kScanBlock < p.blocks))
                from = scan_load2(p.states + ((long long)seq * p.blocks + t / kScanBlock) * p.width + at.c, at.n);
        };
        load();
        for (int left = tiles; left > 0; left -= cluster, parity ^= 1) {
            float2 x[S], b[S], dy[S];
            const uint32_t restart = __ballot_sync(0xFFFFFFFFu, starts);
            float2 h = from;
            const int t1 = t;
#pragma unroll
            for (int i = 0; i < S; ++i) {
                float a;
                const float2 u = fma2(Channels<T>::widen(gr[i]), scale, bias);
                x[i] = Channels<T>::widen(xr[i]);
                dy[i] = Channels<T>::widen(yr[i]);
                scan_gate(u.x, a, b[i].x);
                scan_gate(u.y, a, b[i].y);
            }
            if (t1 < 0 || t1 + S > len) {
#pragma unroll
                for (int i = 0; i < S; ++i)
                    if (t1 + i < 0 || t1 + i >= len) b[i] = make_float2(0.0f, 0.0f);
            }
            t -= tile * cluster;
            if (left > cluster) load();
            // the run from no state, and from no gradient behind it
            float2 l = make_float2(0.0f, 0.0f), r = l, q = make_float2(1.0f, 1.0f);
#pragma unroll
            for (int i = 0; i < S; ++i) {
                if (restart >> i & 1) l = make_float2(0.0f, 0.0f);
                l = fma2(b[i], add2(x[i], make_float2(-l.x, -l.y)), l);
            }
#pragma unroll
            for (int i = S - 1; i >= 0; --i) {
                const float2 m = make_float2(-b[i].x, -b[i].y);
                const float2 d = add2(dy[i], r);
                r = fma2(m, d, d);
                q = fma2(m, q, q);
                if (restart >> i & 1) r = make_float2(0.0f, 0.0f);
            }
            // a product too small for a number is not yet a cut
            q = restart ? make_float2(0.0f, 0.0f) : make_float2(fmaxf(q.x, 1.2e-38f), fmaxf(q.y, 1.2e-38f));
            runs[parity][warp][lane] = make_float4(l.x, l.y, r.x, r.y);
            through[parity][warp][lane] = q;
            __syncthreads();
            for (int w = warp / kPer * kPer; w < warp; ++w) {
                const float4 o = runs[parity][w][lane];
                const float2 k = through[parity][w][lane];
                h.x = k.x == 0.0f ? o.x : fmaf(k.x, h.x, o.x);
                h.y = k.y == 0.0f ? o.y : fmaf(k.y, h.y, o.y);
            }
            auto back = [&](float4 o, float2 k, float2 v) {  // R in o.z, o.w
                return make_float2(k.x == 0.0f ? o.z : fmaf(k.x, v.x, o.z), k.y == 0.0f ? o.w : fmaf(k.y, v.y, o.w));
            };
            float2 in = e;
            if (cluster > 1) {
                if (warp < cluster) {
                    float2 all = make_float2(0.0f, 0.0f), k = make_float2(1.0f, 1.0f);
                    for (int w = W - 1; w >= 0; --w) {
                        const float2 o = through[parity][w][lane];
                        all = back(runs[parity][w][lane], o, all);
                        k.x = o.x == 0.0f || k.x == 0.0f ? 0.0f : fmaxf(k.x * o.x, 1.2e-38f);
                        k.y = o.y == 0.0f || k.y == 0.0f ? 0.0f : fmaxf(k.y * o.y, 1.2e-38f);
                    }
                    for (int to = warp; to < cluster; to += W)
                        scan_store_in(smem_addr(&parts[parity][rank][lane]), (uint32_t)to, make_float4(all.x, all.y, k.x, k.y));
                }
                cluster_sync_all();
                for (int k = 0; k < cluster; ++k) {
                    const float4 o = parts[parity][k][lane];
                    if (k == rank) in = e;
                    e = back(make_float4(0.0f, 0.0f, o.x, o.y), make_float2(o.z, o.w), e);
                }
                for (int w = W - 1; w > warp; --w) in = back(runs[parity][w][lane], through[parity][w][lane], in);
            } else {
                for (int w = W - 1; w >= 0; --w) {
                    if (w == warp) in = e;
                    e = back(runs[parity][w][lane], through[parity][w][lane], e);
                }
            }
            if (t1 < 0 || t1 >= len) continue;
            // x becomes h_{t-1} - x_t
#pragma unroll
            for (int i = 0; i < S; ++i) {
                if (restart >> i & 1) h = make_float2(0.0f, 0.0f);
                x[i] = add2(h, make_float2(-x[i].x, -x[i].y));
                h = fma2(make_float2(-b[i].x, -b[i].y), x[i], h);
            }
            T *dx = (T *)p.dx.p + seq * p.dx.seq + (t1 + S - 1) * p.dx.step + at.c;
            T *dg = (T *)p.dgate.p + seq * p.dgate.seq + (t1 + S - 1) * p.dgate.step + at.c;
            float2 add = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = S - 1; i >= 0; --i, dx -= p.dx.step, dg -= p.dgate.step) {
                const float2 d = add2(dy[i], in), db = mul2(d, b[i]);
                const float2 ad = add2(d, make_float2(-db.x, -db.y));  // a d
                const float2 dz = mul2(mul2(ad, b[i]), x[i]);
                if (t1 + i < len && RSDGC_IN_BOUNDS(t1 + i < p.n_steps)) {
                    if (p.dx.p) Channels<T>::store(dx, at.pair, at.n, db);
                    if (p.dgate.p) Channels<T>::store(dg, at.pair, at.n, dz);
                }
                add = add2(add, dz);
                in = restart >> i & 1 ? make_float2(0.0f, 0.0f) : ad;
            }
            // Kahan's sum: a channel may have millions of steps
            const float2 y = make_float2(add.x - rest.x, add.y - rest.y), s = make_float2(sum.x + y.x, sum.y + y.y);
            rest = make_float2((s.x - sum.x) - y.x, (s.y - sum.y) - y.y);
            sum = s;
        }
        if (p.last && rank == 0 && warp == 0) scan_store2(p.last + (long long)seq * p.width + at.c, at.n, e);
    }
    if (!p.partial) return;
    __syncthreads();
    float2 *all = &through[0][0][0];
    all[warp * 32 + lane] = sum;
    __syncthreads();
    if (warp == 0) {
        for (int w = 1; w < W; ++w) sum = add2(sum, all[w * 32 + lane]);
        const int slot = part * cluster + rank;
        if (RSDGC_IN_BOUNDS(slot < p.seq_parts * cluster)) scan_store2(p.partial + (long long)slot * p.width + at.c, at.n, sum);
    }
}

// dbias = the sum of its parts, in order: eight threads a channel.
template <typename G>
__global__ void __launch_bounds__(256)
k_scan_bias_gradient(const float *__restrict__ partial, int parts, int width, G *__restrict__ dbias)
{
    __shared__ double sums[8][32];
    const int lane = threadIdx.x & 31, row = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    grid_dependency_wait();
    grid_dependency_launch_next();
    double s = 0.0;
    if (c < width)
        for (int i = row; i < parts; i += 8) s += partial[(long long)i * width + c];
    sums[row][lane] = s;
    __syncthreads();
    if (row == 0 && c < width) {
        for (int i = 1; i < 8; ++i) s += sums[i][lane];
        dbias[c] = from_f32<G>((float)s);
    }
}

// ---- host -------------------------------------------------------------------------------------------
RSDGC_DEFINE_DEBUG_BOUNDS(gated_scan_debug_bounds)

namespace {

constexpr int kScanSms = 148;
constexpr int64_t kScanParts = 16 * kScanSms;  // CTAs from which on the backward pass gives one several sequences

int scan_check(int64_t n, int64_t t, int64_t d)
{
    if (n < 0 || t < 0 || d < 1) return RSDGC_ERR_INVALID;
    if (n > (1 << 30) || t > (1 << 30) || d > (1 << 24)) return RSDGC_ERR_CAPACITY;
    const int64_t groups = (d + kScanGroup - 1) / kScanGroup;
    return n * groups > INT_MAX / kScanCluster ? RSDGC_ERR_CAPACITY : RSDGC_OK;
}

inline int scan_groups(int64_t d) { return (int)((d + kScanGroup - 1) / kScanGroup); }
inline int scan_blocks(int64_t t) { return (int)((t + kScanBlock - 1) / kScanBlock); }

// CTAs that share a sequence's group: as many as bring the launch's rounds down, but each with runs of its own.
int scan_cluster(int64_t units, int64_t steps, int tile, int per_sm)
{
    const int64_t slots = (int64_t)per_sm * kScanSms;
    int best = 1;
    for (int k = 2; k <= kScanCluster && (int64_t)(k - 1) * tile < steps; k *= 2)
        if ((units * k + slots - 1) / slots * best < (units * best + slots - 1) / slots * k) best = k;
    return best;
}

int64_t scan_seq_parts(int64_t n, int64_t d)
{
    const int64_t most = kScanParts / scan_groups(d) > 1 ? kScanParts / scan_groups(d) : 1;
    return n < most ? n : most;
}

bool scan_pairs(const ScanView &v, int elem)
{
    return pointer_aligned(v.p, 2 * elem) && v.seq % 2 == 0 && v.step % 2 == 0;
}

template <typename F>
cudaError_t scan_type(int dtype, F f)
{
    return dtype == RSDGC_F32 ? f(float{}) : dtype == RSDGC_BF16 ? f(__nv_bfloat16{}) : f(__half{});
}

constexpr int kS = 16, kWFwd = 4, kWBack = 4;

template <typename T>
cudaError_t scan_forward(ScanParams &p, cudaStream_t s)
{
    const long long units = (long long)p.n_seq * p.groups;
    if (p.n_steps <= kS || units >= 16 * kScanSms)
        return launch_chained(k_scan_forward<T, kS, 1>, (unsigned)((units + kScanLoneWarps - 1) / kScanLoneWarps),
                              32 * kScanLoneWarps, 0, s, 1, p);
    p.cluster = scan_cluster(units, p.n_steps, kS * kWFwd, 4);
    return launch_chained(k_scan_forward<T, kS, kWFwd>, (unsigned)(units * p.cluster), 32 * kWFwd, 0, s, p.cluster, p);
}

template <typename T>
cudaError_t scan_backward(ScanParams &p, cudaStream_t s)
{
    const long long units = (long long)p.seq_parts * p.groups;
    return launch_chained(k_scan_backward<T, kS, kWBack>, (unsigned)(units * p.cluster), 32 * kWBack, 0, s, p.cluster, p);
}

int scan_backward_cluster(int64_t n, int64_t t, int64_t d)
{
    return scan_cluster(scan_seq_parts(n, d) * scan_groups(d), t, kS * kWBack, 3);
}

// A strided operand: its rows do not overlap, its values are aligned.
int scan_view_check(const ScanView &v, int64_t n, int64_t t, int64_t d, int elem)
{
    if (!v.p || (t > 1 && v.step < d) || (n > 1 && v.seq < d)) return RSDGC_ERR_INVALID;
    return pointer_aligned(v.p, elem) ? RSDGC_OK : RSDGC_ERR_ALIGNMENT;
}

}  // namespace
}  // namespace rsdgc

using namespace rsdgc;

extern "C" int64_t rsdgc_gated_scan_workspace_bytes(int64_t n_seq, int64_t n_steps, int64_t width)
{
    const int rc = scan_check(n_seq, n_steps, width);
    return rc ? rc : 4 * width * scan_seq_parts(n_seq, width) * scan_backward_cluster(n_seq, n_steps, width);
}

extern "C" int rsdgc_gated_scan_forward(const void *x_dev, int64_t x_seq, int64_t x_step, const void *gate_dev, int64_t gate_seq,
                                        int64_t gate_step, const void *gate_bias_dev, void *y_dev, int64_t y_seq, int64_t y_step,
                                        const float *first_dev, float *last_dev, const uint8_t *restart_dev,
                                        int64_t restart_stride, const int64_t *lengths_dev, float *states_dev, int64_t n_seq,
                                        int64_t n_steps, int64_t width, int32_t dtype, int32_t param_dtype, void *stream)
{
    int rc = scan_check(n_seq, n_steps, width);
    if (rc) return rc;
    if (!known_dtype(dtype) || (gate_bias_dev && param_dtype != dtype && param_dtype != RSDGC_F32)) return RSDGC_ERR_INVALID;
    if (n_seq == 0) return RSDGC_OK;
    ScanParams p{};
    p.x = {x_dev, x_seq, x_step};
    p.gate = {gate_dev, gate_seq, gate_step};
    p.y = {y_dev, y_seq, y_step};
    const int elem = dtype_bytes(dtype);
    if (n_steps > 0) {
        for (const ScanView *v : {&p.x, &p.gate, &p.y})
            if ((rc = scan_view_check(*v, n_seq, n_steps, width, elem))) return rc;
        if (restart_dev && n_seq > 1 && restart_stride < n_steps) return RSDGC_ERR_INVALID;
    }
    if (!pointer_aligned(gate_bias_dev, dtype_bytes(param_dtype)) || !pointer_aligned(first_dev, 4) || !pointer_aligned(last_dev, 4) ||
        !pointer_aligned(lengths_dev, 8) || !pointer_aligned(states_dev, 4))
        return RSDGC_ERR_ALIGNMENT;
    OperatorRange range("rsdgc_gated_scan_forward");
    p.bias = gate_bias_dev;
    p.bias_type = param_dtype;
    p.first = first_dev;
    p.last = last_dev;
    p.restart = restart_dev;
    p.restart_stride = restart_stride;
    p.lengths = (const long long *)lengths_dev;
    p.states = states_dev;
    p.n_seq = (int)n_seq;
    p.n_steps = (int)n_steps;
    p.width = (int)width;
    p.groups = scan_groups(width);
    p.blocks = scan_blocks(n_steps);
    p.cluster = 1;
    p.vec = scan_pairs(p.x, elem) && scan_pairs(p.gate, elem) && scan_pairs(p.y, elem);
    cudaError_t e = operators_ready();
    if (e == cudaSuccess) e = scan_type(dtype, [&](auto t) { return scan_forward<decltype(t)>(p, (cudaStream_t)stream); });
    return operator_result(e);
}

extern "C" int rsdgc_gated_scan_backward(const void *dy_dev, int64_t dy_seq, int64_t dy_step, const void *x_dev, int64_t x_seq,
                                         int64_t x_step, const void *gate_dev, int64_t gate_seq, int64_t gate_step,
                                         const void *gate_bias_dev, const float *states_dev, const float *dlast_dev, void *dx_dev,
                                         int64_t dx_seq, int64_t dx_step, void *dgate_dev, int64_t dgate_seq, int64_t dgate_step,
                                         void *dbias_dev, float *dfirst_dev, const uint8_t *restart_dev, int64_t restart_stride,
                                         const int64_t *lengths_dev, int64_t n_seq, int64_t n_steps, int64_t width, int32_t dtype,
                                         int32_t param_dtype, int32_t grad_dtype, void *workspace_dev, void *stream)
{
    int rc = scan_check(n_seq, n_steps, width);
    if (rc) return rc;
    if (!known_dtype(dtype) || (gate_bias_dev && param_dtype != dtype && param_dtype != RSDGC_F32)) return RSDGC_ERR_INVALID;
    if (!dx_dev && !dgate_dev && !dbias_dev && !dfirst_dev) return RSDGC_ERR_INVALID;
    if (dbias_dev && !known_dtype(grad_dtype)) return RSDGC_ERR_INVALID;
    ScanParams p{};
    p.x = {x_dev, x_seq, x_step};
    p.gate = {gate_dev, gate_seq, gate_step};
    p.y = {dy_dev, dy_seq, dy_step};
    p.dx = {dx_dev, dx_seq, dx_step};
    p.dgate = {dgate_dev, dgate_seq, dgate_step};
    const int elem = dtype_bytes(dtype);
    if (n_seq > 0 && n_steps > 0) {
        for (const ScanView *v : {&p.x, &p.gate, &p.y})
            if ((rc = scan_view_check(*v, n_seq, n_steps, width, elem))) return rc;
        for (const ScanView *v : {&p.dx, &p.dgate})
            if (v->p && (rc = scan_view_check(*v, n_seq, n_steps, width, elem))) return rc;
        if (!states_dev || (restart_dev && n_seq > 1 && restart_stride < n_steps)) return RSDGC_ERR_INVALID;
        if (dbias_dev && !workspace_dev) return RSDGC_ERR_INVALID;
    }
    if (!pointer_aligned(gate_bias_dev, dtype_bytes(param_dtype)) || !pointer_aligned(dlast_dev, 4) ||
        !pointer_aligned(dfirst_dev, 4) || !pointer_aligned(lengths_dev, 8) || !pointer_aligned(states_dev, 4) ||
        !pointer_aligned(dbias_dev, dtype_bytes(grad_dtype)) || !pointer_aligned(workspace_dev, 16))
        return RSDGC_ERR_ALIGNMENT;
    OperatorRange range("rsdgc_gated_scan_backward");
    cudaStream_t s = (cudaStream_t)stream;
    if (n_seq == 0 || n_steps == 0) {  // sums over nothing; the state's gradient goes through
        cudaError_t e = cudaSuccess;
        const size_t rows = (size_t)n_seq * width * 4;
        if (dbias_dev) e = cudaMemsetAsync(dbias_dev, 0, (size_t)width * dtype_bytes(grad_dtype), s);
        if (e == cudaSuccess && dfirst_dev && rows)
            e = !dlast_dev ? cudaMemsetAsync(dfirst_dev, 0, rows, s)
                : dlast_dev != dfirst_dev ? cudaMemcpyAsync(dfirst_dev, dlast_dev, rows, cudaMemcpyDeviceToDevice, s) : e;
        return operator_result(e);
    }
    p.bias = gate_bias_dev;
    p.bias_type = param_dtype;
    p.first = dlast_dev;
    p.last = dfirst_dev;
    p.restart = restart_dev;
    p.restart_stride = restart_stride;
    p.lengths = (const long long *)lengths_dev;
    p.states = const_cast<float *>(states_dev);
    p.partial = dbias_dev ? (float *)workspace_dev : nullptr;
    p.n_seq = (int)n_seq;
    p.n_steps = (int)n_steps;
    p.width = (int)width;
    p.groups = scan_groups(width);
    p.blocks = scan_blocks(n_steps);
    p.seq_parts = (int)scan_seq_parts(n_seq, width);
    p.cluster = scan_backward_cluster(n_seq, n_steps, width);
    p.vec = scan_pairs(p.x, elem) && scan_pairs(p.gate, elem) && scan_pairs(p.y, elem) && (!dx_dev || scan_pairs(p.dx, elem)) &&
            (!dgate_dev || scan_pairs(p.dgate, elem));
    cudaError_t e = operators_ready();
    if (e == cudaSuccess) e = scan_type(dtype, [&](auto t) { return scan_backward<decltype(t)>(p, s); });
    if (e == cudaSuccess && dbias_dev)
        e = scan_type(grad_dtype, [&](auto g) {
            typedef decltype(g) G;
            return launch_chained(k_scan_bias_gradient<G>, (unsigned)((width + 31) / 32), 256, 0, s, 1, (const float *)p.partial,
                                  p.seq_parts * p.cluster, (int)width, (G *)dbias_dev);
        });
    return operator_result(e);
}
