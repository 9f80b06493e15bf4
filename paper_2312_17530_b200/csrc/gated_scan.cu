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
constexpr int kRun = RSDGC_SCAN_STATE_STEPS;  // steps of a run
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
    float *states;                  // [sequences][runs][width]: the state before each run
    float *partial;                 // backward: [sequence parts x cluster][width], or NULL
    int n_seq, n_steps, width, groups, runs;
    int cluster, seq_parts;
    int vec, wide;                  // pairs of channels may be accessed at once; 16 bytes may be read at once
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

// -b = -1 / (1 + exp(z)) for z log2(e) = u.  It never leaves [-1, 0], whatever u is; NaN stays NaN.
__device__ __forceinline__ float scan_gate(float u)
{
    float e, nb;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(u));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(nb) : "f"(-1.0f - e));
    return nb;
}

// What a run does to the (negated) state that comes into it: m -> m + (L - Q m).  Q = kScanCut: the state does not come through.
constexpr float kScanCut = 2.0f;
__device__ __forceinline__ float scan_apply(float l, float q, float m) { return q == kScanCut ? l : m + (l - q * m); }
__device__ __forceinline__ float2 scan_apply(float4 r, float2 m)
{
    return make_float2(scan_apply(r.x, r.z, m.x), scan_apply(r.y, r.w, m.y));
}
// ... and two runs, the second one behind the first
__device__ __forceinline__ void scan_join(float &l, float &q, float l2, float q2)
{
    const bool cut = q == kScanCut || q2 == kScanCut;
    l = scan_apply(l2, q2, l);
    q = cut ? kScanCut : q + q2 * (1.0f - q);
}
// The same of the gradient: e -> R + P e.  P = 0: it does not come through; a product too small for a number is not yet a cut.
__device__ __forceinline__ float2 scan_back(float4 r, float2 e)
{
    return make_float2(r.z == 0.0f ? r.x : fmaf(r.z, e.x, r.x), r.w == 0.0f ? r.y : fmaf(r.w, e.y, r.y));
}
constexpr float kScanLeast = 1.2e-38f;
__device__ __forceinline__ float scan_through(float p, float q) { return p == 0.0f || q == 0.0f ? 0.0f : fmaxf(p * q, kScanLeast); }

// A warp hands a state on to the next one: written to that warp's place, then the two meet at its barrier.
__device__ __forceinline__ void scan_hand_on(float2 *place, int warp, int lane, float2 v)
{
    place[warp * 32 + lane] = v;
    asm volatile("bar.arrive %0, 64;" ::"r"(1 + warp) : "memory");
}
__device__ __forceinline__ float2 scan_take_over(const float2 *place, int warp, int lane)
{
    asm volatile("bar.sync %0, 64;" ::"r"(1 + warp) : "memory");
    return place[warp * 32 + lane];
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
            if (n > 0) v.x = kScanLog2e * scan_param(p.bias, p.bias_type, c);
            if (n > 1) v.y = kScanLog2e * scan_param(p.bias, p.bias_type, c + 1);
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

__device__ __forceinline__ void scan_copy(uint32_t dst, const void *src, int bytes, int size)  // what is missing becomes zeros
{
    if (size == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(__cvta_generic_to_global(src)), "r"(bytes) : "memory");
    else if (size == 8)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(__cvta_generic_to_global(src)), "r"(bytes) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(__cvta_generic_to_global(src)), "r"(bytes) : "memory");
}

// A warp's own ring in shared memory: two stages with a run's rows of OPS operands each.
template <typename T, int OPS>
struct ScanRing {
    typedef typename Channels<T>::Raw Raw;
    static constexpr int kRow = kScanGroup * (int)sizeof(T), kTileBytes = kRun * kRow, kStage = OPS * kTileBytes, kBytes = 2 * kStage;
    uint32_t base;
    int lane, stage;
    __device__ __forceinline__ ScanRing(unsigned char *smem, int warp, int lane_) : base(smem_addr(smem) + warp * kBytes), lane(lane_), stage(0) {}
    // the rows of a run from step t on; rows outside [0, len) are not read, they become zeros
    __device__ __forceinline__ void fetch(int op, const ScanParams &p, const ScanView &v, int seq, const ScanPlace &at, int t, int len) const
    {
        const uint32_t to = base + stage * kStage + op * kTileBytes;
        const T *src = (const T *)v.p + seq * v.seq;
        if (p.wide) {
            constexpr int kPieces = kRow / 16, kRows = 32 / kPieces, V = 16 / (int)sizeof(T);
            const int row = lane / kPieces, c = (at.c - 2 * lane) + lane % kPieces * V;
            const int bytes = min(max(p.width - c, 0), V) * (int)sizeof(T);
            const T *q = src + (long long)(t + row) * v.step + c;
            const uint32_t dst = to + lane * 16;
            const long long down = kRows * v.step;
#pragma unroll
            for (int j = 0; j < kRun / kRows; ++j, q += down) {
                const bool there = t + row + j * kRows >= 0 && t + row + j * kRows < len && bytes > 0 &&
                                   RSDGC_IN_BOUNDS(seq < p.n_seq && len <= p.n_steps && c + bytes / (int)sizeof(T) <= p.width);
                scan_copy(dst + j * 512, there ? (const void *)q : v.p, there ? bytes : 0, 16);
            }
            return;
        }
        src += (long long)t * v.step + at.c;
        const uint32_t dst = to + lane * 2 * (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < kRun; ++i, src += v.step) {
            const bool there = t + i >= 0 && t + i < len && at.n > 0 &&
                               RSDGC_IN_BOUNDS(seq < p.n_seq && len <= p.n_steps && at.c + at.n <= p.width);
            if (p.vec) {  // (the address is used for nothing where nothing is there, but has to be one)
                scan_copy(dst + i * kRow, there ? (const void *)src : v.p, there ? at.n * (int)sizeof(T) : 0, 2 * (int)sizeof(T));
            } else if constexpr (sizeof(T) == 4) {
                scan_copy(dst + i * kRow, there ? (const void *)src : v.p, there ? 4 : 0, 4);
                scan_copy(dst + i * kRow + 4, there && at.n > 1 ? (const void *)(src + 1) : v.p, there && at.n > 1 ? 4 : 0, 4);
            } else {
                Raw r = Channels<T>::none();
                if (there) r = Channels<T>::load(src, false, at.n);
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst + i * kRow), "r"(r) : "memory");
            }
        }
    }
    __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); stage ^= 1; }
    // the older of two stages has arrived
    __device__ __forceinline__ void wait() const
    {
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();
    }
    __device__ __forceinline__ Raw read(int op, int i) const
    {
        const uint32_t from = base + stage * kStage + op * kTileBytes + i * kRow + lane * 2 * (int)sizeof(T);
        if constexpr (sizeof(T) == 4) {
            Raw r;
            asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(r.x), "=f"(r.y) : "r"(from) : "memory");
            return r;
        } else {
            Raw r;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r) : "r"(from) : "memory");
            return r;
        }
    }
};
// ... and back, negated
template <typename T>
__device__ __forceinline__ void scan_write(const float2 (&m)[kRun], const ScanParams &p, const ScanView &v, int seq,
                                           const ScanPlace &at, int t, int len)
{
    T *dst = (T *)const_cast<void *>(v.p) + seq * v.seq + t * v.step + at.c;
    if (at.pair && t + kRun <= len && RSDGC_IN_BOUNDS(t >= 0 && seq < p.n_seq && len <= p.n_steps && at.c + 2 <= p.width)) {
        const uint32_t step = (uint32_t)v.step;
#pragma unroll
        for (int i = 0; i < kRun; ++i)
            Channels<T>::store(dst + (unsigned long long)step * i, true, 2, make_float2(-m[i].x, -m[i].y));
    } else {
#pragma unroll
        for (int i = 0; i < kRun; ++i, dst += v.step)
            if (t + i < len && RSDGC_IN_BOUNDS(t >= 0 && seq < p.n_seq && len <= p.n_steps))
                Channels<T>::store(dst, at.pair, at.n, make_float2(-m[i].x, -m[i].y));
    }
}

// Whether step t + lane starts a text
__device__ __forceinline__ bool scan_restarts(const ScanParams &p, int seq, int t, int len, int lane)
{
    return p.restart && lane < kRun && t + lane >= 0 && t + lane < len && p.restart[seq * p.restart_stride + t + lane] != 0;
}

// -b of a run's steps; steps that do not exist leave the state as it is
template <typename T, int OPS>
__device__ __forceinline__ void scan_gates(float2 (&nb)[kRun], const ScanRing<T, OPS> &ring, int op, float2 bias, int t, int len)
{
    const float2 scale = make_float2(kScanLog2e, kScanLog2e);
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        const float2 u = fma2(Channels<T>::widen(ring.read(op, i)), scale, bias);
        nb[i] = make_float2(scan_gate(u.x), scan_gate(u.y));
    }
    if (t < 0 || t + kRun > len) {
#pragma unroll
        for (int i = 0; i < kRun; ++i)
            if (t + i < 0 || t + i >= len) nb[i] = make_float2(0.0f, 0.0f);
    }
}
// The run from the negated state m, which each step's y = -x replaces
__device__ __forceinline__ void scan_steps(float2 (&x)[kRun], const float2 (&nb)[kRun], float2 &m, uint32_t restart)
{
    if (!restart) {
#pragma unroll
        for (int i = 0; i < kRun; ++i) x[i] = m = fma2(nb[i], add2(x[i], m), m);
    } else {
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            if (restart >> i & 1) m = make_float2(0.0f, 0.0f);
            x[i] = m = fma2(nb[i], add2(x[i], m), m);
        }
    }
}
__device__ __forceinline__ void scan_save(const ScanParams &p, int seq, const ScanPlace &at, int t, float2 m)
{
    if (p.states && RSDGC_IN_BOUNDS(t / kRun < p.runs && seq < p.n_seq))
        scan_store2(p.states + ((long long)seq * p.runs + t / kRun) * p.width + at.c, at.n, make_float2(-m.x, -m.y));
}

// ---- forward --------------------------------------------------------------------------------------
// The chain: W warps of a CTA take a sequence's runs in turn, all but the recurrence side by side; the state is handed from
// warp to warp.  W = 1: kScanLoneWarps warps with a sequence's group each.
template <typename T, int W>
__global__ void __launch_bounds__(W == 1 ? 32 * kScanLoneWarps : 32 * W) k_scan_forward(const ScanParams p)
{
    __shared__ float2 place[W][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, run = W == 1 ? 0 : warp;
    const int unit = W == 1 ? blockIdx.x * kScanLoneWarps + warp : (int)blockIdx.x;
    grid_dependency_wait();
    grid_dependency_launch_next();
    const int seq = unit / p.groups, group = unit - seq * p.groups;
    if (seq >= p.n_seq) return;  // W = 1 only: a warp too many
    const ScanPlace at(p, group, lane);
    const float2 bias = at.bias(p);
    const int len = scan_length(p, seq);
    float2 m = make_float2(0.0f, 0.0f);  // the state, negated: m + nb (x + m) needs no other negation
    if (p.first && run == 0) {
        m = scan_load2(p.first + (long long)seq * p.width + at.c, at.n);
        m = make_float2(-m.x, -m.y);
    }
    if (len == 0 && run == 0 && p.last) scan_store2(p.last + (long long)seq * p.width + at.c, at.n, make_float2(-m.x, -m.y));
    int t = run * kRun;
    extern __shared__ __align__(16) unsigned char smem[];
    ScanRing<T, 2> ring(smem, warp, lane);
    auto fetch = [&](int at_step) {
        if (at_step < len) {
            ring.fetch(0, p, p.x, seq, at, at_step, len);
            ring.fetch(1, p, p.gate, seq, at, at_step, len);
        }
        ring.commit();
    };
    fetch(t);
    fetch(t + W * kRun);
    bool starts = scan_restarts(p, seq, t, len, lane);
    for (; t < len; t += W * kRun) {
        float2 x[kRun], nb[kRun];
        const uint32_t restart = __ballot_sync(0xFFFFFFFFu, starts);
        ring.wait();
        scan_gates(nb, ring, 1, bias, t, len);
#pragma unroll
        for (int i = 0; i < kRun; ++i) x[i] = Channels<T>::widen(ring.read(0, i));
        __syncwarp();
        fetch(t + 2 * W * kRun);
        starts = scan_restarts(p, seq, t + W * kRun, len, lane);
        if (W > 1 && t > 0) m = scan_take_over(&place[0][0], warp, lane);
        scan_save(p, seq, at, t, m);
        scan_steps(x, nb, m, restart);
        if (t + kRun >= len) {
            if (p.last) scan_store2(p.last + (long long)seq * p.width + at.c, at.n, make_float2(-m.x, -m.y));
        } else if (W > 1) {
            scan_hand_on(&place[0][0], warp + 1 < W ? warp + 1 : 0, lane, m);
        }
        scan_write<T>(x, p, p.y, seq, at, t, len);
    }
}

// Few channels and many steps: W warps of each of p.cluster CTAs take W runs each side by side, from no state; what they do to a
// state is told to all of them, and each starts again from the state that it then knows.
template <typename T, int W>
__global__ void __launch_bounds__(32 * W) k_scan_forward_split(const ScanParams p)
{
    __shared__ float4 runs[2][W][32];              // by round: what each warp's run does
    __shared__ float4 parts[2][kScanCluster][32];  // ... and each CTA's W runs
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cluster = p.cluster, rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int unit = (int)blockIdx.x / cluster;
    grid_dependency_wait();
    grid_dependency_launch_next();
    const int seq = unit / p.groups, group = unit - seq * p.groups;
    if (cluster > 1) cluster_sync_all();  // nothing is written to a CTA that has not begun
    const ScanPlace at(p, group, lane);
    const float2 bias = at.bias(p);
    const int len = scan_length(p, seq), stride = W * kRun * cluster;
    float2 m = make_float2(0.0f, 0.0f);  // the negated state that comes into the round
    if (p.first) {
        m = scan_load2(p.first + (long long)seq * p.width + at.c, at.n);
        m = make_float2(-m.x, -m.y);
    }
    int t = (rank * W + warp) * kRun, parity = 0;
    extern __shared__ __align__(16) unsigned char smem[];
    ScanRing<T, 2> ring(smem, warp, lane);
    auto fetch = [&](int at_step) {
        if (at_step < len) {
            ring.fetch(0, p, p.x, seq, at, at_step, len);
            ring.fetch(1, p, p.gate, seq, at, at_step, len);
        }
        ring.commit();
    };
    fetch(t);
    fetch(t + stride);
    bool starts = scan_restarts(p, seq, t, len, lane);
    for (int t0 = 0; t0 < len; t0 += stride, t += stride, parity ^= 1) {
        float2 x[kRun], nb[kRun];
        const uint32_t restart = __ballot_sync(0xFFFFFFFFu, starts);
        ring.wait();
        scan_gates(nb, ring, 1, bias, t, len);
#pragma unroll
        for (int i = 0; i < kRun; ++i) x[i] = t < len ? Channels<T>::widen(ring.read(0, i)) : make_float2(0.0f, 0.0f);
        __syncwarp();
        fetch(t + 2 * stride);
        starts = scan_restarts(p, seq, t + stride, len, lane);
        float2 l = make_float2(0.0f, 0.0f), nq = l, r = make_float2(1.0f, 1.0f);  // r = 1 - q, of its own digits
        if (!restart) {
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                l = fma2(nb[i], add2(x[i], l), l);
                nq = fma2(nb[i], r, nq);
                r = fma2(nb[i], r, r);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                if (restart >> i & 1) l = make_float2(0.0f, 0.0f);
                l = fma2(nb[i], add2(x[i], l), l);
            }
            nq = make_float2(-kScanCut, -kScanCut);
        }
        runs[parity][warp][lane] = make_float4(l.x, l.y, -nq.x, -nq.y);
        __syncthreads();
        float2 in = m;
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
                if (k == rank) in = m;
                m = scan_apply(parts[parity][k][lane], m);
            }
            for (int w = 0; w < warp; ++w) in = scan_apply(runs[parity][w][lane], in);
        } else {
            for (int w = 0; w < W; ++w) {
                if (w == warp) in = m;
                m = scan_apply(runs[parity][w][lane], m);
            }
        }
        if (t >= len) continue;
        scan_save(p, seq, at, t, in);
        scan_steps(x, nb, in, restart);
        scan_write<T>(x, p, p.y, seq, at, t, len);
    }
    if (p.last && rank == 0 && warp == 0)
        scan_store2(p.last + (long long)seq * p.width + at.c, at.n, make_float2(-m.x, -m.y));
}

// ---- backward -------------------------------------------------------------------------------------
// A run's operands on their way through the ring, the state before it and its restarts in registers
template <typename T>
struct ScanBack {
    ScanRing<T, 3> ring;
    float2 from;
    bool starts;
    __device__ __forceinline__ void rows(const ScanParams &p, int seq, const ScanPlace &at, int t, int len)
    {
        if (t >= 0 && t < len) {
            ring.fetch(0, p, p.x, seq, at, t, len);
            ring.fetch(1, p, p.gate, seq, at, t, len);
            ring.fetch(2, p, p.y, seq, at, t, len);
        }
        ring.commit();
    }
    __device__ __forceinline__ void state(const ScanParams &p, int seq, const ScanPlace &at, int t, int len, int lane)
    {
        starts = scan_restarts(p, seq, t, len, lane);
        from = make_float2(0.0f, 0.0f);
        if (t >= 0 && t < len && RSDGC_IN_BOUNDS(t / kRun < p.runs && seq < p.n_seq))
            from = scan_load2(p.states + ((long long)seq * p.runs + t / kRun) * p.width + at.c, at.n);
    }
    // the run's -b, x and dy; the place is filled again with the run after the next
    __device__ __forceinline__ void take(float2 (&nb)[kRun], float2 (&x)[kRun], float2 (&dy)[kRun], float2 bias, const ScanParams &p,
                                         int seq, const ScanPlace &at, int t, int len, int ahead)
    {
        const bool there = t >= 0 && t < len;
        ring.wait();
        scan_gates(nb, ring, 1, bias, t, len);
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            x[i] = there ? Channels<T>::widen(ring.read(0, i)) : make_float2(0.0f, 0.0f);
            dy[i] = there ? Channels<T>::widen(ring.read(2, i)) : make_float2(0.0f, 0.0f);
        }
        __syncwarp();
        rows(p, seq, at, t - 2 * ahead, len);
    }
};
// x becomes x_t - h_{t-1}, from the state before the run
__device__ __forceinline__ void scan_again(float2 (&x)[kRun], const float2 (&nb)[kRun], float2 from, uint32_t restart)
{
    float2 m = make_float2(-from.x, -from.y);
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        if (restart >> i & 1) m = make_float2(0.0f, 0.0f);
        x[i] = add2(x[i], m);
        m = fma2(nb[i], x[i], m);
    }
}
// dy becomes delta; e: the gradient from behind, and at the end the one that goes on
__device__ __forceinline__ void scan_deltas(float2 (&dy)[kRun], const float2 (&nb)[kRun], float2 &e, uint32_t restart)
{
#pragma unroll
    for (int i = kRun - 1; i >= 0; --i) {
        dy[i] = add2(dy[i], e);
        e = fma2(nb[i], dy[i], dy[i]);
        if (restart >> i & 1) e = make_float2(0.0f, 0.0f);
    }
}
// dx and dgate of a run; adds up dgate
template <typename T>
__device__ __forceinline__ void scan_gradients(float2 (&x)[kRun], float2 (&dy)[kRun], const float2 (&nb)[kRun], float2 &sum, float2 &rest,
                                               const ScanParams &p, int seq, const ScanPlace &at, int t, int len)
{
    float2 add = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        const float2 d = dy[i];
        dy[i] = mul2(nb[i], d);                              // -dx
        x[i] = mul2(mul2(add2(d, dy[i]), nb[i]), x[i]);      // a d (-b) (x - h): dgate
        add = add2(add, x[i]);
        x[i] = make_float2(-x[i].x, -x[i].y);
    }
    if (p.dx.p) scan_write<T>(dy, p, p.dx, seq, at, t, len);
    if (p.dgate.p) scan_write<T>(x, p, p.dgate, seq, at, t, len);
    // Kahan's sum: a channel may have millions of steps
    const float2 y = make_float2(add.x - rest.x, add.y - rest.y), s = make_float2(sum.x + y.x, sum.y + y.y);
    rest = make_float2((s.x - sum.x) - y.x, (s.y - sum.y) - y.y);
    sum = s;
}
// The warps' sums of dgate to the workspace
template <int W>
__device__ __forceinline__ void scan_sums(float2 *place, float2 sum, const ScanParams &p, const ScanPlace &at, int slot, int warp, int lane)
{
    if (!p.partial) return;
    if (W > 1) {
        __syncthreads();
        place[warp * 32 + lane] = sum;
        __syncthreads();
        if (warp) return;
        for (int w = 1; w < W; ++w) sum = add2(sum, place[w * 32 + lane]);
    }
    if (RSDGC_IN_BOUNDS(slot < p.seq_parts * p.cluster)) scan_store2(p.partial + (long long)slot * p.width + at.c, at.n, sum);
}

// The chain, the last run first.  A run's states are computed again from the one saved before it.
template <typename T, int W>
__global__ void __launch_bounds__(W == 1 ? 32 * kScanLoneWarps : 32 * W) k_scan_backward(const ScanParams p)
{
    __shared__ float2 place[W][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, run = W == 1 ? 0 : warp;
    const int unit = W == 1 ? blockIdx.x * kScanLoneWarps + warp : (int)blockIdx.x;
    grid_dependency_wait();
    grid_dependency_launch_next();
    const int part = unit / p.groups, group = unit - part * p.groups;
    if (part >= p.seq_parts) return;  // W = 1 only: a warp too many
    const ScanPlace at(p, group, lane);
    const float2 bias = at.bias(p);
    float2 sum = make_float2(0.0f, 0.0f), rest = sum;  // of dgate, with what the sum's rounding left out
    extern __shared__ __align__(16) unsigned char smem[];
    ScanBack<T> next = {ScanRing<T, 3>(smem, warp, lane), sum, false};
    for (int seq = part; seq < p.n_seq; seq += p.seq_parts) {
        const int len = scan_length(p, seq), runs = (len + kRun - 1) / kRun;
        float2 e = make_float2(0.0f, 0.0f);
        if (p.first && run == 0) e = scan_load2(p.first + (long long)seq * p.width + at.c, at.n);
        if (len == 0 && run == 0 && p.last) scan_store2(p.last + (long long)seq * p.width + at.c, at.n, e);
        int t = (runs - 1 - run) * kRun;
        next.rows(p, seq, at, t, len);
        next.rows(p, seq, at, t - W * kRun, len);
        next.state(p, seq, at, t, len, lane);
        for (; t >= 0; t -= W * kRun) {
            float2 x[kRun], nb[kRun], dy[kRun];
            const uint32_t restart = __ballot_sync(0xFFFFFFFFu, next.starts);
            const float2 from = next.from;
            next.take(nb, x, dy, bias, p, seq, at, t, len, W * kRun);
            next.state(p, seq, at, t - W * kRun, len, lane);
            scan_again(x, nb, from, restart);
            if (W > 1 && t + kRun < len) e = scan_take_over(&place[0][0], warp, lane);
            scan_deltas(dy, nb, e, restart);
            if (t == 0) {
                if (p.last) scan_store2(p.last + (long long)seq * p.width + at.c, at.n, e);
            } else if (W > 1) {
                scan_hand_on(&place[0][0], warp + 1 < W ? warp + 1 : 0, lane, e);
            }
            scan_gradients<T>(x, dy, nb, sum, rest, p, seq, at, t, len);
        }
        if (W > 1) __syncthreads();  // the next sequence's first run waits for no one: the places are to be free
    }
    scan_sums<W>(&place[0][0], sum, p, at, part, run, lane);
}

// Few channels and many steps, as forward: what a run does to the gradient that comes into it from behind is e -> R + P e, P the
// product of its a.
template <typename T, int W>
__global__ void __launch_bounds__(32 * W) k_scan_backward_split(const ScanParams p)
{
    __shared__ float4 runs[2][W][32];              // (R, P) of the two channels
    __shared__ float4 parts[2][kScanCluster][32];  // ... of a CTA's W runs
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cluster = p.cluster, rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int unit = (int)blockIdx.x / cluster;
    grid_dependency_wait();
    grid_dependency_launch_next();
    const int part = unit / p.groups, group = unit - part * p.groups;
    if (cluster > 1) cluster_sync_all();  // nothing is written to a CTA that has not begun
    const ScanPlace at(p, group, lane);
    const float2 bias = at.bias(p);
    constexpr int tile = W * kRun;
    float2 sum = make_float2(0.0f, 0.0f), rest = sum;
    extern __shared__ __align__(16) unsigned char smem[];
    ScanBack<T> next = {ScanRing<T, 3>(smem, warp, lane), sum, false};
    int parity = 0;
    for (int seq = part; seq < p.n_seq; seq += p.seq_parts) {
        const int len = scan_length(p, seq), tiles = (len + tile - 1) / tile;
        float2 e = make_float2(0.0f, 0.0f);  // the gradient that comes into the round from behind
        if (p.first) e = scan_load2(p.first + (long long)seq * p.width + at.c, at.n);
        int t = (tiles - 1 - rank) * tile + warp * kRun;
        next.rows(p, seq, at, t, len);
        next.rows(p, seq, at, t - tile * cluster, len);
        next.state(p, seq, at, t, len, lane);
        for (int left = tiles; left > 0; left -= cluster, t -= tile * cluster, parity ^= 1) {
            float2 x[kRun], nb[kRun], dy[kRun];
            const uint32_t restart = __ballot_sync(0xFFFFFFFFu, next.starts);
            const float2 from = next.from;
            next.take(nb, x, dy, bias, p, seq, at, t, len, tile * cluster);
            next.state(p, seq, at, t - tile * cluster, len, lane);
            float2 r = make_float2(0.0f, 0.0f), q = make_float2(1.0f, 1.0f);
#pragma unroll
            for (int i = kRun - 1; i >= 0; --i) {
                const float2 d = add2(dy[i], r);
                r = fma2(nb[i], d, d);
                q = fma2(nb[i], q, q);
                if (restart >> i & 1) r = make_float2(0.0f, 0.0f);
            }
            q = restart ? make_float2(0.0f, 0.0f) : make_float2(fmaxf(q.x, kScanLeast), fmaxf(q.y, kScanLeast));
            runs[parity][warp][lane] = make_float4(r.x, r.y, q.x, q.y);
            __syncthreads();
            float2 in = e;
            if (cluster > 1) {
                if (warp < cluster) {
                    float2 all = make_float2(0.0f, 0.0f), k = make_float2(1.0f, 1.0f);
                    for (int w = W - 1; w >= 0; --w) {
                        const float4 o = runs[parity][w][lane];
                        all = scan_back(o, all);
                        k = make_float2(scan_through(k.x, o.z), scan_through(k.y, o.w));
                    }
                    for (int to = warp; to < cluster; to += W)
                        scan_store_in(smem_addr(&parts[parity][rank][lane]), (uint32_t)to, make_float4(all.x, all.y, k.x, k.y));
                }
                cluster_sync_all();
                for (int k = 0; k < cluster; ++k) {
                    if (k == rank) in = e;
                    e = scan_back(parts[parity][k][lane], e);
                }
                for (int w = W - 1; w > warp; --w) in = scan_back(runs[parity][w][lane], in);
            } else {
                for (int w = W - 1; w >= 0; --w) {
                    if (w == warp) in = e;
                    e = scan_back(runs[parity][w][lane], e);
                }
            }
            if (t < 0 || t >= len) continue;
            scan_again(x, nb, from, restart);
            scan_deltas(dy, nb, in, restart);
            scan_gradients<T>(x, dy, nb, sum, rest, p, seq, at, t, len);
        }
        if (p.last && rank == 0 && warp == 0) scan_store2(p.last + (long long)seq * p.width + at.c, at.n, e);
    }
    scan_sums<W>(reinterpret_cast<float2 *>(&runs[0][0][0]), sum, p, at, part * cluster + rank, warp, lane);
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
#ifndef SCAN_WARPS_F
#define SCAN_WARPS_F 16
#define SCAN_WARPS_B 12
#define SCAN_SPLIT 6
#endif
constexpr int64_t kScanParts = 16 * kScanSms;  // sequence groups from which on the backward pass gives a warp several

int scan_check(int64_t n, int64_t t, int64_t d)
{
    if (n < 0 || t < 0 || d < 1) return RSDGC_ERR_INVALID;
    if (n > (1 << 30) || t > (1 << 30) || d > (1 << 24)) return RSDGC_ERR_CAPACITY;
    const int64_t groups = (d + kScanGroup - 1) / kScanGroup;
    return n * groups > INT_MAX / kScanCluster ? RSDGC_ERR_CAPACITY : RSDGC_OK;
}

inline int scan_groups(int64_t d) { return (int)((d + kScanGroup - 1) / kScanGroup); }
inline int scan_runs(int64_t t) { return (int)((t + kRun - 1) / kRun); }

// How a call's sequences' groups (units) are dealt: warps of a CTA that form a chain, or CTAs of a cluster that split the steps.
struct ScanShape {
    int warps, cluster;
    bool split;
};
ScanShape scan_shape(int64_t units, int64_t steps, int per_sm, int elem)
{
    const int64_t runs = scan_runs(steps);
    const int wide = elem == 4 ? 8 : 16;
    if (units * 12 < (int64_t)kScanSms * SCAN_SPLIT && runs > 2 * wide) {
        int k = 1;
        while (k < kScanCluster && units * 2 * k <= kScanSms && runs > 2 * k * wide) k *= 2;
        return {wide, k, true};
    }
    int warps = 1;
    for (int w : {2, 4, 8, 12})
        if (units * w <= (int64_t)kScanSms * per_sm && runs >= w && (elem < 4 || w <= 8)) warps = w;
    return {warps, 1, false};
}

int64_t scan_seq_parts(int64_t n, int64_t d)
{
    const int64_t most = kScanParts / scan_groups(d) > 1 ? kScanParts / scan_groups(d) : 1;
    return n < most ? n : most;
}
ScanShape scan_backward_shape(int64_t n, int64_t t, int64_t d, int elem)
{
    return scan_shape(scan_seq_parts(n, d) * scan_groups(d), t, SCAN_WARPS_B, elem);
}

bool scan_pairs(const ScanView &v, int elem)
{
    return pointer_aligned(v.p, 2 * elem) && v.seq % 2 == 0 && v.step % 2 == 0 && v.step >> 32 == 0;
}

bool scan_wide(const ScanView &v, int elem)
{
    return pointer_aligned(v.p, 16) && v.seq * elem % 16 == 0 && v.step * elem % 16 == 0;
}

template <typename F>
cudaError_t scan_type(int dtype, F f)
{
    return dtype == RSDGC_F32 ? f(float{}) : dtype == RSDGC_BF16 ? f(__nv_bfloat16{}) : f(__half{});
}

// Launches a kernel with `bytes` of ring per warp; what the device has to be told before is told once per device.
template <typename K>
cudaError_t scan_launch(K kernel, std::atomic<uint64_t> &ready, unsigned grid, int warps, int bytes, int cluster, cudaStream_t s,
                        const ScanParams &p)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (warps * bytes > (40 << 10) && !(ready.load(std::memory_order_acquire) >> (dev & 63) & 1)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, warps * bytes);
        if (e != cudaSuccess) return e;
        ready.fetch_or(1ull << (dev & 63), std::memory_order_release);
    }
    return launch_chained(kernel, grid, 32 * warps, (size_t)warps * bytes, s, cluster, p);
}
#define SCAN_LAUNCH(kernel, grid, warps, cluster)                                                          \
    [&] {                                                                                                  \
        static std::atomic<uint64_t> ready{0};                                                             \
        return scan_launch(kernel, ready, (unsigned)(grid), warps, bytes, cluster, s, p);                  \
    }()

template <typename T>
cudaError_t scan_forward(ScanParams &p, cudaStream_t s)
{
    const long long units = (long long)p.n_seq * p.groups;
    const ScanShape shape = scan_shape(units, p.n_steps, SCAN_WARPS_F, sizeof(T));
    constexpr int bytes = ScanRing<T, 2>::kBytes, wide = sizeof(T) == 4 ? 8 : 16;
    p.cluster = shape.cluster;
    if (shape.split) return SCAN_LAUNCH((k_scan_forward_split<T, wide>), units * shape.cluster, wide, shape.cluster);
    switch (shape.warps) {
    case 1: return SCAN_LAUNCH((k_scan_forward<T, 1>), (units + kScanLoneWarps - 1) / kScanLoneWarps, kScanLoneWarps, 1);
    case 2: return SCAN_LAUNCH((k_scan_forward<T, 2>), units, 2, 1);
    case 4: return SCAN_LAUNCH((k_scan_forward<T, 4>), units, 4, 1);
    case 8: return SCAN_LAUNCH((k_scan_forward<T, 8>), units, 8, 1);
    }
    if constexpr (sizeof(T) < 4) return SCAN_LAUNCH((k_scan_forward<T, 12>), units, 12, 1);
    return cudaErrorInvalidValue;
}

template <typename T>
cudaError_t scan_backward(ScanParams &p, cudaStream_t s)
{
    const long long units = (long long)p.seq_parts * p.groups;
    const ScanShape shape = scan_backward_shape(p.n_seq, p.n_steps, p.width, sizeof(T));
    constexpr int bytes = ScanRing<T, 3>::kBytes, wide = sizeof(T) == 4 ? 8 : 16;
    p.cluster = shape.cluster;
    if (shape.split) return SCAN_LAUNCH((k_scan_backward_split<T, wide>), units * shape.cluster, wide, shape.cluster);
    switch (shape.warps) {
    case 1: return SCAN_LAUNCH((k_scan_backward<T, 1>), (units + kScanLoneWarps - 1) / kScanLoneWarps, kScanLoneWarps, 1);
    case 2: return SCAN_LAUNCH((k_scan_backward<T, 2>), units, 2, 1);
    case 4: return SCAN_LAUNCH((k_scan_backward<T, 4>), units, 4, 1);
    case 8: return SCAN_LAUNCH((k_scan_backward<T, 8>), units, 8, 1);
    }
    if constexpr (sizeof(T) < 4) return SCAN_LAUNCH((k_scan_backward<T, 12>), units, 12, 1);
    return cudaErrorInvalidValue;
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
    if (rc) return rc;
    // the same for every type: the wider rows split sooner
    const int a = scan_backward_shape(n_seq, n_steps, width, 2).cluster, b = scan_backward_shape(n_seq, n_steps, width, 4).cluster;
    return 4 * width * scan_seq_parts(n_seq, width) * (a > b ? a : b);
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
    p.runs = scan_runs(n_steps);
    p.vec = scan_pairs(p.x, elem) && scan_pairs(p.gate, elem) && scan_pairs(p.y, elem);
    p.wide = scan_wide(p.x, elem) && scan_wide(p.gate, elem);
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
    p.runs = scan_runs(n_steps);
    p.seq_parts = (int)scan_seq_parts(n_seq, width);
    p.vec = scan_pairs(p.x, elem) && scan_pairs(p.gate, elem) && scan_pairs(p.y, elem) && (!dx_dev || scan_pairs(p.dx, elem)) &&
            (!dgate_dev || scan_pairs(p.dgate, elem));
    p.wide = scan_wide(p.x, elem) && scan_wide(p.gate, elem) && scan_wide(p.y, elem);
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
