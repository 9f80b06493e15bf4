// Gated scan: a recurrence over a sequence's steps, channel by channel, forward and backward.
//
//   a_t = 1 / (1 + exp(-(gate_t + bias))),  b_t = 1 - a_t,  h_t = a_t h_{t-1} + b_t x_t,  y_t = h_t
//   delta_t = dy_t + a_{t+1} delta_{t+1},  dx_t = b_t delta_t,  dgate_t = delta_t a_t b_t (h_{t-1} - x_t)
//
// The step is affine in the state, and so is a run of steps: h -> L + P h = h + (L - Q h), P the product of its a, Q = 1 - P, which is how runs are
// computed side by side and joined.  Of a and b the smaller one is formed to its own digits, and a step adds it, times a difference, to what it
// is near to: h + b (x - h) where the gate is open, x + a (h - x) where it is nearly closed.  A slow channel (b of 1e-5) keeps its digits,
// which a, next to 1, would round away, and so does what a closed gate (a of 1e-6) lets through of the state and of the gradient.
//
// A warp takes 64 channels (two a lane) and runs of 16 steps; the next two runs' rows are on their way through its own ring in shared
// memory while a run is computed.  Three ways to deal the runs, by how many (sequence, 64 channels) units there are:
//  - every warp walks a unit of its own (W = 1);
//  - a CTA's W warps take a unit's runs in turn and hand the state on from warp to warp.  With W = 8 and 12 the critical path is not a run's 16
//    steps but one step of its (L, Q), which the warp has formed beforehand: 4 x 8192 x 2048 bfloat16, 128 units: 113 us without, 80 us with;
//  - few units: the CTAs of a cluster take W runs each side by side, tell one another what those do to a state, and each run starts from
//    the state that follows (1 x 65536 x 1024 binary16: 534 us with one CTA a unit, 180 us with 7).
// Runs are joined in the order of time, whoever is first: results are the same bits from call to call.
// Rows that do not start on 16-byte boundaries arrive in 16-byte pieces too, one more a row, and are shifted when they are read
// (8 x 4096 x 2047 bfloat16: 137 us forward, 594 us with loads of single values).
//
// What bounds it: memory where there are units for all multiprocessors (8 x 4096 x 4096 bfloat16: 154 us forward, 5.2 TB/s; 257 us
// backward, 5.2 TB/s), the instructions of a run on the units' multiprocessors where there are not.
#include <atomic>
#include <climits>
#include <mutex>
#include <type_traits>

#include "device_utils.cuh"
#include "operators_internal.cuh"
#include "tensor_core.cuh"

namespace rsdgc {

constexpr int kScanGroup = 64;      // channels of a warp
constexpr int kRun = RSDGC_SCAN_STATE_STEPS;  // steps of a run
constexpr int kScanCluster = 8;     // most CTAs that share a sequence's group
constexpr int kScanLoneWarps = 4;   // of a CTA whose warps walk alone

constexpr int kScanAhead = 8;       // chains of so many warps and more hand a state on before they compute their run's steps

// Warps of a multiprocessor that the registers are cut for.  Few with many registers do better than many with few: backward with
// 8 warps 257 us, with 12 warps 294 us, with 16 379 us, with 6 424 us (8 x 4096 x 4096 bfloat16); a chain of 12 has a multiprocessor to itself.
template <typename T>
constexpr int scan_forward_warps(int w) { return sizeof(T) == 4 || w == 12 ? 12 : 16; }
template <typename T>
constexpr int scan_backward_warps(int w) { return w == 12 ? 12 : 8; }

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
    int vec, wide;                  // results: pairs of channels may be written at once; operands: rows start on 16-byte boundaries
};

// The cluster's barrier in two halves: what lies between them needs nothing of the other CTAs (1 x 65536 x 2048 bfloat16: 358 us with the
// copies' issue and the CTA's own joins before it, 262 us with them between)
__device__ __forceinline__ void scan_cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void scan_cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void scan_store_in(uint32_t addr, uint32_t rank, float4 v)  // to a CTA of the cluster
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr_in(addr, rank)), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// Two neighbouring channels as they lie in memory.  `pair`: one access; otherwise `n` of the two values are there.
template <typename T>
struct Channels {
    typedef uint32_t Raw;
    static __device__ __forceinline__ Raw none() { return 0u; }
    static __device__ __forceinline__ float2 widen(Raw r)
    {
        T v[2];
        *reinterpret_cast<uint32_t *>(v) = r;
        return make_float2(to_f32(v[0]), to_f32(v[1]));
    }
    static __device__ __forceinline__ Raw narrow(float2 v) { return pack2<T>(v.x, v.y); }
    static __device__ __forceinline__ Raw least(Raw a, Raw b)  // of each channel; NaN only of two
    {
        Raw r;
        if constexpr (std::is_same_v<T, __half>)
            asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else
            asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ void store(T *p, bool pair, int n, Raw r)
    {
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
    static __device__ __forceinline__ Raw none() { return make_float2(0.0f, 0.0f); }
    static __device__ __forceinline__ float2 widen(Raw r) { return r; }
    static __device__ __forceinline__ Raw narrow(float2 v) { return v; }
    static __device__ __forceinline__ Raw least(Raw a, Raw b) { return make_float2(fminf(a.x, b.x), fminf(a.y, b.y)); }
    static __device__ __forceinline__ void store(float *p, bool pair, int n, Raw v)
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

__device__ __forceinline__ bool scan_negative(float v) { return __float_as_int(v) < 0; }  // by the sign bit

// A step's coefficient c, from u = z log2(e), by whether some gate of the warp's run is nearly closed (u < kScanShut, a < 1/33).  Where none
// is (SHUT false), c = -b = -1 / (1 + exp(z)), and 1 - b has a to 2^-17 of itself.  Where one is, the smaller one of a and b, to its own digits,
// and which one its sign bit tells: -b where the gate is open (z > 0), a = exp(z) / (1 + exp(z)) where it is not.  That costs a selection a channel
// in each use: with selections in every run 4 x 8192 x 2048 bfloat16 takes 104 us, 80 us so, backward 213 and 136 us.  c never leaves
// [-1, 1/2], whatever u is; NaN stays NaN.
constexpr float kScanShut = -5.0f;
constexpr float kScanStays = -0.0f;  // the coefficient of a step that does not exist: b = 0
template <bool SHUT>
__device__ __forceinline__ float scan_gate(float u)
{
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(SHUT ? -fabsf(u) : u));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(SHUT ? 1.0f + e : -1.0f - e));
    return SHUT ? __uint_as_float(__float_as_uint(e * r) | (~__float_as_uint(u) & 0x80000000u)) : r;
}
__device__ __forceinline__ float2 scan_by_gate(float2 c, float2 open, float2 closed)
{
    return make_float2(scan_negative(c.x) ? open.x : closed.x, scan_negative(c.y) ? open.y : closed.y);
}
// The step from the negated state m; u = x - h, the state before it
template <bool SHUT>
__device__ __forceinline__ float2 scan_step(float2 c, float2 x, float2 m, float2 &u)
{
    u = add2(x, m);
    return fma2(c, u, SHUT ? scan_by_gate(c, m, make_float2(-x.x, -x.y)) : m);
}
// a v
template <bool SHUT>
__device__ __forceinline__ float2 scan_keep(float2 c, float2 v)
{
    return fma2(c, v, SHUT ? scan_by_gate(c, v, make_float2(0.0f, 0.0f)) : v);
}
// -b
template <bool SHUT>
__device__ __forceinline__ float2 scan_take(float2 c)
{
    return SHUT ? add2(c, scan_by_gate(c, make_float2(0.0f, 0.0f), make_float2(-1.0f, -1.0f))) : c;
}

// What a run does to the (negated) state that comes into it, as (L, S): m -> m + (L - Q m) with S = Q where Q is at most 1/2, m -> L + P m with S = -P
// (sign bit set) where P = 1 - Q is: of P and Q the smaller one, to its own digits.  So neither a slow channel's state nor what is left behind
// a large one is rounded away (a token of 1e6 among ordinary ones left 6 % of a unit with Q alone).  S = kScanCut: the state does not come through.
constexpr float kScanCut = 2.0f;
__device__ __forceinline__ float scan_apply(float l, float s, float m)
{
    return s == kScanCut ? l : (scan_negative(s) ? 0.0f : m) + fmaf(-s, m, l);
}
__device__ __forceinline__ float2 scan_apply(float4 r, float2 m)
{
    return make_float2(scan_apply(r.x, r.z, m.x), scan_apply(r.y, r.w, m.y));
}
// ... as it is formed: m -> L + P m.  P's sign bit: the state does not come through.  Q has its own digits where P is above 1/2.
struct ScanRun {
    float2 l, p, q;
    static __device__ __forceinline__ float which(float p, float q) { return scan_negative(p) ? kScanCut : p > 0.5f ? q : -p; }
    __device__ __forceinline__ float4 packed() const { return make_float4(l.x, l.y, which(p.x, q.x), which(p.y, q.y)); }
    // This run and one behind it.  L + P L' will do: what it rounds away is not carried on beyond the joined runs.
    __device__ __forceinline__ void join(const ScanRun &r)
    {
        l = fma2(r.p, l, r.l);
        if (scan_negative(r.p.x)) l.x = r.l.x;
        if (scan_negative(r.p.y)) l.y = r.l.y;
        q = fma2(r.q, p, q);
        p = mul2(p, r.p);
    }
};
// The same of the gradient: e -> R + P e.  P = 0: it does not come through; a product too small for a number is not yet a cut.
__device__ __forceinline__ float2 scan_back(float4 r, float2 e)
{
    return make_float2(r.z == 0.0f ? r.x : fmaf(r.z, e.x, r.x), r.w == 0.0f ? r.y : fmaf(r.w, e.y, r.y));
}
constexpr float kScanLeast = 1.2e-38f;
__device__ __forceinline__ float scan_through(float p, float q) { return p == 0.0f || q == 0.0f ? 0.0f : fmaxf(p * q, kScanLeast); }

// A warp hands a state on to the next one: written to that warp's place, then the two meet at its barrier.
template <int W>
__device__ __forceinline__ void scan_hand_on(float2 *place, int warp, int lane, float2 v)
{
    place[warp * 32 + lane] = v;
    if constexpr (W == 2) {  // constants: with a number from a register a CTA holds all sixteen, of a multiprocessor's 64
        if (warp)
            asm volatile("bar.arrive 2, 64;" ::: "memory");
        else
            asm volatile("bar.arrive 1, 64;" ::: "memory");
    } else {
        asm volatile("bar.arrive %0, 64;" ::"r"(1 + warp) : "memory");
    }
}
template <int W>
__device__ __forceinline__ float2 scan_take_over(const float2 *place, int warp, int lane)
{
    if constexpr (W == 2) {
        if (warp)
            asm volatile("bar.sync 2, 64;" ::: "memory");
        else
            asm volatile("bar.sync 1, 64;" ::: "memory");
    } else {
        asm volatile("bar.sync %0, 64;" ::"r"(1 + warp) : "memory");
    }
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

__device__ __forceinline__ void scan_copy(uint32_t dst, const void *src, int bytes)  // 16 bytes; what is missing becomes zeros
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(__cvta_generic_to_global(src)), "r"(bytes) : "memory");
}

// A warp's own ring in shared memory: two stages with a run's rows of OPS operands each.  Rows arrive in pieces of 16 bytes.  SHIFT: they need not
// start on such a boundary; a row then has one piece more, and its values lie as far into the first one as they do in memory.
template <typename T, int OPS, bool SHIFT>
struct ScanRing {
    typedef typename Channels<T>::Raw Raw;
    static constexpr int kRow = kScanGroup * (int)sizeof(T) + (SHIFT ? 16 : 0), kTileBytes = kRun * kRow, kStage = OPS * kTileBytes,
                         kBytes = 2 * kStage;
    uint32_t base;
    int lane, stage;
    uint32_t first[SHIFT ? OPS : 1], down[SHIFT ? OPS : 1];  // where a run's first row lies in its piece, and how far on the next one
    __device__ __forceinline__ ScanRing(unsigned char *smem, int warp, int lane_) : base(smem_addr(smem) + warp * kBytes), lane(lane_), stage(0) {}
    // ... of a sequence: runs start at multiples of 16 steps, so all of them lie alike
    __device__ __forceinline__ void start(int op, const ScanView &v, int seq, const ScanPlace &at)
    {
        if constexpr (SHIFT) {
            first[op] = (uint32_t)(uintptr_t)((const T *)v.p + seq * v.seq + (at.c - 2 * lane)) & 15u;
            down[op] = (uint32_t)(v.step * (int)sizeof(T)) & 15u;
        }
    }
    // the rows of a run from step t on; rows outside [0, len) are not read, they become zeros
    __device__ __forceinline__ void fetch(int op, const ScanParams &p, const ScanView &v, int seq, const ScanPlace &at, int t, int len) const
    {
        const uint32_t to = base + stage * kStage + op * kTileBytes;
        const T *src = (const T *)v.p + seq * v.seq;
        constexpr int kPieces = kRow / 16, V = 16 / (int)sizeof(T);
        if constexpr (!SHIFT) {
            constexpr int kRows = 32 / kPieces;
            const int row = lane / kPieces, c = (at.c - 2 * lane) + lane % kPieces * V;
            const int bytes = min(max(p.width - c, 0), V) * (int)sizeof(T);
            const T *q = src + (long long)(t + row) * v.step + c;
            const uint32_t dst = to + lane * 16;
            const long long down = kRows * v.step;
#pragma unroll
            for (int j = 0; j < kRun / kRows; ++j, q += down) {
                const bool there = t + row + j * kRows >= 0 && t + row + j * kRows < len && bytes > 0 &&
                                   RSDGC_IN_BOUNDS(seq < p.n_seq && len <= p.n_steps && c + bytes / (int)sizeof(T) <= p.width);
                scan_copy(dst + j * 512, there ? (const void *)q : v.p, there ? bytes : 0);
            }
        } else {
            const int c = at.c - 2 * lane, here = min(max(p.width - c, 0), kScanGroup) * (int)sizeof(T);
            const long long pitch = v.step * (long long)sizeof(T);
            const char *const row0 = reinterpret_cast<const char *>(src + (long long)t * v.step + c);
            const bool inside = here > 0 && RSDGC_IN_BOUNDS(seq < p.n_seq && len <= p.n_steps && c + here / (int)sizeof(T) <= p.width);
            if (row0 - 15 < (const char *)v.p) {
                // a first piece may begin before the operand: its values one by one (what lies before any other row is the operand's)
                for (int i = lane; i < kRun * kScanGroup; i += 32) {
                    const int row = i / kScanGroup, at_byte = i % kScanGroup * (int)sizeof(T);
                    const bool there = t + row >= 0 && t + row < len && at_byte < here && inside;
                    const char *const q = row0 + row * pitch + at_byte;
                    const uint32_t dst = to + row * kRow + ((first[op] + row * down[op]) & 15u) + at_byte;
                    if constexpr (sizeof(T) == 4)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(dst), "f"(there ? *(const float *)q : 0.0f) : "memory");
                    else
                        asm volatile("st.shared.u16 [%0], %1;" ::"r"(dst), "h"(there ? *(const unsigned short *)q : (unsigned short)0)
                                     : "memory");
                }
                return;
            }
            // the rows' last pieces in a round of their own
            constexpr int kMost = kPieces - 1, kRows = 32 / kMost;
            auto copy = [&](const char *row_at, int row, int piece) {
                const uint32_t in = (uint32_t)(uintptr_t)row_at & 15u;
                const int bytes = t + row >= 0 && t + row < len && inside ? min(max((int)in + here - 16 * piece, 0), 16) : 0;
                const char *const q = row_at - in + 16 * piece;
                scan_copy(to + row * kRow + 16 * piece, bytes ? q : reinterpret_cast<const char *>((uintptr_t)v.p & ~(uintptr_t)15), bytes);
            };
            const char *row_at = row0 + lane / kMost * pitch;
#pragma unroll
            for (int j = 0; j < kRun / kRows; ++j, row_at += kRows * pitch) copy(row_at, j * kRows + lane / kMost, lane % kMost);
            if (lane < kRun) copy(row0 + lane * pitch, lane, kMost);
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
        uint32_t from = base + stage * kStage + op * kTileBytes + i * kRow + lane * 2 * (int)sizeof(T);
        if constexpr (SHIFT) from += (first[op] + i * down[op]) & 15u;
        Raw r;
        if constexpr (sizeof(T) == 4) {
            if constexpr (SHIFT) {
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(r.x) : "r"(from) : "memory");
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(r.y) : "r"(from + 4) : "memory");
            } else {
                asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(r.x), "=f"(r.y) : "r"(from) : "memory");
            }
        } else if constexpr (SHIFT) {
            asm volatile("{\n\t.reg .b16 a, b;\n\tld.shared.b16 a, [%1];\n\tld.shared.b16 b, [%1 + 2];\n\tmov.b32 %0, {a, b};\n\t}"
                         : "=r"(r)
                         : "r"(from)
                         : "memory");
        } else {
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r) : "r"(from) : "memory");
        }
        return r;
    }
};
// A run's rows of a result from step t on
template <typename T>
__device__ __forceinline__ void scan_write(const typename Channels<T>::Raw (&v)[kRun], const ScanParams &p, const ScanView &to, int seq,
                                           const ScanPlace &at, int t, int len)
{
    T *dst = (T *)const_cast<void *>(to.p) + seq * to.seq + t * to.step + at.c;
    if (at.pair && t + kRun <= len && RSDGC_IN_BOUNDS(t >= 0 && seq < p.n_seq && len <= p.n_steps && at.c + 2 <= p.width)) {
        const uint32_t step = (uint32_t)to.step;  // pairs: below 2^32
#pragma unroll
        for (int i = 0; i < kRun; ++i) Channels<T>::store(dst + (unsigned long long)step * i, true, 2, v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kRun; ++i, dst += to.step)
            if (t + i < len && RSDGC_IN_BOUNDS(t >= 0 && seq < p.n_seq && len <= p.n_steps))
                Channels<T>::store(dst, at.pair, at.n, v[i]);
    }
}

// Whether step t + lane starts a text
__device__ __forceinline__ bool scan_restarts(const ScanParams &p, int seq, int t, int len, int lane)
{
    return p.restart && lane < kRun && t + lane >= 0 && t + lane < len && p.restart[seq * p.restart_stride + t + lane] != 0;
}

// The coefficients of a run's steps; steps that do not exist leave the state as it is.  Returns, the same for the whole warp, whether a gate of
// the run is nearly closed.
template <bool SHUT, typename T, int OPS, bool SHIFT>
__device__ __forceinline__ bool scan_gates(float2 (&c)[kRun], const ScanRing<T, OPS, SHIFT> &ring, int op, float2 bias, int t, int len)
{
    const float2 scale = make_float2(kScanLog2e, kScanLog2e);
    typename Channels<T>::Raw least;
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        const typename Channels<T>::Raw gate = ring.read(op, i);
        const float2 u = fma2(Channels<T>::widen(gate), scale, bias);
        c[i] = make_float2(scan_gate<SHUT>(u.x), scan_gate<SHUT>(u.y));
        least = i ? Channels<T>::least(least, gate) : gate;
    }
    if (t < 0 || t + kRun > len) {
#pragma unroll
        for (int i = 0; i < kRun; ++i)
            if (t + i < 0 || t + i >= len) c[i] = make_float2(kScanStays, kScanStays);
    }
    const float2 low = fma2(Channels<T>::widen(least), scale, bias);
    return SHUT || __any_sync(0xFFFFFFFFu, fminf(low.x, low.y) < kScanShut);
}
// The run from the negated state m; y = -m, in the operand's type, replaces each step's x
template <bool SHUT, typename T>
__device__ __forceinline__ void scan_steps(typename Channels<T>::Raw (&x)[kRun], const float2 (&c)[kRun], float2 &m, uint32_t restart)
{
    float2 u;
    if (!SHUT && !restart) {
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            m = scan_step<SHUT>(c[i], Channels<T>::widen(x[i]), m, u);
            x[i] = Channels<T>::narrow(make_float2(-m.x, -m.y));
        }
    } else {
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            if (restart >> i & 1) m = make_float2(0.0f, 0.0f);
            m = scan_step<SHUT>(c[i], Channels<T>::widen(x[i]), m, u);
            x[i] = Channels<T>::narrow(make_float2(-m.x, -m.y));
        }
    }
}
// What the run does to a state
template <bool SHUT, typename T>
__device__ __forceinline__ ScanRun scan_whole(const typename Channels<T>::Raw (&x)[kRun], const float2 (&c)[kRun], uint32_t restart)
{
    float2 l = make_float2(0.0f, 0.0f), p = make_float2(-0.0f, -0.0f), nq = p, u;
    if (!restart) {
        // P to its own digits; so is Q while all gates are open, and where one is not, P is at most 1/2
        p = make_float2(1.0f, 1.0f);
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            l = scan_step<SHUT>(c[i], Channels<T>::widen(x[i]), l, u);
            nq = fma2(c[i], p, nq);
            p = scan_keep<SHUT>(c[i], p);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            if (restart >> i & 1) l = make_float2(0.0f, 0.0f);
            l = scan_step<SHUT>(c[i], Channels<T>::widen(x[i]), l, u);
        }
    }
    return {l, p, make_float2(-nq.x, -nq.y)};
}
__device__ __forceinline__ void scan_save(const ScanParams &p, int seq, const ScanPlace &at, int t, float2 m)
{
    if (p.states && RSDGC_IN_BOUNDS(t / kRun < p.runs && seq < p.n_seq))
        scan_store2(p.states + ((long long)seq * p.runs + t / kRun) * p.width + at.c, at.n, make_float2(-m.x, -m.y));
}

// ---- forward --------------------------------------------------------------------------------------
// The chain: W warps of a CTA take a sequence's runs in turn, all but the recurrence side by side; the state is handed from
// warp to warp.  W = 1: kScanLoneWarps warps with a sequence's group each.
template <typename T, int W, bool SHIFT>
__global__ void __launch_bounds__(W == 1 ? 32 * kScanLoneWarps : 32 * W, scan_forward_warps<T>(W) / (W == 1 ? kScanLoneWarps : W)) k_scan_forward(const ScanParams p)
{
    constexpr bool ahead = W >= kScanAhead;
    __shared__ float2 place[W][32];
    __shared__ float4 whole[ahead ? W : 1][32];  // kept here so that it is there before the state is waited for
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
    ScanRing<T, 2, SHIFT> ring(smem, warp, lane);
    ring.start(0, p.x, seq, at);
    ring.start(1, p.gate, seq, at);
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
        typename Channels<T>::Raw x[kRun];
        float2 c[kRun];
        const uint32_t restart = __ballot_sync(0xFFFFFFFFu, starts);
        ring.wait();
        const bool shut = scan_gates<false>(c, ring, 1, bias, t, len);
        if (shut) scan_gates<true>(c, ring, 1, bias, t, len);
#pragma unroll
        for (int i = 0; i < kRun; ++i) x[i] = ring.read(0, i);
        __syncwarp();
        fetch(t + 2 * W * kRun);
        starts = scan_restarts(p, seq, t + W * kRun, len, lane);
        auto walk = [&](auto is_shut) {
            constexpr bool SHUT = decltype(is_shut)::value;
            if constexpr (ahead) whole[warp][lane] = scan_whole<SHUT, T>(x, c, restart).packed();
            if (W > 1 && t > 0) m = scan_take_over<W>(&place[0][0], warp, lane);
            if constexpr (ahead)
                if (t + kRun < len) scan_hand_on<W>(&place[0][0], warp + 1 < W ? warp + 1 : 0, lane, scan_apply(whole[warp][lane], m));
            scan_save(p, seq, at, t, m);
            scan_steps<SHUT, T>(x, c, m, restart);
            if (t + kRun >= len) {
                if (p.last) scan_store2(p.last + (long long)seq * p.width + at.c, at.n, make_float2(-m.x, -m.y));
            } else if (W > 1 && !ahead) {
                scan_hand_on<W>(&place[0][0], warp + 1 < W ? warp + 1 : 0, lane, m);
            }
        };
        if (shut)
            walk(std::true_type());
        else
            walk(std::false_type());
        scan_write<T>(x, p, p.y, seq, at, t, len);
    }
}

// Few channels and many steps: W warps of each of p.cluster CTAs take W runs each side by side, from no state; what they do to a
// state is told to all of them, and each starts again from the state that it then knows.
template <typename T, int W, bool SHIFT>
__global__ void __launch_bounds__(32 * W) k_scan_forward_split(const ScanParams p)
{
    __shared__ ScanRun runs[2][W][32];             // by round: what each warp's run does
    __shared__ float4 parts[2][kScanCluster][32];  // ... and each CTA's W runs
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cluster = p.cluster, rank = (int)cluster_rank();
    const int unit = (int)blockIdx.x / cluster;
    grid_dependency_wait();
    grid_dependency_launch_next();
    const int seq = unit / p.groups, group = unit - seq * p.groups;
    cluster_sync_all();  // nothing is written to a CTA that has not begun
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
    ScanRing<T, 2, SHIFT> ring(smem, warp, lane);
    ring.start(0, p.x, seq, at);
    ring.start(1, p.gate, seq, at);
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
    auto next_rows = [&] {  // into the places just read
        __syncwarp();
        fetch(t + 2 * stride);
        starts = scan_restarts(p, seq, t + stride, len, lane);
    };
    for (int t0 = 0; t0 < len; t0 += stride, t += stride, parity ^= 1) {
        typename Channels<T>::Raw x[kRun];
        float2 c[kRun];
        const uint32_t restart = __ballot_sync(0xFFFFFFFFu, starts);
        ring.wait();
        const bool shut = scan_gates<false>(c, ring, 1, bias, t, len);
        if (shut) scan_gates<true>(c, ring, 1, bias, t, len);
#pragma unroll
        for (int i = 0; i < kRun; ++i) x[i] = t < len ? ring.read(0, i) : Channels<T>::none();
        runs[parity][warp][lane] = shut ? scan_whole<true, T>(x, c, restart) : scan_whole<false, T>(x, c, restart);
        __syncthreads();
        float2 in = m;
        // warp k tells CTA k what this CTA's runs do
        if (warp < cluster) {
            ScanRun all = runs[parity][0][lane];
            for (int w = 1; w < W; ++w) all.join(runs[parity][w][lane]);
            for (int k = warp; k < cluster; k += W) scan_store_in(smem_addr(&parts[parity][rank][lane]), (uint32_t)k, all.packed());
        }
        scan_cluster_arrive();
        next_rows();
        ScanRun before = {make_float2(0.0f, 0.0f), make_float2(1.0f, 1.0f), make_float2(0.0f, 0.0f)};  // what this CTA's runs before this one do
        for (int w = 0; w < warp; ++w) before.join(runs[parity][w][lane]);
        scan_cluster_wait();
        for (int k = 0; k < cluster; ++k) {
            if (k == rank) in = m;
            m = scan_apply(parts[parity][k][lane], m);
        }
        in = scan_apply(before.packed(), in);
        if (t >= len) continue;
        scan_save(p, seq, at, t, in);
        shut ? scan_steps<true, T>(x, c, in, restart) : scan_steps<false, T>(x, c, in, restart);
        scan_write<T>(x, p, p.y, seq, at, t, len);
    }
    if (p.last && rank == 0 && warp == 0)
        scan_store2(p.last + (long long)seq * p.width + at.c, at.n, make_float2(-m.x, -m.y));
}

// ---- backward -------------------------------------------------------------------------------------
// A run's operands on their way through the ring, the state before it and its restarts in registers
template <typename T, bool SHIFT>
struct ScanBack {
    typedef typename Channels<T>::Raw Raw;
    ScanRing<T, 3, SHIFT> ring;
    float2 from;
    bool starts;
    __device__ __forceinline__ void start(const ScanParams &p, int seq, const ScanPlace &at)
    {
        ring.start(0, p.x, seq, at);
        ring.start(1, p.gate, seq, at);
        ring.start(2, p.y, seq, at);
    }
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
    // the run's x and dy
    __device__ __forceinline__ void operands(Raw (&x)[kRun], Raw (&dy)[kRun], int t, int len) const
    {
        const bool there = t >= 0 && t < len;
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            x[i] = there ? ring.read(0, i) : Channels<T>::none();
            dy[i] = there ? ring.read(2, i) : Channels<T>::none();
        }
    }
    // ... and its coefficients; returns whether a gate is nearly closed
    __device__ __forceinline__ bool take(float2 (&c)[kRun], Raw (&x)[kRun], Raw (&dy)[kRun], float2 bias, int t, int len) const
    {
        ring.wait();
        const bool shut = scan_gates<false>(c, ring, 1, bias, t, len);
        operands(x, dy, t, len);
        return shut;
    }
    // ... whose place is filled with the run after the next
    __device__ __forceinline__ void refill(const ScanParams &p, int seq, const ScanPlace &at, int t, int len, int ahead)
    {
        __syncwarp();
        rows(p, seq, at, t - 2 * ahead, len);
    }
};
// What the run does to the gradient that comes into it from behind
template <bool SHUT, typename T>
__device__ __forceinline__ float4 scan_back_whole(const typename Channels<T>::Raw (&dy)[kRun], const float2 (&c)[kRun], uint32_t restart)
{
    float2 r = make_float2(0.0f, 0.0f), q = make_float2(1.0f, 1.0f);
#pragma unroll
    for (int i = kRun - 1; i >= 0; --i) {
        r = scan_keep<SHUT>(c[i], add2(Channels<T>::widen(dy[i]), r));
        q = scan_keep<SHUT>(c[i], q);
        if (restart >> i & 1) r = make_float2(0.0f, 0.0f);
    }
    q = restart ? make_float2(0.0f, 0.0f) : make_float2(fmaxf(q.x, kScanLeast), fmaxf(q.y, kScanLeast));
    return make_float4(r.x, r.y, q.x, q.y);
}
// u_t = x_t - h_{t-1}, from the state before the run
template <bool SHUT, typename T>
__device__ __forceinline__ void scan_again(float2 (&u)[kRun], const typename Channels<T>::Raw (&x)[kRun], const float2 (&c)[kRun],
                                           float2 from, uint32_t restart)
{
    float2 m = make_float2(-from.x, -from.y);
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        if (restart >> i & 1) m = make_float2(0.0f, 0.0f);
        m = scan_step<SHUT>(c[i], Channels<T>::widen(x[i]), m, u[i]);
    }
}
// From the last step to the first: delta, dx, dgate (into dy's and x's places) and dgate's sum.  e: the gradient from behind, and at the
// end the one that goes on.
template <bool SHUT, typename T>
__device__ __forceinline__ void scan_deltas(typename Channels<T>::Raw (&dy)[kRun], typename Channels<T>::Raw (&x)[kRun],
                                            const float2 (&u)[kRun], const float2 (&c)[kRun], float2 &e, float2 &add, uint32_t restart)
{
    add = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = kRun - 1; i >= 0; --i) {
        const float2 d = add2(Channels<T>::widen(dy[i]), e), nb = scan_take<SHUT>(c[i]);
        e = scan_keep<SHUT>(c[i], d);              // a delta
        const float2 z = mul2(mul2(e, nb), u[i]);  // a delta (-b) (x - h)
        const float2 ndx = mul2(nb, d);
        dy[i] = Channels<T>::narrow(make_float2(-ndx.x, -ndx.y));
        x[i] = Channels<T>::narrow(z);
        add = add2(add, z);
        if (restart >> i & 1) e = make_float2(0.0f, 0.0f);
    }
}
// Kahan's sum: a channel may have millions of steps
__device__ __forceinline__ void scan_sum(float2 &sum, float2 &rest, float2 add)
{
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
template <typename T, int W, bool SHIFT>
__global__ void __launch_bounds__(W == 1 ? 32 * kScanLoneWarps : 32 * W, scan_backward_warps<T>(W) / (W == 1 ? kScanLoneWarps : W)) k_scan_backward(const ScanParams p)
{
    constexpr bool ahead = W >= kScanAhead;
    __shared__ float2 place[W][32];
    __shared__ float4 whole[ahead ? W : 1][32];
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
    ScanBack<T, SHIFT> next = {ScanRing<T, 3, SHIFT>(smem, warp, lane), sum, false};
    // chains have one sequence: there are more only where the warps that walk alone fill the device several times
    for (int seq = part; seq < p.n_seq; seq += W == 1 ? p.seq_parts : p.n_seq) {
        const int len = scan_length(p, seq), runs = (len + kRun - 1) / kRun;
        float2 e = make_float2(0.0f, 0.0f);
        if (p.first && run == 0) e = scan_load2(p.first + (long long)seq * p.width + at.c, at.n);
        if (len == 0 && run == 0 && p.last) scan_store2(p.last + (long long)seq * p.width + at.c, at.n, e);
        int t = (runs - 1 - run) * kRun;
        next.start(p, seq, at);
        next.rows(p, seq, at, t, len);
        next.rows(p, seq, at, t - W * kRun, len);
        next.state(p, seq, at, t, len, lane);
        for (; t >= 0; t -= W * kRun) {
            typename Channels<T>::Raw x[kRun], dy[kRun];
            float2 c[kRun], u[kRun], add;
            const uint32_t restart = __ballot_sync(0xFFFFFFFFu, next.starts);
            const float2 from = next.from;
            const bool shut = next.take(c, x, dy, bias, t, len);
            if (!shut) next.refill(p, seq, at, t, len, W * kRun);
            next.state(p, seq, at, t - W * kRun, len, lane);
            // a run with a nearly closed gate is computed again, with selections, and its rows stay until then
            scan_again<false, T>(u, x, c, from, restart);
            if constexpr (ahead) whole[warp][lane] = scan_back_whole<false, T>(dy, c, restart);
            if (shut) {
                scan_gates<true>(c, next.ring, 1, bias, t, len);
                scan_again<true, T>(u, x, c, from, restart);
                if constexpr (ahead) whole[warp][lane] = scan_back_whole<true, T>(dy, c, restart);
            }
            if (W > 1 && t + kRun < len) e = scan_take_over<W>(&place[0][0], warp, lane);
            if constexpr (ahead)
                if (t > 0) scan_hand_on<W>(&place[0][0], warp + 1 < W ? warp + 1 : 0, lane, scan_back(whole[warp][lane], e));
            const float2 behind = e;
            scan_deltas<false, T>(dy, x, u, c, e, add, restart);
            if (shut) {
                next.operands(x, dy, t, len);
                e = behind;
                scan_deltas<true, T>(dy, x, u, c, e, add, restart);
                next.refill(p, seq, at, t, len, W * kRun);
            }
            if (t == 0) {
                if (p.last) scan_store2(p.last + (long long)seq * p.width + at.c, at.n, e);
            } else if (W > 1 && !ahead) {
                scan_hand_on<W>(&place[0][0], warp + 1 < W ? warp + 1 : 0, lane, e);
            }
            if (p.dx.p) scan_write<T>(dy, p, p.dx, seq, at, t, len);
            if (p.dgate.p) scan_write<T>(x, p, p.dgate, seq, at, t, len);
            scan_sum(sum, rest, add);
        }
    }
    scan_sums<W>(&place[0][0], sum, p, at, part, run, lane);
}

// Few channels and many steps, as forward: what a run does to the gradient that comes into it from behind is e -> R + P e, P the
// product of its a.
template <typename T, int W, bool SHIFT>
__global__ void __launch_bounds__(32 * W) k_scan_backward_split(const ScanParams p)
{
    __shared__ float4 runs[2][W][32];              // (R, P) of the two channels
    __shared__ float4 parts[2][kScanCluster][32];  // ... of a CTA's W runs
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cluster = p.cluster, rank = (int)cluster_rank();
    const int unit = (int)blockIdx.x / cluster;
    grid_dependency_wait();
    grid_dependency_launch_next();
    const int seq = unit / p.groups, group = unit - seq * p.groups;
    cluster_sync_all();  // nothing is written to a CTA that has not begun
    const ScanPlace at(p, group, lane);
    const float2 bias = at.bias(p);
    constexpr int tile = W * kRun;
    float2 sum = make_float2(0.0f, 0.0f), rest = sum;
    extern __shared__ __align__(16) unsigned char smem[];
    ScanBack<T, SHIFT> next = {ScanRing<T, 3, SHIFT>(smem, warp, lane), sum, false};
    int parity = 0;
    const int len = scan_length(p, seq), tiles = (len + tile - 1) / tile;
    float2 e = make_float2(0.0f, 0.0f);  // the gradient that comes into the round from behind
    if (p.first) e = scan_load2(p.first + (long long)seq * p.width + at.c, at.n);
    int t = (tiles - 1 - rank) * tile + warp * kRun;
    next.start(p, seq, at);
    next.rows(p, seq, at, t, len);
    next.rows(p, seq, at, t - tile * cluster, len);
    next.state(p, seq, at, t, len, lane);
    for (int left = tiles; left > 0; left -= cluster, t -= tile * cluster, parity ^= 1) {
        typename Channels<T>::Raw x[kRun], dy[kRun];
        float2 c[kRun], u[kRun], add;
        const uint32_t restart = __ballot_sync(0xFFFFFFFFu, next.starts);
        const float2 from = next.from;
        const bool shut = next.take(c, x, dy, bias, t, len);
        if (shut) scan_gates<true>(c, next.ring, 1, bias, t, len);
        runs[parity][warp][lane] = shut ? scan_back_whole<true, T>(dy, c, restart) : scan_back_whole<false, T>(dy, c, restart);
        __syncthreads();
        float2 in = e;
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
        scan_cluster_arrive();
        next.refill(p, seq, at, t, len, tile * cluster);
        next.state(p, seq, at, t - tile * cluster, len, lane);
        float4 behind = make_float4(0.0f, 0.0f, 1.0f, 1.0f);  // what this CTA's runs behind this one do
        for (int w = W - 1; w > warp; --w) {
            const float4 o = runs[parity][w][lane];
            const float2 r = scan_back(o, make_float2(behind.x, behind.y));
            behind = make_float4(r.x, r.y, scan_through(behind.z, o.z), scan_through(behind.w, o.w));
        }
        scan_cluster_wait();
        for (int k = 0; k < cluster; ++k) {
            if (k == rank) in = e;
            e = scan_back(parts[parity][k][lane], e);
        }
        in = scan_back(behind, in);
        if (t < 0 || t >= len) continue;
        shut ? scan_again<true, T>(u, x, c, from, restart) : scan_again<false, T>(u, x, c, from, restart);
        shut ? scan_deltas<true, T>(dy, x, u, c, in, add, restart) : scan_deltas<false, T>(dy, x, u, c, in, add, restart);
        if (p.dx.p) scan_write<T>(dy, p, p.dx, seq, at, t, len);
        if (p.dgate.p) scan_write<T>(x, p, p.dgate, seq, at, t, len);
        scan_sum(sum, rest, add);
    }
    if (p.last && rank == 0 && warp == 0) scan_store2(p.last + (long long)seq * p.width + at.c, at.n, e);
    scan_sums<W>(reinterpret_cast<float2 *>(&runs[0][0][0]), sum, p, at, seq * cluster + rank, warp, lane);
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

// The longest chain of warps per CTA, of at most `most`, with which all units are on the device at a time
template <typename F>
int scan_warps(int64_t units, int64_t steps, int most, F per_sm)
{
    int warps = 1;
    for (int w : {2, 4, 8, 12})
        if (w <= most && units * w <= (int64_t)kScanSms * per_sm(w) && scan_runs(steps) >= w) warps = w;
    return warps;
}
// Most CTAs that may share a unit's steps
int scan_most_cluster(int64_t units)
{
    const int64_t k = units > 0 ? kScanSms / units : 1;
    return k > kScanCluster ? kScanCluster : k < 1 ? 1 : (int)k;
}

int64_t scan_seq_parts(int64_t n, int64_t d)
{
    const int64_t most = kScanParts / scan_groups(d) > 1 ? kScanParts / scan_groups(d) : 1;
    return n < most ? n : most;
}
bool scan_pairs(const ScanView &v, int elem)
{
    return pointer_aligned(v.p, 2 * elem) && v.seq % 2 == 0 && v.step % 2 == 0 && v.step >> 32 == 0;
}

// The strides of what there is one of are free: they decide nothing.
void scan_free_strides(ScanView &v, int64_t n, int64_t t)
{
    if (n == 1) v.seq = 0;
    if (t == 1) v.step = 0;
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
cudaError_t scan_ready(K kernel, std::atomic<uint64_t> &ready, int bytes, int *dev)
{
    cudaError_t e = cudaGetDevice(dev);
    if (e != cudaSuccess || bytes <= (40 << 10) || (ready.load(std::memory_order_acquire) >> (*dev & 63) & 1)) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) ready.fetch_or(1ull << (*dev & 63), std::memory_order_release);
    return e;
}
// What the calling thread's latest launch took: warps of a sequence's group per CTA, CTAs of it
thread_local int scan_way_warps = 0, scan_way_ctas = 0;
void scan_took(int warps, int ctas)
{
    scan_way_warps = warps;
    scan_way_ctas = ctas;
}

template <typename K>
cudaError_t scan_launch(K kernel, std::atomic<uint64_t> &ready, unsigned grid, int chain, int bytes, cudaStream_t s, const ScanParams &p)
{
    const int warps = chain == 1 ? kScanLoneWarps : chain;
    int dev = 0;
    scan_took(chain, 1);
    const cudaError_t e = scan_ready(kernel, ready, warps * bytes, &dev);
    return e != cudaSuccess ? e : launch_chained(kernel, grid, 32 * warps, (size_t)warps * bytes, s, 1, p);
}
#define SCAN_LAUNCH(kernel, grid, chain)                                                                   \
    [&] {                                                                                                  \
        static std::atomic<uint64_t> ready{0};                                                             \
        return scan_launch(kernel, ready, (unsigned)(grid), chain, bytes, s, p);                           \
    }()

// The kernel that splits the steps, in clusters of p.cluster CTAs; *done = false if fewer than `least` would be on the device at
// a time with all units: a second wave costs more than the split gains (16 units of 65536 steps, binary16: 278 us with 8 CTAs each, of which
// 15 clusters fit, 180 us with 7).
template <typename K>
cudaError_t scan_split(K kernel, std::atomic<uint64_t> &ready, std::atomic<int> (&fit)[64][kScanCluster + 1], long long units, int warps,
                       int bytes, int least, cudaStream_t s, ScanParams &p, bool *done)
{
    *done = false;
    int k = scan_most_cluster(units);
    while (k > 1 && p.runs < 2 * k * warps) --k;
    if (k < least) return cudaSuccess;
    int dev = 0;
    cudaError_t e = scan_ready(kernel, ready, warps * bytes, &dev);
    for (; e == cudaSuccess && k >= least; --k) {
        std::atomic<int> &known = fit[dev & 63][k];
        int n = known.load(std::memory_order_relaxed);
        if (n == 0) {
            cudaLaunchConfig_t cfg{};
            cfg.gridDim = (unsigned)k * kScanSms;
            cfg.blockDim = 32 * warps;
            cfg.dynamicSmemBytes = (size_t)warps * bytes;
            cudaLaunchAttribute at{};
            at.id = cudaLaunchAttributeClusterDimension;
            at.val.clusterDim.x = k;
            at.val.clusterDim.y = at.val.clusterDim.z = 1;
            cfg.attrs = &at;
            cfg.numAttrs = 1;
            e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
            if (e != cudaSuccess) return e;
            known.store(n < 1 ? -1 : n, std::memory_order_relaxed);
        }
        if (n < units) continue;
        p.cluster = k;
        *done = true;
        scan_took(warps, k);
        return launch_chained(kernel, (unsigned)(units * k), 32 * warps, (size_t)warps * bytes, s, k, p);
    }
    return e;
}
#define SCAN_SPLIT(kernel, units, warps, least, done)                                                      \
    [&] {                                                                                                  \
        static std::atomic<uint64_t> ready{0};                                                             \
        static std::atomic<int> fit[64][kScanCluster + 1] = {};                                            \
        return scan_split(kernel, ready, fit, units, warps, bytes, least, s, p, done);                     \
    }()

template <typename T, bool SHIFT>
cudaError_t scan_forward(ScanParams &p, cudaStream_t s)
{
    const long long units = (long long)p.n_seq * p.groups;
    constexpr int bytes = ScanRing<T, 2, SHIFT>::kBytes, wide = sizeof(T) == 4 ? 8 : 16;
    p.cluster = 1;
    bool done = false;
    // Two CTAs of 8 warps, binary32's, do not make up for their joins: 2 x 8192 x 2048 104 us, 80 us with a chain of 12.  Two of 16 warps do (bfloat16
    // 72 and 78 us, 3 x 4000 x 1400 binary16 51 and 60), and so do two in the backward pass (113 and 129 us, binary32 158 and 159).
    const cudaError_t e = SCAN_SPLIT((k_scan_forward_split<T, wide, SHIFT>), units, wide, wide == 16 ? 2 : 3, &done);
    if (done || e != cudaSuccess) return e;
    switch (scan_warps(units, p.n_steps, 12, scan_forward_warps<T>)) {
    case 1: return SCAN_LAUNCH((k_scan_forward<T, 1, SHIFT>), (units + kScanLoneWarps - 1) / kScanLoneWarps, 1);
    case 2: return SCAN_LAUNCH((k_scan_forward<T, 2, SHIFT>), units, 2);
    case 4: return SCAN_LAUNCH((k_scan_forward<T, 4, SHIFT>), units, 4);
    case 8: return SCAN_LAUNCH((k_scan_forward<T, 8, SHIFT>), units, 8);
    }
    return SCAN_LAUNCH((k_scan_forward<T, 12, SHIFT>), units, 12);
}

template <typename T, bool SHIFT>
cudaError_t scan_backward(ScanParams &p, cudaStream_t s)
{
    const long long units = (long long)p.seq_parts * p.groups;
    constexpr int bytes = ScanRing<T, 3, SHIFT>::kBytes, wide = sizeof(T) == 4 ? 8 : SHIFT ? 12 : 16;  // what shared memory holds
    p.cluster = 1;
    bool done = false;
    cudaError_t e = cudaSuccess;
    if (p.seq_parts == p.n_seq) e = SCAN_SPLIT((k_scan_backward_split<T, wide, SHIFT>), units, wide, 2, &done);  // (as it is with few units)
    if (done || e != cudaSuccess) return e;
    switch (p.seq_parts < p.n_seq ? 1 : scan_warps(units, p.n_steps, sizeof(T) == 4 ? 8 : 12, scan_backward_warps<T>)) {
    case 1: return SCAN_LAUNCH((k_scan_backward<T, 1, SHIFT>), (units + kScanLoneWarps - 1) / kScanLoneWarps, 1);
    case 2: return SCAN_LAUNCH((k_scan_backward<T, 2, SHIFT>), units, 2);
    case 4: return SCAN_LAUNCH((k_scan_backward<T, 4, SHIFT>), units, 4);
    case 8: return SCAN_LAUNCH((k_scan_backward<T, 8, SHIFT>), units, 8);
    }
    if constexpr (sizeof(T) < 4) return SCAN_LAUNCH((k_scan_backward<T, 12, SHIFT>), units, 12);
    return cudaErrorInvalidValue;
}

// A strided operand: its values are aligned, the rows of a result do not overlap.
int scan_view_check(const ScanView &v, int64_t n, int64_t t, int64_t d, int elem, bool result)
{
    if (!v.p || (t > 1 && v.step < d) || (n > 1 && v.seq < d)) return RSDGC_ERR_INVALID;
    if (result && !rows_apart(n, v.seq, t, v.step, d)) return RSDGC_ERR_INVALID;
    return pointer_aligned(v.p, elem) ? RSDGC_OK : RSDGC_ERR_ALIGNMENT;
}

}  // namespace
}  // namespace rsdgc

using namespace rsdgc;

extern "C" int64_t rsdgc_gated_scan_workspace_bytes(int64_t n_seq, int64_t n_steps, int64_t width)
{
    const int rc = scan_check(n_seq, n_steps, width);
    if (rc) return rc;
    const int64_t parts = scan_seq_parts(n_seq, width);
    return 4 * width * parts * scan_most_cluster(parts * scan_groups(width));
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
            if ((rc = scan_view_check(*v, n_seq, n_steps, width, elem, v == &p.y))) return rc;
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
    for (ScanView *v : {&p.x, &p.gate, &p.y}) scan_free_strides(*v, n_seq, n_steps);
    p.vec = scan_pairs(p.y, elem);
    p.wide = scan_wide(p.x, elem) && scan_wide(p.gate, elem);
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e = operators_ready();
    if (e == cudaSuccess) e = scan_type(dtype, [&](auto t) { return p.wide ? scan_forward<decltype(t), false>(p, s) : scan_forward<decltype(t), true>(p, s); });
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
            if ((rc = scan_view_check(*v, n_seq, n_steps, width, elem, false))) return rc;
        for (const ScanView *v : {&p.dx, &p.dgate})
            if (v->p && (rc = scan_view_check(*v, n_seq, n_steps, width, elem, true))) return rc;
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
    for (ScanView *v : {&p.x, &p.gate, &p.y, &p.dx, &p.dgate}) scan_free_strides(*v, n_seq, n_steps);
    p.vec = (!dx_dev || scan_pairs(p.dx, elem)) && (!dgate_dev || scan_pairs(p.dgate, elem));
    p.wide = scan_wide(p.x, elem) && scan_wide(p.gate, elem) && scan_wide(p.y, elem);
    cudaError_t e = operators_ready();
    if (e == cudaSuccess) e = scan_type(dtype, [&](auto t) { return p.wide ? scan_backward<decltype(t), false>(p, s) : scan_backward<decltype(t), true>(p, s); });
    if (e == cudaSuccess && dbias_dev)
        e = scan_type(grad_dtype, [&](auto g) {
            typedef decltype(g) G;
            return launch_chained(k_scan_bias_gradient<G>, (unsigned)((width + 31) / 32), 256, 0, s, 1, (const float *)p.partial,
                                  p.seq_parts * p.cluster, (int)width, (G *)dbias_dev);
        });
    return operator_result(e);
}

extern "C" int rsdgc_selftest_scan_way(int32_t *warps_host, int32_t *ctas_host)
{
    if (!warps_host || !ctas_host) return RSDGC_ERR_INVALID;
    *warps_host = scan_way_warps;
    *ctas_host = scan_way_ctas;
    return RSDGC_OK;
}
