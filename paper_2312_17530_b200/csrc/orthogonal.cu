// Orthogonalised update: a matrix is brought near to one with the same singular directions and all singular values near 1, by a few
// odd polynomials of it (Newton-Schulz steps), which need products only.
//
//   Y = X / (|X|_F + eps);   A = Y Y^T,  B = b A + c A^2,  Y <- a Y + B Y   with (a, b, c) of the step;   A = Y^T Y and Y <- a Y + Y B for
//   matrices with more rows than columns, so that A has the shorter side
//
// Numbers.  The products' operands are binary16 (11 bits; bfloat16's 8 leave an error of 0.01, and 0.07 where a few directions carry the
// gradient), scaled by powers of two: Y by 2^12, A by 2^13, B by 2^13 or, where it is larger than 7.5, 2^12 or 2^11.  The host refuses
// coefficients with which Y could outgrow them.  The small directions are brought up by a, step after step, while B Y is small there: so
// Y itself is kept in two binary16 planes, the rounded value and the rest (22 bits), for a Y, which is added in binary32.  That costs
// bytes and no product (gradient of 16 directions plus 3 % noise: error 1.6e-4 with it, 9e-3 without).  A matrix whose norm is small
// beside eps begins with small singular values in all directions: its planes have a power of two more, step by step, so that they are as
// full as another's.  Where one product's 11 bits do not do - a binary16 result, small matrices - A and B have two planes too and each
// product is three: hi hi + hi lo + lo hi.
//
// The products are one tile kernel, pairs of CTAs as for the vocabulary head: TMA brings the operands through a ring, one
// thread issues the MMAs, sixteen warps empty the accumulator.  A and B are symmetric: tiles on and below the diagonal are computed, and
// written a second time across it.  Y is read as it lies, once with its rows and once with its columns contracted.  Where A has
// few tiles and a long contraction, the contraction is cut into parts which k_ortho_join adds up, in order.
//
// What bounds it.  Large matrices: the tensor cores are busy for 52 to 62 % of a product (4096 x 4096; a step of the main loop takes 1088 cycles of
// which 1024 are MMAs), the rest are the first operands' way, epilogues that nothing covers and rounds of tiles that are not full.  Small ones:
// latency (256 x 512: 143 us, 17 launches of 8 us each: 0.8 us until the first operands are there, 0.16 us a contraction step, 2.5 us of epilogue, the
// rest is a launch's; all products in one launch, whose CTAs count one another's epilogues, were 8 % faster at 256 x 512 and 9 % slower at
// 2048 x 2048: not worth its waits).  One side far longer than the other: the epilogue's memory traffic (tensor cores 26 %, 3 TB/s).
#include <climits>
#include <cmath>
#include <cstring>
#include <mutex>

#include "device_utils.cuh"
#include "operators_internal.cuh"
#include "tensor_core.cuh"

namespace rsdgc {

constexpr int kOrthoWarps = 16;                           // of the epilogue, four per quarter of an accumulator's columns
constexpr int kOrthoThreads = 128 + 32 * kOrthoWarps;     // producer, MMA, two idle warps, epilogue
constexpr int kOrthoStaging = 2048;                       // per epilogue warp: 32 rows of 64 bytes
constexpr int kOrthoSmem = kRingBlocks * kBlockBytes + kOrthoWarps * kOrthoStaging + 1024;
constexpr int kOrthoMaxSteps = 32;
constexpr float kOrthoScale = 4096.0f;                    // of Y's planes
constexpr float kOrthoScaleA = 8192.0f;                   // of A's, and of most B's
constexpr int kOrthoMostPower = 100;                      // of two that a matrix's Y may have beside its scale; what that leaves out is below 1e-30

// What becomes of a product.  kGram: A; kGramPart: binary32 parts of A; kPoly: B from A A; kSquare: a + B from the square of a shifted A;
// kUpdate: the next Y; kResult: the result.
enum { kGram = 0, kGramPart = 1, kPoly = 2, kUpdate = 3, kResult = 4, kSquare = 5 };

struct __align__(64) OrthoParams {
    CUtensorMap a, b;        // [matrix x plane][rows][columns], boxes of 64 x 64
    int a_mn, b_mn;          // the operand lies with its rows (not k) contiguous
    int a_planes, b_planes;  // stored
    int segments;            // products: hi hi, or hi hi + hi lo + lo hi
    int k_steps;             // of one of them
    int m_tiles, n_tiles, per, band;  // tiles of a matrix: per, in bands of `band` tile rows
    int symmetric;           // only tiles that reach the diagonal or lie below it
    int cols, halves;        // columns of an accumulator, accumulators of a tile
    int splits, split_steps; // parts of the contraction
    int tiles, stages;
    int rows, columns;       // of the product
    long long pitch;         // of the planes below, a multiple of 8
    float diag;              // added to the product's diagonal
    const __half *in;        // kPoly: A, kUpdate and kResult: Y; in_planes (0: none) planes of rows x pitch per matrix
    __half *out;             // out_planes planes
    int in_planes, out_planes;
    float in_scale, acc_scale;
    const float2 *powers;    // [matrix][kOrthoMaxSteps]: what the powers of two of Y, before and behind each step, make of a product's scale: A's, Y's
    int step;
    float *part;             // kGramPart: [matrix][split][rows][pitch]
    void *result;            // kResult: row and matrix stride in elements
    long long result_row, result_matrix;
    int result_wide;         // its rows lie on 16-byte boundaries
    unsigned int *status;
    unsigned polls;
};

struct OrthoTile {
    int matrix, split, m, n, k0, steps;
};
__device__ __forceinline__ OrthoTile ortho_tile(const OrthoParams &p, int t)
{
    OrthoTile r;
    const int each = p.per * p.splits;
    r.matrix = t / each;
    t -= r.matrix * each;
    r.split = t / p.per;
    t -= r.split * p.per;
    r.k0 = r.split * p.split_steps;
    r.steps = min(p.split_steps, p.segments * p.k_steps - r.k0);
    if (p.symmetric) {
        const int wide = p.cols * p.halves;
        for (r.m = 0; r.m < p.m_tiles; ++r.m) {
            const int here = min(p.n_tiles, ((r.m + 1) * kTile + wide - 1) / wide);
            if (t < here) break;
            t -= here;
        }
        r.n = t;
    } else {
        const int per = p.band * p.n_tiles, b = t / per, i = t - b * per, rows = min(p.band, p.m_tiles - b * p.band);
        r.n = i / rows;
        r.m = b * p.band + i - r.n * rows;
    }
    return r;
}

__device__ __forceinline__ void load_shared16(uint32_t addr, uint32_t &a, uint32_t &b, uint32_t &c, uint32_t &d)
{
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(addr) : "memory");
}

// A warp's 32 rows x 32 16-bit values between its lanes' rows and memory, where four lanes take a row's 64 bytes, eight rows at
// a time.  In shared memory the 16-byte piece c of row r lies at c ^ (r / 2 & 3): neither side meets a bank conflict.
struct OrthoStage {
    uint32_t buf;
    int lane;
    __device__ __forceinline__ uint32_t at(int row, int piece) const { return buf + row * 64 + ((piece ^ ((row >> 1) & 3)) << 4); }
    // this lane's four pieces of rows row0.. and columns col.. of a plane (rows x pitch values)
    __device__ __forceinline__ void fetch(uint4 (&v)[4], const __half *plane, long long pitch, int row0, int rows, int col) const
    {
        const int c = col + (lane & 3) * 8;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = row0 + j * 8 + (lane >> 2);
            v[j] = make_uint4(0, 0, 0, 0);
            if (row < rows && c < pitch && RSDGC_IN_BOUNDS(row >= 0 && c >= 0 && c + 8 <= pitch))
                v[j] = *reinterpret_cast<const uint4 *>(plane + row * pitch + c);
        }
    }
    __device__ __forceinline__ void deal(const uint4 (&v)[4]) const
    {
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 4; ++j) store_shared16(at(j * 8 + (lane >> 2), lane & 3), v[j].x, v[j].y, v[j].z, v[j].w);
        __syncwarp();
    }
    // adds scale * (this lane's row) to z
    __device__ __forceinline__ void add_row(float (&z)[32], float scale) const
    {
        const float2 s = make_float2(scale, scale);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t v[4];
            load_shared16(at(lane, i), v[0], v[1], v[2], v[3]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&v[j]));
                const float2 y = fma2(x, s, make_float2(z[8 * i + 2 * j], z[8 * i + 2 * j + 1]));
                z[8 * i + 2 * j] = y.x;
                z[8 * i + 2 * j + 1] = y.y;
            }
        }
    }
    template <typename T>
    __device__ __forceinline__ void put_row(const float (&z)[32]) const
    {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i)
            store_shared16(at(lane, i), pack2<T>(z[8 * i], z[8 * i + 1]), pack2<T>(z[8 * i + 2], z[8 * i + 3]),
                           pack2<T>(z[8 * i + 4], z[8 * i + 5]), pack2<T>(z[8 * i + 6], z[8 * i + 7]));
        __syncwarp();
    }
    // the block across the diagonal: this lane's row becomes a column
    __device__ __forceinline__ void put_column(const float (&z)[32]) const
    {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const __half h = __float2half_rn(z[i]);
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(at(i, lane >> 3) + (lane & 7) * 2), "h"(*reinterpret_cast<const uint16_t *>(&h))
                         : "memory");
        }
        __syncwarp();
    }
    __device__ __forceinline__ void store(__half *plane, long long pitch, int row0, int rows, int col) const
    {
        const int c = col + (lane & 3) * 8;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = row0 + j * 8 + (lane >> 2);
            uint4 v;
            load_shared16(at(j * 8 + (lane >> 2), lane & 3), v.x, v.y, v.z, v.w);
            if (row < rows && c < pitch && RSDGC_IN_BOUNDS(row >= 0 && c >= 0 && c + 8 <= pitch))
                *reinterpret_cast<uint4 *>(plane + row * pitch + c) = v;
        }
    }
    // 32 x 32 binary32 values, 16 columns at a time
    __device__ __forceinline__ void store_part(const float (&z)[32], float *plane, long long pitch, int row0, int rows, int col) const
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store_shared16(at(lane, i), __float_as_uint(z[16 * h + 4 * i]), __float_as_uint(z[16 * h + 4 * i + 1]),
                               __float_as_uint(z[16 * h + 4 * i + 2]), __float_as_uint(z[16 * h + 4 * i + 3]));
            __syncwarp();
            const int c = col + 16 * h + (lane & 3) * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = row0 + j * 8 + (lane >> 2);
                uint4 v;
                load_shared16(at(j * 8 + (lane >> 2), lane & 3), v.x, v.y, v.z, v.w);
                if (row < rows && c < pitch && RSDGC_IN_BOUNDS(row >= 0 && c >= 0 && c + 4 <= pitch))
                    *reinterpret_cast<uint4 *>(plane + row * pitch + c) = v;
            }
        }
    }
    // ... to the caller's matrix, which has neither padding nor alignment
    __device__ __forceinline__ void store_result(uint16_t *dst, long long stride, int row0, int rows, int col, int columns, bool wide) const
    {
        if (wide) {
            const int c = col + (lane & 3) * 8;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = row0 + j * 8 + (lane >> 2);
                uint4 v;
                load_shared16(at(j * 8 + (lane >> 2), lane & 3), v.x, v.y, v.z, v.w);
                if (row >= rows || !RSDGC_IN_BOUNDS(row >= 0 && c >= 0)) continue;
                uint16_t *q = dst + row * stride + c;
                if (c + 8 <= columns) {
                    *reinterpret_cast<uint4 *>(q) = v;
                } else {
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + i < columns) q[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
                }
            }
        } else {  // a row per round, a column per lane
            for (int r = 0; r < min(32, rows - row0); ++r) {
                uint16_t v;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at(r, lane >> 3) + (lane & 7) * 2) : "memory");
                if (col + lane < columns && RSDGC_IN_BOUNDS(row0 >= 0 && col >= 0)) dst[(row0 + r) * stride + col + lane] = v;
            }
        }
    }
};

// By a power of two, which is 1 as a rule
__device__ __forceinline__ void ortho_scale(float (&z)[32], float power)
{
    if (power != 1.0f) {
#pragma unroll
        for (int i = 0; i < 32; ++i) z[i] *= power;
    }
}
// What rounding to binary16 leaves of the values
__device__ __forceinline__ void ortho_rest(float (&z)[32])
{
#pragma unroll
    for (int i = 0; i < 32; ++i) z[i] -= __half2float(__float2half_rn(z[i]));
}

// A parameter that stays in a register: what the issuing loops need of the kernel's parameters is otherwise read anew in each round, at some
// 150 cycles a time.
template <typename V>
__device__ __forceinline__ V ortho_keep(V v)
{
    asm volatile("" : "+r"(v));
    return v;
}

// T: type of the result (kResult)
template <int KIND, typename T>
__global__ void __launch_bounds__(kOrthoThreads, 1) k_ortho(const __grid_constant__ OrthoParams p)
{
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], drain;
    __shared__ uint32_t tmem_base;
    __shared__ volatile int dead;
    // after a give-up: which CTAs had one; stages each CTA's producer issued, and its bytes in the latest of each place
    __shared__ int failed[2], issued[2], sent[2][kMaxStages];

    const uint32_t ring = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int stages = ortho_keep(p.stages), stage_bytes = ortho_keep((1 + p.halves) * kBlockBytes);
    const unsigned polls = ortho_keep(p.polls);

    if (warp == 0) {  // a lane per barrier
        if (lane < kMaxStages) {
            barrier_init(smem_addr(&full[lane]), 1);
            barrier_init(smem_addr(&empty[lane]), 1);
        } else if (lane < kMaxStages + 2) {
            barrier_init(smem_addr(&acc_full[lane - kMaxStages]), 1);
            barrier_init(smem_addr(&acc_empty[lane - kMaxStages]), 2 * kOrthoWarps);
        } else if (lane == 31) {
            barrier_init(smem_addr(&drain), 1);
            dead = 0;
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3 && lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(lane ? &p.b : &p.a) : "memory");
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_base))
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    tmem_fence_before();
    __syncthreads();
    cluster_sync_all();  // the peer's barriers exist before anything arrives on them
    tmem_fence_after();
    grid_dependency_wait();
    grid_dependency_launch_next();

    // Bounded: a wait that gives up marks the CTA dead, raises the status bit, and every role leaves its loop.
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
        if (barrier_try(bar, parity)) return true;
        for (unsigned i = 1; i < polls; ++i) {
            if (dead) return false;
            if (barrier_try(bar, parity)) return true;
        }
        dead = 1;
        atomicOr(p.status, RSDGC_STATUS_TIMEOUT);
        return false;
    };

    if (warp < 4) {
        // One thread of each of two warps walks alone: a stage of the ring is 256 to 512 cycles of MMAs, which a loop that the whole warp
        // walks, with coordinates formed and parameters read anew for each box, takes longer to issue (some 700 cycles a step; 320 so.  2048 x 2048: 425 us
        // then, 275 us with this and what else has changed since).
        if (warp == 0 && elect_one()) {  // ---- producer, in both CTAs; all bytes count on the first CTA's barriers
            int stage = 0, it = 0;
            uint32_t parity = 0, dst = ring;
            bool ok = true;
            asm volatile("fence.proxy.async.global;" ::: "memory");  // TMA reads what ordinary stores wrote
            const int halves = ortho_keep(p.halves);
            const uint32_t bytes = ortho_keep(2u * (uint32_t)(kBlockBytes + halves * p.cols * kStepK));
            const uint32_t full0 = ortho_keep(leader_addr(smem_addr(&full[0]))), empty0 = ortho_keep(smem_addr(&empty[0]));
            // coordinates of a box: (k, row), or (row, k) where the rows are contiguous: then of an operand's 128 rows in this CTA two boxes
            const int ak = ortho_keep(p.a_mn ? 0 : kStepK), bk = ortho_keep(p.b_mn ? 0 : kStepK), br = ortho_keep(p.b_mn ? 64 : 0);
            const int a_two = ortho_keep((int)p.a_mn), b_two = ortho_keep((int)(p.b_mn && p.cols == kTile));
            auto next = [&] {
                ++it;
                ++stage;
                parity ^= (uint32_t)(stage == stages);
                dst = stage == stages ? ring : dst + stage_bytes;
                stage = stage == stages ? 0 : stage;
            };
            auto announce = [&] {
                if (rank == 0) barrier_expect(smem_addr(&full[stage]), bytes);
                sent[rank][stage] = (int)(bytes / 2);
            };
            for (int t = pair; t < p.tiles && ok; t += pairs) {
                const OrthoTile tp = ortho_tile(p, t);
                const int ra = tp.m * kTile + (int)rank * kHalf, rb = tp.n * halves * p.cols + (int)rank * (p.cols >> 1);
                const int steps = ortho_keep(tp.steps);
                int seg = tp.k0 / p.k_steps, at = tp.k0 - seg * p.k_steps;
                for (int k = 0; k < steps && ok;) {
                    // the steps up to the segment's end
                    const int end = min(steps, k + p.k_steps - at), za = tp.matrix * p.a_planes + (seg == 2),
                              zb = tp.matrix * p.b_planes + (seg == 1), kc = at * kStepK;
                    int ax = p.a_mn ? ra : kc, ay = p.a_mn ? kc : ra, bx = p.b_mn ? rb : kc, by = p.b_mn ? kc : rb;
                    const bool inside = RSDGC_IN_BOUNDS(ra >= 0 && rb >= 0 && at >= 0 && ra % 64 == 0 && rb % 64 == 0 && seg < p.segments &&
                                                        tp.m < p.m_tiles && tp.n < p.n_tiles && tp.k0 + steps <= p.segments * p.k_steps);
                    for (; k < end; ++k) {
                        ok = wait(empty0 + 8 * stage, parity ^ 1u);
                        if (!ok) break;
                        if (inside) {
                            const uint32_t bar = full0 + 8 * stage;
                            announce();
                            load_box(dst, &p.a, ax, ay, za, bar);
                            if (a_two) load_box(dst + kBoxBytes, &p.a, ax + 64, ay, za, bar);
                            load_box(dst + kBlockBytes, &p.b, bx, by, zb, bar);
                            if (b_two) load_box(dst + kBlockBytes + kBoxBytes, &p.b, bx + 64, by, zb, bar);
                            if (halves == 2) {
                                load_box(dst + 2 * kBlockBytes, &p.b, bx + 4 * br, by + 4 * (64 - br), zb, bar);
                                if (b_two) load_box(dst + 2 * kBlockBytes + kBoxBytes, &p.b, bx + 5 * 64, by, zb, bar);
                            }
                            ax += ak;
                            ay += kStepK - ak;
                            bx += bk;
                            by += kStepK - bk;
                        }
                        next();
                    }
                    at = 0;
                    ++seg;
                }
            }
            // the last commits arrive on this CTA's barriers: it must not leave before they have
            for (int i = 0; i < stages && ok; ++i) {
                ok = wait(empty0 + 8 * stage, parity ^ 1u);
                if (++stage == stages) {
                    stage = 0;
                    parity ^= 1u;
                }
            }
            issued[rank] = it;
        }
        if (warp == 1 && rank == 0 && elect_one()) {  // ---- MMA, the pair's first CTA
            int stage = 0, sub = 0;    // sub: accumulators used so far; they alternate
            const uint32_t tmem = ortho_keep(tmem_base);
            uint32_t parity = 0;
            bool ok = true;
            const int halves = ortho_keep(p.halves);
            const uint32_t idesc = ortho_keep((1u << 4) | ((uint32_t)p.a_mn << 15) | ((uint32_t)p.b_mn << 16) |
                                              ((uint32_t)(p.cols >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24));  // binary16 operands, binary32 sums
            const uint32_t da = ortho_keep(p.a_mn ? 2048u >> 4 : 32u >> 4), db = ortho_keep(p.b_mn ? 2048u >> 4 : 32u >> 4);
            const uint64_t a_base = operand_desc(ring, p.a_mn), b_base = operand_desc(ring + kBlockBytes, p.b_mn);
            const uint32_t full0 = ortho_keep(smem_addr(&full[0])), empty0 = ortho_keep(smem_addr(&empty[0])),
                           acc_full0 = ortho_keep(smem_addr(&acc_full[0])), acc_empty0 = ortho_keep(smem_addr(&acc_empty[0]));
            auto issue = [&](int st, int h, int acc, int k) {
                const uint64_t a = a_base + (uint32_t)(st * (stage_bytes >> 4));
                const uint64_t b = b_base + (uint32_t)(st * (stage_bytes >> 4) + h * (kBlockBytes >> 4));
#pragma unroll
                for (int i = 0; i < kStepK / 16; ++i)
                    mma_f16(tmem + (uint32_t)acc * kTile, a + i * da, b + i * db, idesc, (uint32_t)(k | i));
            };
            for (int t = pair; t < p.tiles; t += pairs) {
                const int steps = ortho_keep(ortho_tile(p, t).steps);
                const int acc0 = sub & 1, acc1 = acc0 ^ 1;
                const uint32_t parity0 = (uint32_t)((sub >> 1) & 1) ^ 1u, parity1 = (uint32_t)(((sub + 1) >> 1) & 1) ^ 1u;
                ok = wait(acc_empty0 + 8 * acc0, parity0);
                if (!ok) break;
                tmem_fence_after();
                if (halves == 1) {
                    for (int k = 0; k < steps; ++k) {
                        if (!(ok = wait(full0 + 8 * stage, parity))) break;
                        issue(stage, 0, acc0, k);
                        mma_commit_both(empty0 + 8 * stage);
                        ++stage;
                        parity ^= (uint32_t)(stage == stages);
                        stage = stage == stages ? 0 : stage;
                    }
                    if (!ok) break;
                    mma_commit_both(acc_full0 + 8 * acc0);
                    ++sub;
                    continue;
                }
                // With two accumulators the second may still be read when the first is free: its products follow
                // as soon as it is, at the latest when the ring is full of stages that wait for it.
                bool second = false;
                int behind = 0, tail = stage, kb = 0;
                for (int k = 0; k < steps; ++k) {
                    ok = wait(full0 + 8 * stage, parity);
                    if (!ok) break;
                    issue(stage, 0, acc0, k);
                    if (k + 1 == steps) mma_commit_both(acc_full0 + 8 * acc0);
                    ++behind;
                    if (!second) {
                        if (behind == stages || k + 1 == steps) {
                            ok = wait(acc_empty0 + 8 * acc1, parity1);
                            if (!ok) break;
                            second = true;
                        } else {
                            second = barrier_test(acc_empty0 + 8 * acc1, parity1);
                        }
                        if (second) tmem_fence_after();
                    }
                    for (; second && behind; --behind, ++kb) {
                        issue(tail, 1, acc1, kb);
                        mma_commit_both(empty0 + 8 * tail);
                        if (++tail == stages) tail = 0;
                    }
                    if (++stage == stages) {
                        stage = 0;
                        parity ^= 1u;
                    }
                }
                if (!ok) break;
                mma_commit_both(acc_full0 + 8 * acc1);
                sub += 2;
            }
        }
    } else {  // ---- epilogue: a thread owns one row and a quarter of an accumulator's columns
        const int quad = warp & 3, quarter = (warp - 4) >> 2;
        const OrthoStage stg = {ring + kRingBlocks * kBlockBytes + (warp - 4) * kOrthoStaging, lane};
        const int width = p.cols >> 2;  // columns of this thread: 64 or 32
        const long long plane = (long long)p.rows * p.pitch;
        const int tile_cols = p.cols * p.halves;
        int sub = 0;
        bool ok = true;
        for (int t = pair; t < p.tiles && ok; t += pairs) {
            const OrthoTile tp = ortho_tile(p, t);
            const int row0 = tp.m * kTile + (int)rank * kHalf + quad * 32, row = row0 + lane;
            const __half *in = KIND == kPoly || KIND == kUpdate || KIND == kResult ? p.in + (long long)tp.matrix * p.in_planes * plane : nullptr;
            __half *out = KIND != kGramPart && KIND != kResult ? p.out + (long long)tp.matrix * p.out_planes * plane : nullptr;
            for (int h = 0; h < p.halves; ++h, ++sub) {
                const int acc = sub & 1, col0 = (tp.n * p.halves + h) * p.cols + quarter * width;
                const uint32_t src = tmem_base + (uint32_t)acc * kTile + quarter * width + ((uint32_t)(quad * 32) << 16);
                [[maybe_unused]] uint4 hi[4], lo[4];  // of the tile of A or Y that is added, fetched ahead
                auto fetch = [&](int col) {
                    stg.fetch(hi, in, p.pitch, row0, p.rows, col);
                    if (p.in_planes > 1) stg.fetch(lo, in + plane, p.pitch, row0, p.rows, col);
                };
                constexpr bool adds = KIND == kPoly || KIND == kUpdate || KIND == kResult;
                if (adds && p.in_planes > 0) fetch(col0);
                ok = __all_sync(0xFFFFFFFFu, wait(smem_addr(&acc_full[acc]), (uint32_t)((sub >> 1) & 1)));
                if (!ok) break;
                tmem_fence_after();
#pragma unroll 1
                for (int at = 0; at < width; at += 32) {
                    const int col = col0 + at;
                    uint32_t raw[32];
                    __syncwarp();
                    tmem_load32(src + at, raw);
                    tmem_wait_load(raw);
                    if (at + 32 == width) {  // the accumulator is read: the tile after the next may overwrite it
                        tmem_fence_before();
                        __syncwarp();
                        if (lane == 0) barrier_arrive_leader(smem_addr(&acc_empty[acc]));
                    }
                    float z[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) z[i] = __uint_as_float(raw[i]) * p.acc_scale;
                    if (row0 >= p.rows || col >= (KIND == kResult ? p.columns : p.pitch)) continue;
                    // read anew in each round, from L1: held in a register, other values are spilled (32000 x 1024: 853 us, 832 us so)
                    [[maybe_unused]] const float2 *const powers = p.powers + tp.matrix * kOrthoMaxSteps + p.step;
                    if constexpr (KIND == kGram || KIND == kGramPart) ortho_scale(z, powers->x);
                    if constexpr (KIND == kGramPart) {
                        float *dst = p.part + (long long)(tp.matrix * p.splits + tp.split) * p.rows * p.pitch;
                        stg.store_part(z, dst, p.pitch, row0, p.rows, col);
                        continue;
                    }
                    if (adds && p.in_planes > 0) {
                        stg.deal(hi);
                        stg.add_row(z, p.in_scale);
                        if (p.in_planes > 1) {
                            stg.deal(lo);
                            stg.add_row(z, p.in_scale);
                        }
                        if (at + 32 < width) fetch(col + 32);
                    }
                    if constexpr (KIND == kUpdate || KIND == kResult) ortho_scale(z, powers->y);
                    if constexpr (KIND == kGram || KIND == kSquare) {
                        if (p.diag != 0.0f && col <= row0 + 31 && col + 31 >= row0) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (col + i == row && row < p.rows) z[i] += p.diag;
                        }
                    }
                    if constexpr (KIND == kResult) {
                        stg.template put_row<T>(z);
                        stg.store_result((uint16_t *)p.result + tp.matrix * p.result_matrix, p.result_row, row0, p.rows, col, p.columns,
                                         p.result_wide);
                        continue;
                    }
                    // across the diagonal unless the tile there is computed itself
                    const bool across = KIND != kUpdate && row0 / tile_cols * tile_cols >= (col / kTile + 1) * kTile;
                    for (int i = 0;; ++i) {
                        stg.template put_row<__half>(z);
                        stg.store(out + i * plane, p.pitch, row0, p.rows, col);
                        if (across) {
                            stg.put_column(z);
                            stg.store(out + i * plane, p.pitch, col, p.rows, row0);
                        }
                        if (i + 1 == p.out_planes) break;
                        ortho_rest(z);
                    }
                }
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (threadIdx.x < 2) store_in(smem_addr(&failed[rank]), dead, threadIdx.x);
    __syncwarp();
    cluster_sync_all();  // the peer may still signal this CTA's barriers, and its MMAs read this CTA's memory
    if (failed[0] | failed[1]) {
        // A wait gave up in one of the CTAs, and both have left their loops: what they have in flight still reads and
        // writes their shared memory and TMEM.  Let it end (bounded).
        if (rank == 1 && warp == 0 && lane <= stages)
            store_in(lane < stages ? smem_addr(&sent[1][lane]) : smem_addr(&issued[1]), lane < stages ? sent[1][lane] : issued[1], 0);
        __syncwarp();
        cluster_sync_all();
        if (warp == 0 && rank == 0 && lane < stages) {
            // a lane per place in the ring, its latest stage `i`; a producer is at most a ring ahead of the other, so that the
            // barrier is in that stage's phase and lacks at most what only one of the two has issued
            const int most = max(issued[0], issued[1]), i = most - 1 - (most - 1 - lane + stages) % stages;
            if (i >= 0 && i < most) {
                const uint32_t bar = smem_addr(&full[lane]);
                if (i >= issued[1]) barrier_complete(bar, (uint32_t)sent[0][lane]);
                if (i >= issued[0]) barrier_expect(bar, (uint32_t)sent[1][lane]);
                for (unsigned n = 0; n < kOperatorPolls && !barrier_try(bar, (uint32_t)(i / stages) & 1u); ++n) {}
            }
        }
        if (warp == 1) {
            if (rank == 0 && elect_one()) mma_commit_both(smem_addr(&drain));  // by the thread that issued them
            __syncwarp();
            for (unsigned n = 0; n < kOperatorPolls && !barrier_try(smem_addr(&drain), 0); ++n) {}
        }
        __syncwarp();
        __syncthreads();
        cluster_sync_all();
    }
    if (warp == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem_base));
}

// ---- the kernels around the products ------------------------------------------------------------------
constexpr int kOrthoItem = 1024;   // columns of a row that a warp takes at a time, eight per lane
constexpr int kOrthoLoadWarps = 8;

// Eight values of a row from p on, of which n exist.
template <typename T>
__device__ __forceinline__ void ortho_load8(float (&v)[8], const T *p, int n, bool wide)
{
    if (wide && n >= 8) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        } else {
            const uint4 a = __ldg(reinterpret_cast<const uint4 *>(p));
            T t[8];
            *reinterpret_cast<uint4 *>(t) = a;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = to_f32(t[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32(p[i]) : 0.0f;
    }
}

// |X|^2 of each matrix in `parts` parts, in binary64 (neither the squares of large nor of small gradients leave its range).
template <typename T>
__global__ void __launch_bounds__(32 * kOrthoLoadWarps)
k_ortho_norm(const T *__restrict__ x, long long row_stride, long long matrix_stride, int rows, int cols, int wide, int parts,
             double *__restrict__ partial)
{
    __shared__ double sums[kOrthoLoadWarps];
    const int matrix = blockIdx.x / parts, part = blockIdx.x - matrix * parts, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_dependency_wait();
    grid_dependency_launch_next();
    const T *m = x + matrix * matrix_stride;
    const int across = (cols + kOrthoItem - 1) / kOrthoItem;
    double some[4] = {};
    for (long long i = part * kOrthoLoadWarps + warp; i < (long long)rows * across; i += parts * kOrthoLoadWarps) {
        const long long row = i / across;
        const int c0 = (int)(i - row * across) * kOrthoItem;
#pragma unroll
        for (int j = 0; j < kOrthoItem / 256; ++j) {
            const int c = c0 + j * 256 + lane * 8;
            float v[8];
            if (c < cols) {
                ortho_load8(v, m + row * row_stride + c, cols - c, wide);
#pragma unroll
                for (int k = 0; k < 8; ++k) some[k & 3] = fma((double)v[k], (double)v[k], some[k & 3]);
            }
        }
    }
    double s = (some[0] + some[1]) + (some[2] + some[3]);
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    if (lane == 0) sums[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kOrthoLoadWarps; ++w) s += sums[w];
        partial[blockIdx.x] = s;
    }
}

// By what a step may enlarge singular values at most: max |a + b s^2 + c s^4|
struct OrthoGrowth {
    float by[kOrthoMaxSteps];
    int steps;
};
// With all singular values at most `bound`, a power of two that they may have beside Y's scale
__device__ __forceinline__ int ortho_room(double bound)
{
    const int e = bound > 0.0 ? 1022 - (__double2hiint(bound) >> 20) : 0;  // bound 2^e is in [1/2, 1); NaN and zero: none
    return min(max(e, 0), kOrthoMostPower);
}

// Y = X / (|X| + eps), scaled, in two binary16 planes.  A matrix of zeros stays one; one that is not finite becomes NaN.
template <typename T>
__global__ void __launch_bounds__(32 * kOrthoLoadWarps)
k_ortho_load(const T *__restrict__ x, long long row_stride, long long matrix_stride, int rows, int cols, int wide, int parts,
             const double *__restrict__ partial, float eps, __half *__restrict__ y, long long pitch, const OrthoGrowth growth,
             float2 *__restrict__ powers)
{
    const int matrix = blockIdx.x / parts, part = blockIdx.x - matrix * parts, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_dependency_wait();
    grid_dependency_launch_next();
    double s = 0.0;
    for (int i = lane; i < parts; i += 32) s += partial[matrix * parts + i];
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    const double norm = sqrt(s);
    // in two factors, so that neither leaves binary32's range
    const double first = norm < 1e-20 ? 0x1p60 : norm > 1e20 ? 0x1p-60 : 1.0;
    double bound = norm / (norm + eps);
    const float f1 = (float)first,
                f2 = norm == 0.0 ? 0.0f : norm < INFINITY ? (float)(ldexp((double)kOrthoScale, ortho_room(bound)) / ((norm + eps) * first)) : NAN;
    if (part == 0 && threadIdx.x == 0) {
        float2 *const to = powers + matrix * kOrthoMaxSteps;
        for (int i = 0, k = ortho_room(bound); i < growth.steps; ++i) {
            bound *= growth.by[i];
            const int after = i + 1 < growth.steps ? ortho_room(bound) : 0;
            to[i] = make_float2(exp2f((float)(-2 * k)), exp2f((float)(after - k)));
            k = after;
        }
    }
    const T *m = x + matrix * matrix_stride;
    __half *hi = y + matrix * 2 * (long long)rows * pitch, *lo = hi + (long long)rows * pitch;
    const int across = (cols + kOrthoItem - 1) / kOrthoItem;
    for (long long i = part * kOrthoLoadWarps + warp; i < (long long)rows * across; i += parts * kOrthoLoadWarps) {
        const long long row = i / across;
        const int c0 = (int)(i - row * across) * kOrthoItem;
#pragma unroll
        for (int j = 0; j < kOrthoItem / 256; ++j) {
            const int c = c0 + j * 256 + lane * 8;
            if (c >= pitch || !RSDGC_IN_BOUNDS(row < rows && c + 8 <= pitch)) continue;
            float v[8];
            ortho_load8(v, m + row * row_stride + c, cols - c, wide);
            uint32_t a[4], b[4];
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const float u = v[k] * f1 * f2, w = v[k + 1] * f1 * f2;
                a[k >> 1] = pack2<__half>(u, w);
                b[k >> 1] = pack2<__half>(u - __half2float(__float2half_rn(u)), w - __half2float(__float2half_rn(w)));
            }
            *reinterpret_cast<uint4 *>(hi + row * pitch + c) = make_uint4(a[0], a[1], a[2], a[3]);
            *reinterpret_cast<uint4 *>(lo + row * pitch + c) = make_uint4(b[0], b[1], b[2], b[3]);
        }
    }
}

// A = the sum of its parts, in order: a CTA per block of 32 x 32 on or below the diagonal, which it also writes across it.
__global__ void __launch_bounds__(256)
k_ortho_join(const float *__restrict__ part, int splits, int n, long long pitch, int blocks, float diag, __half *__restrict__ out, int planes)
{
    __shared__ float block[32][33];
    int i = blockIdx.x % (blocks * (blocks + 1) / 2);
    const int matrix = blockIdx.x / (blocks * (blocks + 1) / 2);
    int bi = (int)((sqrtf(8.0f * i + 1.0f) - 1.0f) * 0.5f);
    while (bi * (bi + 1) / 2 > i) --bi;
    while ((bi + 1) * (bi + 2) / 2 <= i) ++bi;
    i -= bi * (bi + 1) / 2;
    const int lane = threadIdx.x & 31, row0 = threadIdx.x >> 5;
    grid_dependency_wait();
    grid_dependency_launch_next();
    const long long plane = (long long)n * pitch;
    out += matrix * planes * plane;
    part += matrix * splits * plane;
    auto put = [&](int r, int c, float v) {
        if (r >= n || c >= pitch || !RSDGC_IN_BOUNDS(r >= 0 && c >= 0)) return;
        const __half h = __float2half_rn(v);
        out[r * pitch + c] = h;
        if (planes > 1) out[plane + r * pitch + c] = __float2half_rn(v - __half2float(h));
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = bi * 32 + row0 + 8 * j, c = i * 32 + lane;
        float v = 0.0f;
        if (r < n && c < pitch)
            for (int s = 0; s < splits; ++s) v += part[s * plane + r * pitch + c];
        if (r == c) v += diag;
        block[row0 + 8 * j][lane] = v;
        put(r, c, v);
    }
    if (bi == i) return;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) put(i * 32 + row0 + 8 * j, bi * 32 + lane, block[lane][row0 + 8 * j]);
}

// ---- host -----------------------------------------------------------------------------------------------
RSDGC_DEFINE_DEBUG_BOUNDS(orthogonal_debug_bounds)

namespace {

constexpr int kOrthoPairs = 74;          // of CTAs on the device, for what workspaces depend on
constexpr int kOrthoLoadParts = 1184;    // most CTAs per matrix of the two passes over X: eight a multiprocessor (two: 32000 x 1024 36 us more)
// Shorter sides up to this take three products for every result: there they cost a fifth of the call at most, beyond it more and more (bfloat16
// results, one product and three: 128 x 512 122 and 142 us, 256 x 512 126 and 151, 24 x 256 x 1024 217 and 257, 512 x 1024 153 and 196, 8 x 512 x
// 1024 192 and 261, 1024 x 1024 171 and 271).
constexpr int64_t kOrthoPrecise = 256;

inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }
inline int tiles_of(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// What a call does with its sizes.
struct OrthoLayout {
    int64_t batch, rows, cols, side, pitch, side_pitch;  // side: of A
    bool tall;
    int segments, planes, parts, splits, split_steps;
    int64_t y[2], a, b, norm, powers, sums, bytes;
};

OrthoLayout ortho_layout(int64_t batch, int64_t rows, int64_t cols, int out_dtype)
{
    OrthoLayout L{};
    L.batch = batch;
    L.rows = rows;
    L.cols = cols;
    L.tall = rows > cols;
    L.side = L.tall ? cols : rows;
    L.pitch = up(cols, 8);
    L.side_pitch = up(L.side, 8);
    L.planes = out_dtype == RSDGC_F16 || L.side <= kOrthoPrecise ? 2 : 1;
    L.segments = L.planes == 2 ? 3 : 1;
    const int64_t items = rows * ((cols + kOrthoItem - 1) / kOrthoItem), want = (items + kOrthoLoadWarps - 1) / kOrthoLoadWarps;
    L.parts = (int)(want < kOrthoLoadParts ? want : kOrthoLoadParts);
    // A's tiles are few where it is small: its contraction is cut so that every pair of CTAs has a part, where the steps that this
    // saves are more than the second kernel takes (about 7 us, 26 steps; a part's bytes about two)
    const int64_t m = tiles_of(L.side, kTile), tiles = batch * m * (m + 1) / 2;
    const int64_t steps = (int64_t)L.segments * tiles_of(L.tall ? rows : cols, kStepK);
    int64_t s = 1, least = steps;
    for (int64_t i = 2; i <= (tiles > 0 ? kOrthoPairs / tiles : 1) && i <= steps / 8; ++i)
        if ((steps + i - 1) / i + 26 + 2 * i < least) least = (steps + i - 1) / i + 26 + 2 * i, s = i;
    L.split_steps = (int)((steps + s - 1) / s);
    L.splits = (int)((steps + L.split_steps - 1) / L.split_steps);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t p = at;
        at = up(at + bytes, 256);
        return p;
    };
    for (int i = 0; i < 2; ++i) L.y[i] = take(batch * 2 * rows * L.pitch * 2);
    L.a = take(batch * L.planes * L.side * L.side_pitch * 2);
    L.b = take(batch * L.planes * L.side * L.side_pitch * 2);
    L.norm = take(batch * L.parts * 8);
    L.powers = take(rows > 0 && cols > 0 ? batch * kOrthoMaxSteps * 8 : 0);
    L.sums = take(L.splits > 1 ? batch * L.splits * L.side * L.side_pitch * 4 : 0);
    L.bytes = at;
    return L;
}

int ortho_check(int64_t batch, int64_t rows, int64_t cols, int out_dtype)
{
    if (batch < 0 || rows < 0 || cols < 0 || (out_dtype != RSDGC_BF16 && out_dtype != RSDGC_F16)) return RSDGC_ERR_INVALID;
    if (rows > (1 << 24) || cols > (1 << 24) || (rows < cols ? rows : cols) > (1 << 15) || batch > (1 << 20)) return RSDGC_ERR_CAPACITY;
    // tiles of 256 x 128 of all matrices, and the grids of the other kernels
    const int64_t tiles = batch * tiles_of(rows, kTile) * tiles_of(cols, kTile / 2) * 64;
    return tiles > INT_MAX || batch * kOrthoLoadParts > INT_MAX ? RSDGC_ERR_CAPACITY : RSDGC_OK;
}

// The polynomials as a whole keep singular values within [0, most], at most 2 and what the roundings add, and |b x + c x^2| <= 30 for x = s^2: what the scaled
// binary16 planes hold, with B's scale halved twice at most.  s is at most 1 at first; a step's largest value lies at an end or where a + 3 b s^2 + 5 c s^4 = 0.
struct OrthoSteps {
    bool square[kOrthoMaxSteps];  // whether they hold A + b / 2c and a + b x + c x^2 = c (x + b / 2c)^2 + a - b^2 / 4c as well
    float b_scale[kOrthoMaxSteps];  // B's beside kOrthoScaleA: 1, 1/2 or 1/4
    OrthoGrowth growth;
};
bool ortho_bounded(const float *coef, int steps, OrthoSteps *out)
{
    out->growth.steps = steps;
    double most = 1.0;
    for (int i = 0; i < steps; ++i) {
        const double a = coef[3 * i], b = coef[3 * i + 1], c = coef[3 * i + 2];
        if (!(std::fabs(a) < 1e3 && std::fabs(b) < 1e3 && std::fabs(c) < 1e3)) return false;
        double top = 0.0, poly = 0.0, grows = 0.0;
        auto at = [&](double s2) {
            if (!(s2 >= 0.0 && s2 <= most * most)) return;
            const double v = std::fabs(std::sqrt(s2) * (a + s2 * (b + s2 * c)));
            if (v > top) top = v;
        };
        auto inner = [&](double s2) {
            if (!(s2 >= 0.0 && s2 <= most * most)) return;
            const double v = std::fabs(s2 * (b + s2 * c));
            if (v > poly) poly = v;
            grows = std::fmax(grows, std::fabs(a + s2 * (b + s2 * c)));
        };
        inner(0.0);
        at(most * most);
        inner(most * most);
        // the roots of a + 3 b x + 5 c x^2 without a difference of near values, whatever c is
        const double root = 9.0 * b * b - 20.0 * a * c;
        if (root >= 0.0) {
            const double sum = -0.5 * (3.0 * b + std::copysign(std::sqrt(root), b));
            if (sum != 0.0) at(a / sum);
            if (c != 0.0) at(sum / (5.0 * c));
        }
        if (c != 0.0) inner(-b / (2.0 * c));
        out->square[i] = std::fabs(c) > 0.1 && std::fabs(b / (2.0 * c)) + most * most <= 7.5 && std::fabs(a) + poly <= 7.5;
        most = top * (1.0 + 0x1p-7);  // and what the roundings add
        out->growth.by[i] = (float)(grows * (1.0 + 0x1p-7));
        if (top > 2.0 || poly > 30.0) return false;
        out->b_scale[i] = poly <= 7.5 ? 1.0f : poly <= 15.0 ? 0.5f : 0.25f;
    }
    return true;
}

// [matrix x plane][rows][cols] binary16 values, boxes of 64 columns; what lies outside reads as zero
cudaError_t ortho_map(CUtensorMap *map, const void *base, int64_t slabs, int64_t rows, int64_t cols, int64_t pitch, int box_rows)
{
    EncodeFn fn = encode_fn();
    if (!fn) return cudaErrorNotSupported;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)slabs};
    const cuuint64_t strides[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)pitch * 2 * (cuuint64_t)rows};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(base), dims, strides, box, one,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// ... with boxes of 64 rows, and of 128: all rows of a CTA's block, where they do not lie contiguous
struct OrthoMaps {
    CUtensorMap of[2];
};
cudaError_t ortho_maps(OrthoMaps *m, const void *base, int64_t slabs, int64_t rows, int64_t cols, int64_t pitch)
{
    const cudaError_t e = ortho_map(&m->of[0], base, slabs, rows, cols, pitch, 64);
    return e != cudaSuccess ? e : ortho_map(&m->of[1], base, slabs, rows, cols, pitch, kHalf);
}

// Pairs of CTAs that the device holds at a time; 0 and an error in *e if the kernel cannot run.
template <int KIND, typename T>
int ortho_pairs(cudaError_t *e)
{
    static std::mutex mu;
    static int most[64];
    int dev = 0;
    *e = cudaGetDevice(&dev);
    if (*e != cudaSuccess) return 0;
    std::lock_guard<std::mutex> lock(mu);
    int &m = most[dev & 63];
    if (m) return m;
    *e = cudaFuncSetAttribute(k_ortho<KIND, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kOrthoSmem);
    if (*e != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = (unsigned)current_device_sms();
    cfg.blockDim = kOrthoThreads;
    cfg.dynamicSmemBytes = kOrthoSmem;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 2;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    int n = 0;
    *e = cudaOccupancyMaxActiveClusters(&n, k_ortho<KIND, T>, &cfg);
    if (*e == cudaSuccess && n < 1) *e = cudaErrorLaunchOutOfResources;
    return *e == cudaSuccess ? m = n : 0;
}

// Tiles of 256 x 128, 256 x 256 or 256 x 512 by the cycles that they take dealt to the pairs (512 per contraction step and
// 256 columns, some 6000 to empty an accumulator; 1.25 and 1.6 times that for the lost operand reuse of 256 and 128 columns).
void ortho_columns(OrthoParams &p, int64_t batch, int pairs)
{
    double best = 0.0;
    for (int wide = kTile / 2; wide <= 2 * kTile; wide *= 2) {
        if (wide > kTile && p.columns <= kTile) break;
        const int across = tiles_of(p.columns, wide);
        long long per = (long long)p.m_tiles * across;
        if (p.symmetric) {
            per = 0;
            for (int m = 0; m < p.m_tiles; ++m) {
                const int here = ((m + 1) * kTile + wide - 1) / wide;
                per += here < across ? here : across;
            }
        }
        const long long tiles = per * batch * p.splits;
        const double part = (double)wide / kTile, loss = wide > kTile ? 1.0 : wide == kTile ? 1.25 : 1.6;
        const double cost = (double)((tiles + pairs - 1) / pairs) * loss * part * (512.0 * p.split_steps + 6000.0);
        if (best > 0.0 && cost > best) continue;
        best = cost;
        p.halves = wide > kTile ? 2 : 1;
        p.cols = wide < kTile ? wide : kTile;
        p.n_tiles = across;
        p.per = (int)per;
        p.tiles = (int)tiles;
    }
    p.stages = kRingBlocks / (1 + p.halves);
}

struct OrthoCall {
    OrthoLayout l;
    const void *x;
    int64_t x_row, x_matrix;
    int dtype;
    void *out;
    int64_t out_row, out_matrix;
    int out_dtype;
    const float *coef;
    const OrthoSteps *about;
    int steps;
    float eps;
    unsigned char *workspace;
    cudaStream_t s;
};

template <int KIND, typename T>
cudaError_t ortho_product(OrthoParams &p, const OrthoMaps &left, const OrthoMaps &right, const OrthoCall &c)
{
    cudaError_t e = cudaSuccess;
    const int most = ortho_pairs<KIND, T>(&e);
    if (e != cudaSuccess) return e;
    ortho_columns(p, c.l.batch, most);
    p.a = left.of[!p.a_mn];
    p.b = right.of[!p.b_mn && p.cols == kTile];
    const unsigned pairs = (unsigned)(p.tiles < most ? p.tiles : most);
    return launch_chained(k_ortho<KIND, T>, 2 * pairs, kOrthoThreads, kOrthoSmem, c.s, 2, p);
}

template <typename T>
cudaError_t ortho_load(const OrthoCall &c)
{
    const OrthoLayout &L = c.l;
    const unsigned grid = (unsigned)(L.batch * L.parts);
    const int wide = pointer_aligned(c.x, 16) && c.x_row * sizeof(T) % 16 == 0 && c.x_matrix * sizeof(T) % 16 == 0;
    double *norm = (double *)(c.workspace + L.norm);
    cudaError_t e = launch_chained(k_ortho_norm<T>, grid, 32 * kOrthoLoadWarps, 0, c.s, 1, (const T *)c.x, (long long)c.x_row,
                                   (long long)c.x_matrix, (int)L.rows, (int)L.cols, wide, L.parts, norm);
    if (e == cudaSuccess)
        e = launch_chained(k_ortho_load<T>, grid, 32 * kOrthoLoadWarps, 0, c.s, 1, (const T *)c.x, (long long)c.x_row,
                           (long long)c.x_matrix, (int)L.rows, (int)L.cols, wide, L.parts, (const double *)norm, c.eps,
                           (__half *)(c.workspace + L.y[0]), (long long)L.pitch, c.about->growth, (float2 *)(c.workspace + L.powers));
    return e;
}

cudaError_t orthogonalize(const OrthoCall &c)
{
    const OrthoLayout &L = c.l;
    cudaError_t e = operators_ready();
    OrthoParams base;
    std::memset(&base, 0, sizeof base);
    base.polls = operator_polls();
    base.segments = L.segments;
    base.splits = 1;
    base.powers = (const float2 *)(c.workspace + L.powers);
    if (e == cudaSuccess) e = operator_status_ptr(&base.status);
    OrthoMaps y[2], a, b;
    for (int i = 0; i < 2 && e == cudaSuccess; ++i) e = ortho_maps(&y[i], c.workspace + L.y[i], 2 * L.batch, L.rows, L.cols, L.pitch);
    if (e == cudaSuccess) e = ortho_maps(&a, c.workspace + L.a, L.planes * L.batch, L.side, L.side, L.side_pitch);
    if (e == cudaSuccess) e = ortho_maps(&b, c.workspace + L.b, L.planes * L.batch, L.side, L.side, L.side_pitch);
    if (e == cudaSuccess)
        e = c.dtype == RSDGC_F32 ? ortho_load<float>(c) : c.dtype == RSDGC_BF16 ? ortho_load<__nv_bfloat16>(c) : ortho_load<__half>(c);
    __half *const ap = (__half *)(c.workspace + L.a), *const bp = (__half *)(c.workspace + L.b);
    for (int i = 0; i < c.steps && e == cudaSuccess; ++i) {
        const OrthoMaps &from = y[i & 1];
        __half *const yp = (__half *)(c.workspace + L.y[i & 1]);
        const double ca = c.coef[3 * i], cb = c.coef[3 * i + 1], cc = c.coef[3 * i + 2];
        // Three products: 22 bits hold a + B as well as B, so that a Y needs no addition of its own; nor does b A with the square completed.
        // The epilogues then read nothing (256 x 1024: 24 matrices' update 34 us with that, 25 us without).
        const bool square = L.segments == 3 && c.about->square[i];
        OrthoParams p = base;  // A = Y Y^T or Y^T Y
        p.step = i;
        p.diag = square ? (float)(cb / (2.0 * cc)) * kOrthoScaleA : 0.0f;
        p.a_mn = p.b_mn = L.tall;
        p.a_planes = p.b_planes = 2;
        p.k_steps = tiles_of(L.tall ? L.rows : L.cols, kStepK);
        p.rows = p.columns = (int)L.side;
        p.pitch = L.side_pitch;
        p.m_tiles = tiles_of(L.side, kTile);
        p.symmetric = 1;
        p.splits = L.splits;
        p.split_steps = L.split_steps;
        p.acc_scale = 0x1p-11f;  // 2^24 to 2^13
        p.out = ap;
        p.out_planes = L.planes;
        p.part = (float *)(c.workspace + L.sums);
        if (L.splits > 1) {
            e = ortho_product<kGramPart, __half>(p, from, from, c);
            const int blocks = tiles_of(L.side, 32);
            if (e == cudaSuccess)
                e = launch_chained(k_ortho_join, (unsigned)(L.batch * blocks * (blocks + 1) / 2), 256, 0, c.s, 1, (const float *)p.part,
                                   L.splits, (int)L.side, (long long)L.side_pitch, blocks, p.diag, ap, L.planes);
        } else {
            e = ortho_product<kGram, __half>(p, from, from, c);
        }
        if (e != cudaSuccess) break;
        // B = b A + c A A
        p.a_mn = p.b_mn = 0;
        p.a_planes = p.b_planes = L.planes;
        p.in_planes = square ? 0 : L.planes;
        p.k_steps = tiles_of(L.side, kStepK);
        p.splits = 1;
        p.split_steps = L.segments * p.k_steps;
        p.in = ap;
        p.in_scale = (float)cb * c.about->b_scale[i];
        p.acc_scale = (float)cc * 0x1p-13f * c.about->b_scale[i];
        p.diag = square ? (float)(ca - cb * cb / (4.0 * cc)) * kOrthoScaleA : 0.0f;
        p.out = bp;
        e = square ? ortho_product<kSquare, __half>(p, a, a, c) : ortho_product<kPoly, __half>(p, a, a, c);
        if (e != cudaSuccess) break;
        // B Y, or Y B where B is as good as its transpose
        const OrthoMaps &left = L.tall ? from : b, &right = L.tall ? b : from;
        p.b_mn = !L.tall;
        p.a_planes = L.tall ? 2 : L.planes;
        p.b_planes = L.tall ? L.planes : 2;
        p.symmetric = 0;
        p.rows = (int)L.rows;
        p.columns = (int)L.cols;
        p.pitch = L.pitch;
        p.m_tiles = tiles_of(L.rows, kTile);
        p.band = p.m_tiles < 16 ? p.m_tiles : 16;
        p.in = yp;
        p.in_planes = square ? 0 : 2;
        p.in_scale = (float)ca;
        p.acc_scale = 0x1p-13f / c.about->b_scale[i];
        p.diag = 0.0f;
        p.out = (__half *)(c.workspace + L.y[(i + 1) & 1]);
        p.out_planes = 2;
        if (i + 1 < c.steps) {
            e = ortho_product<kUpdate, __half>(p, left, right, c);
        } else {
            p.in_scale *= 1.0f / kOrthoScale;
            p.acc_scale *= 1.0f / kOrthoScale;
            p.result = c.out;
            p.result_row = c.out_row;
            p.result_matrix = c.out_matrix;
            p.result_wide = pointer_aligned(c.out, 16) && c.out_row % 8 == 0 && c.out_matrix % 8 == 0;
            e = c.out_dtype == RSDGC_BF16 ? ortho_product<kResult, __nv_bfloat16>(p, left, right, c) : ortho_product<kResult, __half>(p, left, right, c);
        }
    }
    return e;
}

}  // namespace
}  // namespace rsdgc

using namespace rsdgc;

extern "C" int64_t rsdgc_orthogonalize_workspace_bytes(int64_t n_matrices, int64_t n_rows, int64_t n_cols, int32_t out_dtype)
{
    const int rc = ortho_check(n_matrices, n_rows, n_cols, out_dtype);
    return rc ? rc : ortho_layout(n_matrices, n_rows, n_cols, out_dtype).bytes;
}

extern "C" int rsdgc_orthogonalize(const void *x_dev, int64_t x_row_stride, int64_t x_matrix_stride, int32_t dtype, void *out_dev,
                                   int64_t out_row_stride, int64_t out_matrix_stride, int32_t out_dtype, int64_t n_matrices,
                                   int64_t n_rows, int64_t n_cols, const float *coefficients_host, int32_t n_steps, float eps,
                                   void *workspace_dev, void *stream)
{
    const int rc = ortho_check(n_matrices, n_rows, n_cols, out_dtype);
    if (rc) return rc;
    if (!known_dtype(dtype) || !coefficients_host || n_steps < 1 || n_steps > kOrthoMaxSteps || !(eps >= 0.0f && eps < INFINITY))
        return RSDGC_ERR_INVALID;
    OrthoSteps about;
    if (!ortho_bounded(coefficients_host, n_steps, &about)) return RSDGC_ERR_INVALID;
    if (n_matrices == 0 || n_rows == 0 || n_cols == 0) return RSDGC_OK;
    if (!x_dev || !out_dev || !workspace_dev || (n_rows > 1 && (x_row_stride < n_cols || out_row_stride < n_cols)) ||
        (n_matrices > 1 && (x_matrix_stride < n_cols || out_matrix_stride < n_cols)) ||
        !rows_apart(n_matrices, out_matrix_stride, n_rows, out_row_stride, n_cols))
        return RSDGC_ERR_INVALID;
    if (!pointer_aligned(x_dev, dtype_bytes(dtype)) || !pointer_aligned(out_dev, 2) || !pointer_aligned(workspace_dev, 256))
        return RSDGC_ERR_ALIGNMENT;
    OperatorRange range("rsdgc_orthogonalize");
    if (n_matrices == 1) x_matrix_stride = out_matrix_stride = 0;  // free, and so are a single row's
    if (n_rows == 1) x_row_stride = out_row_stride = 0;
    const OrthoCall c = {ortho_layout(n_matrices, n_rows, n_cols, out_dtype), x_dev, x_row_stride, x_matrix_stride, dtype, out_dev,
                         out_row_stride, out_matrix_stride, out_dtype, coefficients_host, &about, n_steps, eps, (unsigned char *)workspace_dev,
                         (cudaStream_t)stream};
    return operator_result(orthogonalize(c));
}
