// The vocabulary head: softmax cross entropy and distillation from a teacher's top logits, forward and
// backward, straight from the hidden states and the vocabulary matrix, without keeping the logits.
//
//   z = h W^T (n x V),  c = 1 / T,  lse_n = log sum_v exp(c z_nv)
//   labels:    loss_n = lse_n - z_{n, y_n}                                             (T = 1)
//   top logits: q = softmax of the k given logits / T, loss_n = T^2 sum_j q_j (log q_j - (c z_{n, i_j} - lse_n))
//   gradient:  dz_nv = g_n T (softmax(c z)_nv - target_nv),  dh = dz W,  dW = dz^T h
//
// Both losses are the same computation: a target distribution with k entries per row.  Three matrix products
// carry it, all by one persistent kernel (k_head) that differs only in what it does with a finished tile:
//   forward   z tile -> per row the maximum and the sum of exponentials of the tile's columns, and z at the targets
//   backward  z tile again (recomputed) -> dz of one piece of the vocabulary, 16 bits, in the workspace
//             dz W_piece -> added to dh;  dz^T h -> the piece's rows of dW
// A launch of the backward pass holds both products of one piece and the dz of the next, from one queue of tiles.
//
// The tile kernel: pairs of CTAs (cluster of 2, one pair per two multiprocessors) compute tiles of 256 rows and 128 to 512
// columns with tcgen05.mma.cta_group::2, K in steps of 64.  One warp brings the operands by TMA (128-byte swizzle) through a
// ring of 4 to 6 stages, 192 KB per CTA; one thread issues the MMAs; sixteen warps empty an accumulator from tensor memory
// while the other one (256 columns each, 512 in all) is filled.  Operands whose contraction index is not the contiguous one
// (W in dz W, both in dz^T h) are read as they lie in memory: the MMA takes them as MN-major.
//
// What bounds it: the tensor cores, and in long runs the power limit.  Rates by the products that are computed (one
// forward, three backward), bfloat16, sizes as tokens x vocabulary x width, medians of 12 graphs of five calls: 2048 x 32000 x
// 2048 forward 174 us, 1.54 PFLOP/s, backward 539 us, 1.49; x 4096 330 us, 1.63, and 1.06 to 1.11 ms, 1.45 to 1.52; 8192 x
// 128000 x 4096 5.8 to 6.1 ms, 1.41 to 1.48, and 19.0 ms, 1.36.  (Whole calls for seconds on end: 8192 x 128000 x 4096 25.0 ms
// for both, 1.37.)  With up to a few hundred tokens it is W's way from memory: 64 x 32000 x 8192 forward takes 98 us, W at 5.3
// TB/s, backward 332 us (W twice and dW at 4.7).  Small calls are bound by the launches and the fill of the ring: 5 x 1000 x 256
// takes 9 us forward and 20 backward.  Widths that are no multiple of 8, whose outputs leave value by value: 2048 x 32000 x 2047
// 175 and 559 us, 300 x 4000 x 2001 backward 74 us where 2008 takes 67.
#include <cuda.h>

#include <climits>
#include <cmath>
#include <cstring>
#include <mutex>
#include <type_traits>
#include <utility>

#include "device_utils.cuh"
#include "operators_internal.cuh"

namespace rsdgc {

constexpr int kTile = 256;          // rows of a pair's tile, and columns of one accumulator
constexpr int kHalf = 128;          // rows of an operand block that one CTA holds
constexpr int kStepK = 64;          // contraction step: 64 x 2 bytes = the 128-byte swizzle span
constexpr int kBoxBytes = 64 * kStepK * 2;
constexpr int kBlockBytes = 2 * kBoxBytes;
constexpr int kRingBlocks = 12;     // of A and B blocks: 4 stages of 1 + 2 blocks, or 6 stages of 1 + 1
constexpr int kMaxStages = kRingBlocks / 2;
constexpr int kEpilogueWarps = 16;                       // four per quarter of an accumulator's columns
constexpr int kHeadThreads = 128 + 32 * kEpilogueWarps;  // producer, MMA, two idle warps, epilogue
constexpr int kStagingBytes = 2048;  // per epilogue warp: 32 rows of 64 bytes on their way out
constexpr int kHeadSmem = kRingBlocks * kBlockBytes + kEpilogueWarps * kStagingBytes + 1024;
constexpr int kSlots = 4;                                // tiles announced ahead
constexpr int kMaxTargets = 1024;
constexpr int kNoTarget = INT_MAX;
constexpr int kMaxJobs = 3;

enum { kForward = 0, kLogitGrad = 1, kHiddenGrad = 2, kWeightGrad = 3 };

// One matrix product C (m x n) = A B^T over k: tensor maps with boxes of 64 x 64 elements, and what becomes of C.
enum { kOut16 = 0, kOutF32 = 1, kOutAddF32 = 2 };

struct __align__(64) HeadJob {
    CUtensorMap a, b, out;   // out: boxes of 32 rows x 64 bytes
    int a_mn, b_mn;          // the operand lies with its rows (not k) contiguous
    int m_tiles, n_tiles, k_steps, band;
    long long columns;       // of C
    int halves, cols;        // accumulators of a tile, and their columns: 256 x 512, 256 x 256 or 256 x 128 tiles
    int splits, split_steps; // parts of the contraction, each a tile of its own
    int plane;               // few tokens: dz comes in two planes, the second one this many rows on; 0: in one
    int plane_steps;         // dW: contraction steps of a plane
    int kind;
    int vocab;               // entries of the vocabulary this job is about (all, or a piece's)
    long long v0;            // first of them
    void *out_ptr;           // C is written through `out`, or, where its rows are not 16-byte aligned, by plain stores
    long long out_stride;
    int out_rows, out_cols, out_parts, out_mode, out_plain;
    int out_bulk;            // columns in whole 16-byte granules: a bulk store writes no less
};

struct HeadParams {
    HeadJob job[kMaxJobs];
    int n_jobs, tiles, stages;
    int n;                   // tokens
    long long vocab_total;
    float c2;                // log2(e) / T
    // targets: labels (k == 0), or k sorted entries per row, [k][n]
    const long long *labels;
    const int *target_index;
    const float *target_q;
    int k;
    // forward
    float2 *partial;         // [tile columns][n]: (maximum in log2 units, sum)
    int parts;
    float *target_z;         // [max(k, 1)][n]
    // gradients
    const float *lse, *grad, *entropy, *scale;
    float temperature;
    int *next_tile;          // counter of tiles handed out beyond the first round; NULL: fixed rounds
    int *clear;              // counters of the launches after this one
    int n_clear;
    unsigned int *status;
    unsigned polls;          // of a wait before it gives up
};

// ---- PTX ----------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t addr_in(uint32_t a, uint32_t rank)  // the same variable in a CTA of the pair
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t leader_addr(uint32_t a) { return addr_in(a, 0); }
__device__ __forceinline__ void cluster_sync_all()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ bool barrier_test(uint32_t bar, uint32_t parity)  // without waiting
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool barrier_try_cluster(uint32_t bar, uint32_t parity)  // sees what the peer wrote before arriving
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ void barrier_arrive_in(uint32_t bar, uint32_t rank)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr_in(bar, rank)) : "memory");
}
// An arrival that publishes no memory: what it orders are TMEM reads (by their own fence) and values already used.
__device__ __forceinline__ void barrier_arrive_leader(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_addr(bar)) : "memory");
}
__device__ __forceinline__ void store_in(uint32_t addr, int value, uint32_t rank)
{
    asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(addr_in(addr, rank)), "r"(value) : "memory");
}
// `bytes` of a stage whose copies were announced and will not come
__device__ __forceinline__ void barrier_complete(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
        "[%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void mma_f16(uint32_t tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_commit_both(uint32_t bar)  // arrives on both CTAs' barrier when the MMAs so far are done
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
        "h"((uint16_t)3)
        : "memory");
}
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
        "%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
// The loaded registers pass through the wait, so that nothing reads them before it.
__device__ __forceinline__ void tmem_wait_load(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                   "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                   "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])::"memory");
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// One thread of the converged warp, the same one each time; its branch is known to be taken by a single thread.
__device__ __forceinline__ bool elect_one()
{
    uint32_t is;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xFFFFFFFF;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(is));
    return is != 0;
}
__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Shared-memory descriptor of an operand stage, 128-byte swizzle.  K-major: rows of 128 bytes, groups of 8 rows
// 1024 bytes apart.  MN-major: per k a run of 64 elements (128 bytes), groups of 8 k 1024 bytes apart, the next
// 64 elements of the row index one box further.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, int mn)
{
    const uint64_t lead = mn ? (uint64_t)(kBoxBytes >> 4) : 1u;
    return (uint64_t)((addr >> 4) & 0x3FFFu) | (lead << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

struct TilePos {
    int job, m, n, split, k0, steps;
};
// Tiles of a job, part by part of the contraction, in bands of `band` tile rows, a band column by column: what runs
// at a time shares its operands in L2.
__device__ __forceinline__ TilePos tile_pos(const HeadParams &p, int t)
{
    TilePos r;
    r.job = 0;
    int area = p.job[0].m_tiles * p.job[0].n_tiles;
    while (r.job + 1 < p.n_jobs && t >= area * p.job[r.job].splits) {
        t -= area * p.job[r.job].splits;
        ++r.job;
        area = p.job[r.job].m_tiles * p.job[r.job].n_tiles;
    }
    const HeadJob &j = p.job[r.job];
    r.split = t / area;
    t -= r.split * area;
    r.k0 = r.split * j.split_steps;
    r.steps = min(j.split_steps, j.k_steps - r.k0);
    const int per = j.band * j.n_tiles, b = t / per, i = t - b * per, rows = min(j.band, j.m_tiles - b * j.band);
    r.n = i / rows;
    r.m = b * j.band + i - r.n * rows;
    return r;
}

__device__ __forceinline__ void store_shared16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap *map, int x, int y, int z, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x),
                 "r"(y), "r"(z), "r"(src)
                 : "memory");
}
__device__ __forceinline__ void add_box(const CUtensorMap *map, int x, int y, int z, uint32_t src)
{
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map),
                 "r"(x), "r"(y), "r"(z), "r"(src)
                 : "memory");
}

// z[i], bit by bit of i: 31 selections
__device__ __forceinline__ float pick32(const uint32_t (&z)[32], int i)
{
    uint32_t v[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = i & 16 ? z[j + 16] : z[j];
#pragma unroll
    for (int half = 8; half; half >>= 1)
#pragma unroll
        for (int j = 0; j < half; ++j) v[j] = i & half ? v[j + half] : v[j];
    return __uint_as_float(v[0]);
}
__device__ __forceinline__ void subtract32(float (&z)[32], int i, float x)
{
#pragma unroll
    for (int j = 0; j < 32; ++j) z[j] -= i == j ? x : 0.0f;
}

// What rounding to T leaves of the values
template <typename T>
__device__ __forceinline__ void remainders(float (&z)[32])
{
#pragma unroll
    for (int j = 0; j < 32; ++j) z[j] -= to_f32(from_f32<T>(z[j]));
}

// A row's targets from a column on, in ascending order; entry j of the rows lies at [j][row], so that a warp's rows, whose
// places differ little, share the sectors they read.  The entry after the next is loaded ahead.
struct Targets {
    int j, next, after;
    __device__ __forceinline__ int at(const HeadParams &p, int i, int row) const
    {
        return i < p.k ? p.target_index[i * p.n + row] : kNoTarget;
    }
    __device__ __forceinline__ void start(const HeadParams &p, int row, int col, bool live)
    {
        j = 0;
        next = after = kNoTarget;
        if (!live) return;
        int hi = p.k;
        while (j < hi) {
            const int mid = (j + hi) >> 1;
            if (p.target_index[mid * p.n + row] < col) j = mid + 1; else hi = mid;
        }
        next = at(p, j, row);
        after = at(p, j + 1, row);
    }
    __device__ __forceinline__ void advance(const HeadParams &p, int row)
    {
        next = after;
        ++j;
        after = at(p, j + 1, row);
    }
    __device__ __forceinline__ void skip_to(const HeadParams &p, int col, int row)
    {
        while (next < col) advance(p, row);
    }
};

// A warp's 32 rows x 64 bytes on their way to global memory: staged in shared memory in the 64-byte swizzle (the
// 16-byte piece c of row r lies at c ^ (r / 2 & 3), so neither side meets a bank conflict), then one bulk store per box.
// Stores straight from the rows' registers take 1.6 cycles per 16 bytes of a row, 6700 cycles per 128 x 256 accumulator.
template <typename T>
struct RowsOut {
    uint32_t buf;
    int lane;
    __device__ __forceinline__ uint32_t piece(int i) const { return buf + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4); }
    __device__ __forceinline__ void put16(const float (&z)[32]) const  // 32 columns
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            store_shared16(piece(i), pack2<T>(z[8 * i], z[8 * i + 1]), pack2<T>(z[8 * i + 2], z[8 * i + 3]),
                           pack2<T>(z[8 * i + 4], z[8 * i + 5]), pack2<T>(z[8 * i + 6], z[8 * i + 7]));
    }
    template <int PART>
    __device__ __forceinline__ void put32(const float (&z)[32]) const  // columns 16 PART .. 16 PART + 15
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            store_shared16(piece(i), __float_as_uint(z[16 * PART + 4 * i]), __float_as_uint(z[16 * PART + 4 * i + 1]),
                           __float_as_uint(z[16 * PART + 4 * i + 2]), __float_as_uint(z[16 * PART + 4 * i + 3]));
    }
    __device__ __forceinline__ void wait_free() const  // the last box has left the buffer
    {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
    }
    // row0, col: of the box in C
    __device__ __forceinline__ void flush(const HeadJob &j, int row0, int col, int split) const
    {
        if (!j.out_plain) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0 && row0 < j.out_rows && col < j.out_bulk &&
                RSDGC_IN_BOUNDS(row0 >= 0 && col >= 0 && split >= 0 && split < j.out_parts &&
                                col % (j.out_mode == kOut16 ? 8 : 4) == 0)) {
                if (j.out_mode == kOutAddF32)
                    add_box(&j.out, col, row0, split, buf);
                else
                    store_box(&j.out, col, row0, split, buf);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
            // the values of a row's last, partial granule, from the lane's own row of the box
            const int elems = j.out_mode == kOut16 ? 32 : 16;
            if (j.out_bulk < j.out_cols && col < j.out_cols && col + elems > j.out_bulk && row0 + lane < j.out_rows)
                for (int c = max(col, j.out_bulk); c < min(col + elems, j.out_cols); ++c) {
                    const long long at = (long long)(row0 + lane) * j.out_stride + c;
                    if (!RSDGC_IN_BOUNDS(row0 >= 0 && c >= 0 && c < j.out_cols)) continue;
                    if (j.out_mode == kOut16) {
                        uint16_t v;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(piece((c - col) >> 3) + ((c - col) & 7) * 2));
                        ((uint16_t *)j.out_ptr)[at] = v;
                    } else {
                        float v;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(piece((c - col) >> 2) + ((c - col) & 3) * 4));
                        ((float *)j.out_ptr)[at] = v;
                    }
                }
            return;
        }
        __syncwarp();
        const int rows = min(32, j.out_rows - row0);
        if (j.out_mode == kOut16) {  // a row per round, a column per lane
            uint16_t *dst = (uint16_t *)j.out_ptr + (long long)row0 * j.out_stride + col + lane;
            for (int r = 0; r < rows; ++r, dst += j.out_stride) {
                uint16_t v;
                asm volatile("ld.shared.u16 %0, [%1];"
                             : "=h"(v)
                             : "r"(buf + r * 64 + (((lane >> 3) ^ ((r >> 1) & 3)) << 4) + (lane & 7) * 2));
                if (col + lane < j.out_cols && RSDGC_IN_BOUNDS(row0 >= 0 && row0 + r < j.out_rows && col >= 0)) *dst = v;
            }
        } else {  // two rows per round
            const int c = lane & 15;
            for (int r = lane >> 4; r < rows; r += 2) {
                float v;
                asm volatile("ld.shared.f32 %0, [%1];"
                             : "=f"(v)
                             : "r"(buf + r * 64 + (((c >> 2) ^ ((r >> 1) & 3)) << 4) + (c & 3) * 4));
                if (col + c < j.out_cols && RSDGC_IN_BOUNDS(row0 >= 0 && row0 + r < j.out_rows && col >= 0))
                    ((float *)j.out_ptr)[(long long)(row0 + r) * j.out_stride + col + c] = v;
            }
        }
    }
};

// T: type of the operands (bfloat16 or binary16).  BACK: the launch's jobs are gradients.
template <bool BACK, typename T>
__global__ void __launch_bounds__(kHeadThreads, 1) k_head(const __grid_constant__ HeadParams p)
{
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], drain;
    __shared__ __align__(8) unsigned long long slot_full[kSlots], slot_empty[kSlots];
    __shared__ int slot_tile[kSlots];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int dead;
    // after a give-up: which CTAs had one; stages each CTA's producer issued, and its bytes in the latest of each place
    __shared__ int failed[2], issued[2], sent[2][kMaxStages];

    const uint32_t ring = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int stages = p.stages, stage_bytes = kRingBlocks / stages * kBlockBytes;

    if (warp == 0) {  // a lane per barrier
        if (lane < kMaxStages) {
            barrier_init(smem_addr(&full[lane]), 1);
            barrier_init(smem_addr(&empty[lane]), 1);
        } else if (lane < kMaxStages + 2) {
            barrier_init(smem_addr(&acc_full[lane - kMaxStages]), 1);
            barrier_init(smem_addr(&acc_empty[lane - kMaxStages]), 2 * kEpilogueWarps);
        } else if (lane < kMaxStages + 2 + kSlots) {
            barrier_init(smem_addr(&slot_full[lane - kMaxStages - 2]), 1);
            barrier_init(smem_addr(&slot_empty[lane - kMaxStages - 2]), 2 * (1 + kEpilogueWarps));
        } else if (lane == 31) {
            barrier_init(smem_addr(&drain), 1);
            dead = 0;
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3 && lane < 3 * p.n_jobs) {
        const HeadJob &j = p.job[lane / 3];
        const CUtensorMap *map = lane % 3 == 0 ? &j.a : lane % 3 == 1 ? &j.b : &j.out;
        if (lane % 3 < 2 || (BACK && !j.out_plain)) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_base))
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    tmem_fence_before();
    __syncthreads();
    cluster_sync_all();  // the peer's barriers exist before anything arrives on them
    tmem_fence_after();
    // what earlier kernels of the stream wrote may be touched from here on (each role calls it when it is set up)
    auto start = [&]() {
        grid_dependency_wait();
        grid_dependency_launch_next();
    };

    // Bounded: a wait that gives up marks the CTA dead, raises the status bit, and every role leaves its loop.
    auto give_up = [&]() -> bool {
        dead = 1;
        atomicOr(p.status, RSDGC_STATUS_TIMEOUT);
        return false;
    };
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
        for (unsigned i = 0; i < p.polls; ++i) {
            if (barrier_try(bar, parity)) return true;
            if (dead) return false;
        }
        return give_up();
    };
    // The pair's next tile, announced by the first CTA's producer `i` tiles after the first; -1 after a wait that gave up.
    auto next_tile = [&](int i) -> int {
        const uint32_t bar = smem_addr(&slot_full[i % kSlots]), parity = (uint32_t)(i / kSlots) & 1u;
        for (unsigned n = 0; n < p.polls; ++n) {
            if (barrier_try_cluster(bar, parity)) return *(volatile int *)&slot_tile[i % kSlots];
            if (dead) return -1;
        }
        give_up();
        return -1;
    };

    if (warp < 4) {
        auto wait_warp = [&](uint32_t bar, uint32_t ph) -> bool { return __all_sync(0xFFFFFFFFu, wait(bar, ph)); };
        // ---- producer, in both CTAs; all bytes count on the first CTA's barriers.  As the MMAs, the copies are issued by
        // one elected thread of a warp that walks together: a thread of a diverged warp takes some 200 cycles for each.
        if (warp == 0) {
            int stage = 0, it = 0;
            uint32_t parity = 0;
            bool ok = true;
            TilePos tp = tile_pos(p, pair);
            start();
            asm volatile("fence.proxy.async.global;" ::: "memory");  // TMA reads what ordinary stores wrote
            for (int t = pair, i = 0; t < p.tiles; ++i) {
                // the tile after this one: asked for here, announced behind this one's loads
                int after = 0;
                if (rank == 0 && lane == 0) after = p.next_tile ? pairs + atomicAdd(p.next_tile, 1) : t + pairs;
                if (i) tp = tile_pos(p, t);
                const HeadJob &j = p.job[tp.job];
                const int halves = j.halves, a_mn = j.a_mn, b_mn = j.b_mn;
                const uint32_t bytes = 2u * (uint32_t)(kBlockBytes + halves * j.cols * kStepK);
                // dh from two planes: a tile's second half is the second plane's rows
                const int ra = tp.m * kTile + (int)rank * (j.plane && !a_mn ? j.plane : kHalf);
                const int rb = tp.n * halves * j.cols + (int)rank * (j.cols >> 1);
                const bool whole = j.cols == kTile;  // of an accumulator's columns a CTA holds half: one box or two
                // coordinates of a box: (k, row), or (row, k) where the rows are contiguous
                for (int k = 0; k < tp.steps; ++k) {
                    ok = wait_warp(smem_addr(&empty[stage]), parity ^ 1u);
                    if (!ok) break;
                    const uint32_t bar = leader_addr(smem_addr(&full[stage])), dst = ring + stage * stage_bytes;
                    int kc = (tp.k0 + k) * kStepK, ka = kc;
                    if (a_mn && j.plane && tp.k0 + k >= j.plane_steps) {  // dW: the second plane, the same tokens again
                        kc -= j.plane_steps * kStepK;
                        ka = j.plane + kc;
                    }
                    // a row coordinate in front of a contiguous row index starts a copy: 16-byte boundaries
                    if (elect_one() && RSDGC_IN_BOUNDS(kc >= 0 && ka >= 0 && ra >= 0 && rb >= 0 && (!a_mn || ra % 64 == 0) &&
                                                       (!b_mn || rb % 64 == 0) && (a_mn || ka % 64 == 0) && (b_mn || kc % 64 == 0) &&
                                                       stage < stages && tp.job < p.n_jobs && tp.m < j.m_tiles && tp.n < j.n_tiles)) {
                        if (rank == 0) barrier_expect(smem_addr(&full[stage]), bytes);
                        sent[rank][stage] = (int)(bytes / 2);
                        if (a_mn) {
                            load_box(dst, &j.a, ra, ka, bar);
                            load_box(dst + kBoxBytes, &j.a, ra + 64, ka, bar);
                        } else {
                            load_box(dst, &j.a, kc, ra, bar);
                            load_box(dst + kBoxBytes, &j.a, kc, ra + 64, bar);
                        }
                        if (b_mn) {
                            for (int h = 0; h < halves; ++h) {
                                load_box(dst + (1 + h) * kBlockBytes, &j.b, rb + h * kTile, kc, bar);
                                if (whole) load_box(dst + (1 + h) * kBlockBytes + kBoxBytes, &j.b, rb + h * kTile + 64, kc, bar);
                            }
                        } else {
                            for (int h = 0; h < halves; ++h) {
                                load_box(dst + (1 + h) * kBlockBytes, &j.b, kc, rb + h * kTile, bar);
                                if (whole) load_box(dst + (1 + h) * kBlockBytes + kBoxBytes, &j.b, kc, rb + h * kTile + 64, bar);
                            }
                        }
                    }
                    __syncwarp();
                    ++it;
                    if (++stage == stages) {
                        stage = 0;
                        parity ^= 1u;
                    }
                }
                if (!ok) break;
                if (rank == 0) {
                    ok = wait_warp(smem_addr(&slot_empty[i % kSlots]), ((uint32_t)(i / kSlots) & 1u) ^ 1u);
                    if (!ok) break;
                    after = __shfl_sync(0xFFFFFFFFu, after, 0);
                    if (elect_one()) {
                        for (uint32_t r = 0; r < 2; ++r) {
                            store_in(smem_addr(&slot_tile[i % kSlots]), after, r);
                            barrier_arrive_in(smem_addr(&slot_full[i % kSlots]), r);
                        }
                    }
                    __syncwarp();
                    t = after;
                } else {
                    t = next_tile(i);
                    ok = __all_sync(0xFFFFFFFFu, t >= 0);
                    if (!ok) break;
                    if (elect_one()) barrier_arrive_leader(smem_addr(&slot_empty[i % kSlots]));
                    __syncwarp();
                }
            }
            // the last commits arrive on this CTA's barriers: it must not leave before they have
            for (int i = 0; i < stages && ok; ++i) {
                ok = wait_warp(smem_addr(&empty[stage]), parity ^ 1u);
                if (++stage == stages) {
                    stage = 0;
                    parity ^= 1u;
                }
            }
            if (lane == 0) issued[rank] = it;
        }
        if (warp == 1 && rank == 0) {  // ---- MMA, the pair's first CTA: the warp walks together, one thread issues
            int stage = 0, sub = 0;    // sub: accumulators used so far; they alternate
            uint32_t parity = 0;
            bool ok = true;
            constexpr uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            for (int t = pair, i = 0; t < p.tiles; ++i) {
                const TilePos tp = tile_pos(p, t);
                const HeadJob &j = p.job[tp.job];
                const int a_mn = j.a_mn, b_mn = j.b_mn, steps = tp.steps, halves = j.halves;
                const uint32_t idesc = (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)a_mn << 15) |
                                       ((uint32_t)b_mn << 16) | ((uint32_t)(j.cols >> 3) << 17) |
                                       ((uint32_t)(kTile >> 4) << 24);
                const uint32_t da = a_mn ? 2048 >> 4 : 32 >> 4, db = b_mn ? 2048 >> 4 : 32 >> 4;
                const uint64_t a_base = operand_desc(ring, a_mn), b_base = operand_desc(ring + kBlockBytes, b_mn);
                auto issue = [&](int st, int h, int acc, int k) {
                    const uint64_t a = a_base + (uint32_t)(st * (stage_bytes >> 4));
                    const uint64_t b = b_base + (uint32_t)(st * (stage_bytes >> 4) + h * (kBlockBytes >> 4));
#pragma unroll
                    for (int i = 0; i < kStepK / 16; ++i)
                        mma_f16(tmem_base + (uint32_t)acc * kTile, a + i * da, b + i * db, idesc, (uint32_t)(k | i));
                };
                const int acc0 = sub & 1, acc1 = acc0 ^ 1;
                const uint32_t parity0 = (uint32_t)((sub >> 1) & 1) ^ 1u, parity1 = (uint32_t)(((sub + 1) >> 1) & 1) ^ 1u;
                ok = wait_warp(smem_addr(&acc_empty[acc0]), parity0);
                if (!ok) break;
                tmem_fence_after();
                // With two accumulators the second may still be read when the first is free: its products follow
                // as soon as it is, at the latest when the ring is full of stages that wait for it.
                bool second = halves == 1;
                int behind = 0, tail = stage, kb = 0;
                for (int k = 0; k < steps; ++k) {
                    ok = wait_warp(smem_addr(&full[stage]), parity);
                    if (!ok) break;
                    if (elect_one()) {
                        issue(stage, 0, acc0, k);
                        if (k + 1 == steps) mma_commit_both(smem_addr(&acc_full[acc0]));
                    }
                    __syncwarp();
                    ++behind;
                    if (!second) {
                        if (behind == stages || k + 1 == steps) {
                            ok = wait_warp(smem_addr(&acc_empty[acc1]), parity1);
                            if (!ok) break;
                            second = true;
                        } else {
                            second = __all_sync(0xFFFFFFFFu, barrier_test(smem_addr(&acc_empty[acc1]), parity1));
                        }
                        if (second) tmem_fence_after();
                    }
                    for (; second && behind; --behind, ++kb) {
                        if (elect_one()) {
                            if (halves == 2) issue(tail, 1, acc1, kb);
                            mma_commit_both(smem_addr(&empty[tail]));
                        }
                        __syncwarp();
                        if (++tail == stages) tail = 0;
                    }
                    if (++stage == stages) {
                        stage = 0;
                        parity ^= 1u;
                    }
                }
                if (!ok) break;
                if (halves == 2 && elect_one()) mma_commit_both(smem_addr(&acc_full[acc1]));
                __syncwarp();
                sub += halves;
                t = next_tile(i);
                ok = __all_sync(0xFFFFFFFFu, t >= 0);
                if (!ok) break;
                if (elect_one()) barrier_arrive_leader(smem_addr(&slot_empty[i % kSlots]));
                __syncwarp();
            }
        }
    } else {  // ---- epilogue: a thread owns one row and a quarter of an accumulator's columns
        const int quad = warp & 3, quarter = (warp - 4) >> 2;
        const float c2 = p.c2;
        const RowsOut<T> out = {ring + kRingBlocks * kBlockBytes + (warp - 4) * kStagingBytes, lane};
        int sub = 0;
        bool ok = true;
        // The four warps of a quad meet at a named barrier, which has no limit, once per accumulator of the forward pass.  So a
        // warp that leaves its loop early (`dead` is set by then) arrives on the barrier that the others meet at next; they
        // see `dead` behind it and leave too.
        auto leave_quad = [&]() {
            if (!BACK) asm volatile("bar.arrive %0, 128;" ::"r"(1 + quad) : "memory");
        };
        TilePos tp = tile_pos(p, pair);
        start();
        if (BACK && blockIdx.x == 0)
            for (int i = threadIdx.x - 128; i < p.n_clear; i += 32 * kEpilogueWarps) p.clear[i] = 0;
        for (int t = pair, i = 0; t < p.tiles; ++i) {
            if (i) tp = tile_pos(p, t);
            const HeadJob &j = p.job[tp.job];
            const int row0 = tp.m * kTile + (int)rank * kHalf + quad * 32, row = row0 + lane;
            const bool live = row < p.n, logits = !BACK || j.kind == kLogitGrad;
            const int width = j.cols >> 2;          // columns of this thread: 64 or 32
            // what a row needs, loaded before the tile is ready
            [[maybe_unused]] float gs = 0.0f, l2 = 0.0f;
            [[maybe_unused]] Targets tg;
            [[maybe_unused]] int label = INT_MAX;   // relative to the job's first column
            const int v0 = (int)j.v0;
            if (logits) {
                const long long y = live && !p.k ? p.labels[row] : -1;
                if (p.k)
                    tg.start(p, row, v0 + tp.n * j.halves * j.cols + quarter * width, live);
                else if (y >= j.v0 && y < j.v0 + j.vocab)
                    label = (int)(y - j.v0);
                if (BACK && live) {
                    const bool wanted = p.k ? p.entropy[row] < INFINITY : y >= 0 && y < p.vocab_total;
                    gs = wanted ? p.grad[row] * p.temperature * p.scale[0] : 0.0f;
                    l2 = p.lse[row] * 1.4426950408889634f;
                }
            }
            const float back = BACK && !logits ? p.scale[1] : 1.0f;
            // where the rows go: dh of the second plane is a part of its own
            const bool apart = BACK && j.plane && j.kind == kHiddenGrad;
            [[maybe_unused]] const int out_row0 = apart ? quad * 32 : row0, out_part = apart ? 2 * tp.split + (int)rank : tp.split;
            for (int h = 0; h < j.halves; ++h, ++sub) {
                const int acc = sub & 1;
                const int col0 = (tp.n * j.halves + h) * j.cols + quarter * width;
                const uint32_t src = tmem_base + (uint32_t)acc * kTile + quarter * width + ((uint32_t)(quad * 32) << 16);
                if (logits && p.k) tg.skip_to(p, v0 + col0, row);
                ok = __all_sync(0xFFFFFFFFu, wait(smem_addr(&acc_full[acc]), (uint32_t)((sub >> 1) & 1)));
                if (!ok) break;
                tmem_fence_after();
                [[maybe_unused]] float m = -INFINITY, s = 0.0f;
                // A loop of 32 columns that stays rolled: unrolled over all columns the code outgrows the
                // instruction cache and fetching it takes longer (5000 cycles per accumulator) than running it.
#pragma unroll 1
                for (int at = 0; at < width; at += 32) {
                    const int col = col0 + at;
                    uint32_t raw[32];
                    __syncwarp();  // lanes part over their rows' targets; the load is one of the whole warp
                    tmem_load32(src + at, raw);
                    tmem_wait_load(raw);
                    if (at + 32 == width) {  // the accumulator is read: the tile after the next may overwrite it
                        tmem_fence_before();
                        __syncwarp();
                        if (lane == 0) barrier_arrive_leader(smem_addr(&acc_empty[acc]));
                    }
                    if constexpr (!BACK) {
                        if (p.k) {
                            while (tg.next < col + 32) {
                                if (RSDGC_IN_BOUNDS(tg.j >= 0 && tg.j < p.k && row < p.n && tg.next >= col))
                                    p.target_z[tg.j * p.n + row] = pick32(raw, tg.next - col);
                                tg.advance(p, row);
                            }
                        } else if (label >= col && label < col + 32) {
                            if (RSDGC_IN_BOUNDS(row < p.n)) p.target_z[row] = pick32(raw, label - col);
                        }
                        if (col + 32 > j.vocab) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (col + i >= j.vocab) raw[i] = 0xFF800000u;  // -inf
                        }
                        // two and four chains, so that their latencies overlap
                        float top[2] = {__uint_as_float(raw[0]), __uint_as_float(raw[1])};
#pragma unroll
                        for (int i = 2; i < 30; i += 4) {
                            top[0] = max3(top[0], __uint_as_float(raw[i]), __uint_as_float(raw[i + 1]));
                            top[1] = max3(top[1], __uint_as_float(raw[i + 2]), __uint_as_float(raw[i + 3]));
                        }
                        top[0] = max3(top[0], __uint_as_float(raw[30]), __uint_as_float(raw[31]));
                        const float now = max3(m, top[0] * c2, top[1] * c2);
                        const float ref = now == -INFINITY ? 0.0f : now;
                        const float2 cc = make_float2(c2, c2), rr = make_float2(-ref, -ref);
                        float2 add[4];
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const float2 x = fma2(make_float2(__uint_as_float(raw[i]), __uint_as_float(raw[i + 1])), cc, rr);
                            const float2 y = make_float2(exp2_approx(x.x), exp2_approx(x.y));
                            add[(i >> 1) & 3] = i < 8 ? y : add2(add[(i >> 1) & 3], y);
                        }
                        const float2 sum = add2(add2(add[0], add[1]), add2(add[2], add[3]));
                        s = fmaf(s, exp2_approx(m - ref), sum.x + sum.y);
                        m = now;
                    } else {
                        float z[32];
                        if (logits) {
                            const float2 cc = make_float2(c2, c2), ll = make_float2(-l2, -l2), gg = make_float2(gs, gs);
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const float2 x = fma2(make_float2(__uint_as_float(raw[i]), __uint_as_float(raw[i + 1])), cc, ll);
                                const float2 y = mul2(make_float2(exp2_approx(x.x), exp2_approx(x.y)), gg);
                                z[i] = y.x;
                                z[i + 1] = y.y;
                            }
                            if (p.k) {
                                while (tg.next < v0 + col + 32) {
                                    if (RSDGC_IN_BOUNDS(tg.j >= 0 && tg.j < p.k && row < p.n && tg.next >= v0 + col))
                                        subtract32(z, tg.next - v0 - col, gs * p.target_q[tg.j * p.n + row]);
                                    tg.advance(p, row);
                                }
                            } else if (label >= col && label < col + 32) {
                                subtract32(z, label - col, gs);
                            }
                            if (col + 32 > j.vocab || gs == 0.0f) {
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (col + i >= j.vocab || gs == 0.0f) z[i] = 0.0f;
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) z[i] = __uint_as_float(raw[i]) * back;
                        }
                        // dz leaves in 16 bits, as both products' operand: their sums run over it in binary32
                        out.wait_free();
                        if (j.out_mode == kOut16) {
                            out.put16(z);
                        } else {
                            out.template put32<0>(z);
                            out.flush(j, out_row0, col, out_part);
                            out.wait_free();
                            out.template put32<1>(z);
                        }
                        out.flush(j, out_row0, j.out_mode == kOut16 ? col : col + 16, out_part);
                        if (logits && j.plane) {
                            remainders<T>(z);
                            out.wait_free();
                            out.put16(z);
                            out.flush(j, row0, col, 1);
                        }
                    }
                }
                if constexpr (!BACK) {  // the row's four quarters are joined before they leave
                    const uint32_t slot = ring + kRingBlocks * kBlockBytes + ((sub & 1) * 4 * kHalf + quad * 32 + lane) * 8;
                    asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(slot + quarter * kHalf * 8), "f"(m), "f"(s) : "memory");
                    asm volatile("bar.sync %0, 128;" ::"r"(1 + quad) : "memory");
                    ok = __all_sync(0xFFFFFFFFu, !dead);
                    if (!ok) break;
                    const int part = tp.n * j.halves + h;
                    if (quarter == 0 && live && part < p.parts) {
#pragma unroll
                        for (int q = 1; q < 4; ++q) {
                            float om, os;
                            asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(om), "=f"(os) : "r"(slot + q * kHalf * 8));
                            const float now = fmaxf(m, om), ref = now == -INFINITY ? 0.0f : now;
                            s = s * exp2_approx(m - ref) + os * exp2_approx(om - ref);
                            m = now;
                        }
                        p.partial[(long long)part * p.n + row] = make_float2(m, s);
                    }
                }
            }
            if (!ok) break;
            t = next_tile(i);
            ok = __all_sync(0xFFFFFFFFu, t >= 0);
            if (!ok) break;
            if (lane == 0) barrier_arrive_leader(smem_addr(&slot_empty[i % kSlots]));
        }
        if (!ok) leave_quad();
        if (BACK && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
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

// ---- the small kernels around the tiles -----------------------------------------------------------
// Latency bounds them all: a few dependent loads and a launch.  Alone and with cold caches, at 2048 x 32000 x 2048:
// k_head_targets with 64 targets 8.7 us, k_head_scale for labels 6.1, k_head_join 6.7, k_head_hidden_sum 11.9 (two parts, 42 MB);
// in a stream each starts while the one before it ends.

// Top logits -> per row the sorted vocabulary indices with their probabilities q (binary32 softmax of the k
// logits / T) and sum q log q.  Entries with a negative index are left out; a row without entries gets +inf
// (no loss), one with an index beyond the vocabulary NaN (its loss is NaN, it has no gradient).  A warp per row.  The
// (index, place) pairs are ordered by counting smaller ones, k^2 / 32 steps, up to kCountTargets of them; beyond, by a
// bitonic network of `wide` >= k places, a power of two.  (Forward call, all kernels: 64 x 8000 x 512 with k = 64 16.0 us
// counted, 16.7 sorted; 2048 x 32000 x 512 with k = 512 297 us counted, 163 sorted.)
constexpr int kPrepWarps = 4;
constexpr int kCountTargets = 64;
template <typename L>
__global__ void __launch_bounds__(32 * kPrepWarps)
k_head_targets(const long long *__restrict__ index, long long is, const L *__restrict__ logit, long long ls, int n, int k,
               int wide, long long vocab, float inv_t, int *__restrict__ out_index, float *__restrict__ out_q,
               float *__restrict__ entropy)
{
    extern __shared__ unsigned long long keys[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x * kPrepWarps + warp;
    grid_dependency_wait();
    grid_dependency_launch_next();
    if (row >= n) return;
    unsigned long long *const mine = keys + warp * wide;
    bool bad = false;
    float top = -INFINITY;
    for (int j = lane; j < wide; j += 32) {
        const long long i = j < k ? index[row * is + j] : -1;
        const bool in = i >= 0 && i < vocab;
        bad |= i >= vocab;
        mine[j] = (unsigned long long)(in ? (int)i : kNoTarget) << 32 | (unsigned)j;
        if (in) {
            const float u = to_f32(logit[row * ls + j]) * inv_t;
            top = u > top || u != u ? u : top;
        }
    }
    bad = __any_sync(0xFFFFFFFFu, bad);
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const float o = __shfl_xor_sync(0xFFFFFFFFu, top, d);
        top = o > top || o != o ? o : top;
    }
    __syncwarp();
    if (bad || top == -INFINITY) {  // nothing to aim at
        for (int j = lane; j < k; j += 32) out_index[j * n + row] = kNoTarget;
        if (lane == 0) entropy[row] = bad ? NAN : INFINITY;
        return;
    }
    float sum = 0.0f;
    for (int j = lane; j < k; j += 32)
        if ((int)(mine[j] >> 32) != kNoTarget) sum += expf(to_f32(logit[row * ls + j]) * inv_t - top);
    sum = warp_sum(sum);
    const float log_sum = logf(sum), inv = 1.0f / sum;
    float ent = 0.0f;
    auto emit = [&](int place, unsigned long long key) {
        const int i = (int)(key >> 32), from = (int)(unsigned)key;
        float q = 0.0f;
        if (i != kNoTarget) {
            const float u = to_f32(logit[row * ls + from]) * inv_t - top;
            q = expf(u) * inv;
            if (!(q == 0.0f)) ent = fmaf(q, u - log_sum, ent);
        }
        if (!RSDGC_IN_BOUNDS(place >= 0 && place < k && from >= 0 && from < (i == kNoTarget ? wide : k))) return;
        out_index[place * n + row] = i;
        out_q[place * n + row] = q;
    };
    if (k <= kCountTargets) {
        for (int j = lane; j < k; j += 32) {
            const unsigned long long key = mine[j];
            int place = 0;
            for (int o = 0; o < k; ++o) place += mine[o] < key;
            emit(place, key);
        }
    } else {
        for (int run = 2; run <= wide; run *= 2)
            for (int step = run / 2; step; step /= 2) {
                __syncwarp();
                for (int t = lane; t < wide / 2; t += 32) {
                    const int lo = 2 * t - (t & (step - 1)), hi = lo + step;
                    const unsigned long long a = mine[lo], b = mine[hi];
                    if ((a > b) == ((lo & run) == 0)) {
                        mine[lo] = b;
                        mine[hi] = a;
                    }
                }
            }
        __syncwarp();
        for (int j = lane; j < k; j += 32) emit(j, mine[j]);
    }
    ent = warp_sum(ent);
    if (lane == 0) entropy[row] = ent;
}

// dz is scaled so that the largest |grad| T becomes kTop, and scale[1] takes it back.  The largest gradient is mapped to a
// power of two, not only near one, because equal gradients (a mean over the tokens) are the rule: the entries at the labels,
// which carry most of dz, are then (p - 1) kTop, next to a power of two and rounded by almost nothing while p is small.
// Scaled by powers of two alone they are all rounded the same way, by up to half a unit, which no sum averages out (512 x
// 20000 x 256, gradients of 257 / 65536, bfloat16: 0.0036 relative error of dh against 0.0017 now).  For binary16 kTop = 2^13
// also keeps probabilities down to 2^-27 of the largest gradient's normal numbers.
constexpr float kTop = 8192.0f;
__global__ void __launch_bounds__(1024)
k_head_scale(const float *__restrict__ grad, const long long *__restrict__ labels, const float *__restrict__ entropy, int n,
             long long vocab, float temperature, float *__restrict__ scale)
{
    __shared__ float part[32];
    grid_dependency_wait();
    grid_dependency_launch_next();
    float top = 0.0f;
    for (int i = threadIdx.x; i < n; i += 1024) {
        const bool wanted = labels ? labels[i] >= 0 && labels[i] < vocab : entropy[i] < INFINITY;
        if (wanted) top = fmaxf(top, fabsf(grad[i]));
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 32; ++i) top = fmaxf(top, part[i]);
        top *= temperature;
        if (!(top > 0.0f && top < INFINITY)) top = kTop;
        if (top < 0x1p-100f) top = 0x1p-100f;  // kTop / top stays in range
        scale[0] = kTop / top;
        scale[1] = top / kTop;
    }
}

// Joins a row's partial maxima and sums (one per accumulator, 128 or 256 columns) to its log-sum-exp, and forms the loss.  Eight rows
// per CTA; the partials of a row are dealt to 32 threads, four loads at a time.
constexpr int kJoinRows = 8;
__global__ void __launch_bounds__(256)
k_head_join(const float2 *__restrict__ partial, int parts, int n, const long long *__restrict__ labels, long long vocab,
            const int *__restrict__ target_index, const float *__restrict__ target_q, const float *__restrict__ target_z,
            const float *__restrict__ entropy, int k, float inv_t, float z_scale, float *__restrict__ loss,
            float *__restrict__ lse)
{
    __shared__ float sm[8][kJoinRows], ss[8][kJoinRows], row_lse[kJoinRows];
    const int r = threadIdx.x % kJoinRows, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row0 = blockIdx.x * kJoinRows;
    grid_dependency_wait();
    grid_dependency_launch_next();
    float m = -INFINITY, s = 0.0f;
    auto join = [&](float om, float os) {
        const float now = fmaxf(m, om), ref = now == -INFINITY ? 0.0f : now;
        s = s * exp2_approx(m - ref) + os * exp2_approx(om - ref);
        m = now;
    };
    if (row0 + r < n) {
        const float2 *src = partial + row0 + r;
        for (int i = threadIdx.x / kJoinRows; i < parts; i += 128) {
            float2 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                v[u] = i + 32 * u < parts ? src[(long long)(i + 32 * u) * n] : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int u = 0; u < 4; ++u) join(v[u].x, v[u].y);
        }
    }
#pragma unroll
    for (int d = kJoinRows; d < 32; d <<= 1) {
        const float om = __shfl_xor_sync(0xFFFFFFFFu, m, d), os = __shfl_xor_sync(0xFFFFFFFFu, s, d);
        join(om, os);
    }
    if (lane < kJoinRows) {
        sm[warp][lane] = m;
        ss[warp][lane] = s;
    }
    __syncthreads();
    if (threadIdx.x < kJoinRows && row0 + r < n) {
        for (int w = 0; w < 8; ++w)
            if (w != 0) join(sm[w][r], ss[w][r]);
        const float l = (m + log2f(s)) * 0.6931471805599453f;
        row_lse[r] = l;
        if (lse) lse[row0 + r] = l;
        if (!k) {
            const long long y = labels[row0 + r];
            loss[row0 + r] = y < 0 ? 0.0f : y >= vocab ? NAN : l - target_z[row0 + r] * z_scale;
        }
    }
    if (!k) return;
    __syncthreads();
    const int row = row0 + r;
    float cross = 0.0f;
    if (row < n)
        for (int j = threadIdx.x / kJoinRows; j < k; j += 32) {
            const int at = j * n + row;
            if (target_index[at] != kNoTarget) {
                const float q = target_q[at];
                if (!(q == 0.0f)) cross = fmaf(q, row_lse[r] - target_z[at] * z_scale, cross);
            }
        }
#pragma unroll
    for (int d = kJoinRows; d < 32; d <<= 1) cross += __shfl_xor_sync(0xFFFFFFFFu, cross, d);
    if (lane < kJoinRows) ss[warp][lane] = cross;
    __syncthreads();
    if (threadIdx.x < kJoinRows && row < n) {
        for (int w = 1; w < 8; ++w) cross += ss[w][r];
        const float e = entropy[row];
        loss[row] = e == INFINITY ? 0.0f : (e + cross) / (inv_t * inv_t);
    }
}

// dh = the sum of its parts, in order, rounded once: a thread per four columns.
template <typename T>
__global__ void __launch_bounds__(256)
k_head_hidden_sum(const float *__restrict__ sum, long long pitch, int parts, int n, int d, T *__restrict__ dh,
                  long long stride)
{
    grid_dependency_wait();
    grid_dependency_launch_next();
    const int row = blockIdx.y, col = 4 * (blockIdx.x * 256 + threadIdx.x);
    if (col >= d || !RSDGC_IN_BOUNDS(row < n && col + 4 <= pitch)) return;
    const float *src = sum + (long long)row * pitch + col;
    const long long slab = (long long)n * pitch;
    float4 t = *reinterpret_cast<const float4 *>(src);
#pragma unroll 8
    for (int i = 1; i < parts; ++i) {
        const float4 o = *reinterpret_cast<const float4 *>(src + i * slab);
        t.x += o.x;
        t.y += o.y;
        t.z += o.z;
        t.w += o.w;
    }
    T *dst = dh + (long long)row * stride + col;
    const float v[4] = {t.x, t.y, t.z, t.w};
    if (col + 4 <= d && ((uintptr_t)dst & 7) == 0) {
        *reinterpret_cast<uint2 *>(dst) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < d) dst[i] = from_f32<T>(v[i]);
    }
}

// ---- host ---------------------------------------------------------------------------------------
RSDGC_DEFINE_DEBUG_BOUNDS(head_debug_bounds)

namespace {

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                             const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn()
{
    static EncodeFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) == cudaSuccess &&
            r == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeFn>(p);
        else
            (void)cudaGetLastError();
    });
    return fn;
}

// rows x cols values of 16 bits, boxes of 64 x 64; what lies outside reads as zero
cudaError_t encode(CUtensorMap *map, int dtype, const void *base, long long rows, long long cols, long long stride)
{
    EncodeFn fn = encode_fn();
    if (!fn) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {64, 64}, one[2] = {1, 1};
    const CUresult r = fn(map, dtype == RSDGC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                          const_cast<void *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// C of a job: parts x rows x cols values of `elem` bytes in boxes of 32 rows x 64 bytes, the columns beyond whole 16-byte granules
// by plain stores; all of it by plain stores where rows do not start on 16-byte boundaries.  (A bulk store clips a box to the
// tensor by granules, not by elements: the rest of a granule would be overwritten with zeros.)
cudaError_t set_output(HeadJob &j, int mode, int dtype, void *base, long long rows, long long cols, long long stride,
                       long long parts = 1)
{
    const int elem = mode == kOut16 ? 2 : 4;
    j.out_mode = mode;
    j.out_ptr = base;
    j.out_stride = stride;
    j.out_rows = (int)rows;
    j.out_cols = (int)cols;
    j.out_parts = (int)parts;
    j.out_bulk = (int)(cols / (16 / elem) * (16 / elem));
    j.out_plain = !pointer_aligned(base, 16) || (stride * elem) % 16 != 0 || j.out_bulk == 0;
    if (j.out_plain || j.out_bulk < cols) {
        if (parts > 1 || mode == kOutAddF32) return cudaErrorInvalidValue;  // the workspace's rows are whole
        if (j.out_plain) return cudaSuccess;
    }
    EncodeFn fn = encode_fn();
    if (!fn) return cudaErrorNotSupported;
    const cuuint64_t dims[3] = {(cuuint64_t)j.out_bulk, (cuuint64_t)rows, (cuuint64_t)parts};
    const cuuint64_t strides[2] = {(cuuint64_t)stride * elem, (cuuint64_t)stride * elem * rows};
    const cuuint32_t box[3] = {(cuuint32_t)(64 / elem), 32, 1}, one[3] = {1, 1, 1};
    const CUresult r = fn(&j.out, mode != kOut16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                  : dtype == RSDGC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                        : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                          3, base, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
                          CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }
inline int tiles_of(int64_t a) { return (int)((a + kTile - 1) / kTile); }

// A piece of the vocabulary: dz (n x piece, 16 bits) of at most kPieceBytes, in two buffers (one is written while the
// other is read); never under kPieceMin columns, because every piece adds to dh once.  A launch ends on its longest
// tiles, so few large pieces are better than what L2 would hold: 8192 x 128000 x 4096 backward takes 19.8 / 19.0 /
// 18.7 ms with pieces of 64 / 128 / 256 MB (the last is not worth twice the memory).
constexpr int64_t kPieceBytes = 128ll << 20;
constexpr int64_t kPieceMin = 2048;
// With few tokens dh has few tiles, each with a contraction over the whole piece: it is cut into parts that are added
// up at the end, in order, so that about kSplitTiles tiles share a launch with dW's, none longer than the launch's fair
// share.  More parts cost more in sums than they balance (1023 x 50001 x 1000 backward: 431 us with one part, 294 with
// 3, 270 with 5, 275 with 10).
constexpr int64_t kSplitTiles = 37, kSplitSteps = 8;

// With few tokens there is little to average a rounding out over: a row of dW is one dz times a row of h where a token stands
// alone.  dz is then kept in two planes of 16 bits, the rounded values and what the rounding left (16 bits together in bfloat16,
// 22 in binary16).  Up to kHalf tokens that costs no product more: the second plane takes a tile's empty second half for dh, and
// as many contraction steps again for dW.  (Backward, in two planes and in one: 64 x 8000 x 512 binary16 30.5 and 27.8 us, 64 x
// 32000 x 4096 bfloat16 179 and 166, 128 x 32000 x 2048 115 and 97; relative errors of the gradients 1.0 and 1.4 to 2.2 times
// those of one rounding.)
constexpr int64_t kFewTokens = kHalf;

struct HeadLayout {
    int64_t piece, pieces, splits, planes;
    int64_t partial, target_z, index, q, entropy, scale, counter, dz[2], dh_sum, forward_bytes, bytes;
    int64_t dh_pitch;
};

HeadLayout head_layout(int64_t n, int64_t v, int64_t d, int64_t k)
{
    HeadLayout L{};
    L.planes = n <= kFewTokens ? 2 : 1;
    int64_t most = kPieceBytes / (2 * L.planes * (n > 0 ? n : 1)) / kTile * kTile;
    if (most < kPieceMin) most = kPieceMin;
    L.pieces = (v + most - 1) / most;
    L.piece = up((v + L.pieces - 1) / L.pieces, kTile);
    L.pieces = (v + L.piece - 1) / L.piece;
    L.dh_pitch = up(d, 4);
    const int64_t area = tiles_of(n) * ((tiles_of(d) + 1) / 2), steps = L.piece / kStepK;
    L.splits = area > 0 ? (kSplitTiles + area - 1) / area : 1;
    if (L.splits > steps / kSplitSteps) L.splits = steps / kSplitSteps;
    if (L.splits < 1) L.splits = 1;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t p = at;
        at = up(at + bytes, 256);
        return p;
    };
    L.target_z = take(4 * n * k);
    L.index = take(4 * n * k);
    L.q = take(4 * n * k);
    L.entropy = take(4 * n);
    L.scale = take(8);
    L.counter = take(4 * ((v + kPieceMin - 1) / kPieceMin));  // a piece each
    const int64_t shared = at;  // the forward pass's partials and the backward pass's dz share the rest
    L.partial = take(8 * n * ((v + kTile / 2 - 1) / (kTile / 2)));  // at most one per 128 columns
    L.forward_bytes = L.bytes = at;
    at = shared;
    L.dz[0] = take(2 * L.planes * n * L.piece);
    L.dz[1] = take(L.pieces > 1 ? 2 * L.planes * n * L.piece : 0);
    L.dh_sum = take(L.pieces > 1 || L.splits * L.planes > 1 ? 4 * n * L.dh_pitch * L.splits * L.planes : 0);
    if (at > L.bytes) L.bytes = at;
    return L;
}

// What a call of n tokens, or fewer, needs at most: fewer tokens may come in more parts, in two planes, or in fewer and larger
// pieces.  The layout's own sizes where they grow with n, bounds of the others'.
int64_t head_bytes(int64_t n, int64_t v, int64_t d, int64_t k)
{
    const HeadLayout L = head_layout(n, v, d, k);
    const int64_t few = n < kFewTokens ? n : kFewTokens, rows = n > 2 * few ? n : 2 * few;  // of dz's planes
    // dz: one buffer of the whole vocabulary, or two of at most a piece
    const int64_t whole = 2 * rows * up(v, kTile), least = 2 * rows * kPieceMin, piece = least > kPieceBytes ? least : kPieceBytes;
    int64_t dz = whole;
    if (whole > kPieceBytes && v > kPieceMin) {
        dz = whole + 2 * 2 * rows * kTile;
        if (dz > 2 * piece) dz = 2 * piece;
    }
    // dh's parts: n ceil(kSplitTiles / (m across)) rows for n <= m kTile tokens
    const int64_t across = (tiles_of(d) + 1) / 2, longest = up(v, kTile) / kStepK / kSplitSteps;
    int64_t most = (kSplitTiles + across - 1) / across;
    if (most > longest) most = longest > 1 ? longest : 1;
    int64_t parts = 2 * few * most;
    if (n > kFewTokens && (most > 1 || L.pieces > 1)) {
        const int64_t spread = (kTile * kSplitTiles + across - 1) / across + n, all = n * most < spread ? n * most : spread;
        if (all > parts) parts = all;
    }
    const int64_t back = L.partial + up(dz, 256) + 256 + up(4 * parts * L.dh_pitch, 256);
    return back > L.bytes ? back : L.bytes;
}

int head_check(int64_t n, int64_t v, int64_t d, int64_t k)
{
    if (n < 0 || v < 1 || d < 1 || k < 1) return RSDGC_ERR_INVALID;
    if (n > (1 << 24) || v > (1 << 28) || d > (1 << 20) || k > kMaxTargets || n * k > INT_MAX) return RSDGC_ERR_CAPACITY;
    return RSDGC_OK;
}

struct HeadCall {
    const void *hidden, *weight;
    int64_t hs, ws;
    const long long *labels;      // or
    const long long *top_index;
    const void *top_logit;
    int64_t is, ls;
    int32_t top_dtype;
    int64_t k;                    // 0: labels
    float temperature;
    int64_t n, v, d;
    int32_t dtype;
    unsigned char *workspace;
    cudaStream_t s;
};

int call_check(const HeadCall &c)
{
    int rc = head_check(c.n, c.v, c.d, c.k ? c.k : 1);
    if (rc) return rc;
    if (c.dtype != RSDGC_BF16 && c.dtype != RSDGC_F16) return RSDGC_ERR_INVALID;
    if (!(c.temperature > 0.0f) || !(c.temperature < INFINITY)) return RSDGC_ERR_INVALID;
    if (!c.weight || c.ws < c.d) return RSDGC_ERR_INVALID;
    if (c.k && !known_dtype(c.top_dtype)) return RSDGC_ERR_INVALID;
    if (c.n > 0) {
        if (!c.hidden || c.hs < c.d || !c.workspace) return RSDGC_ERR_INVALID;
        if (c.k ? !c.top_index || !c.top_logit || c.is < c.k || c.ls < c.k : !c.labels) return RSDGC_ERR_INVALID;
        if (!pointer_aligned(c.hidden, 16) || (c.hs & 7) || !pointer_aligned(c.workspace, 256) ||
            !pointer_aligned(c.labels, 8) || !pointer_aligned(c.top_index, 8) ||
            (c.k && !pointer_aligned(c.top_logit, dtype_bytes(c.top_dtype))))
            return RSDGC_ERR_ALIGNMENT;
    }
    if (!pointer_aligned(c.weight, 16) || (c.ws & 7)) return RSDGC_ERR_ALIGNMENT;
    return RSDGC_OK;
}

// Clusters of two that the device holds at a time; 0 and an error in *e if the kernel cannot run.
template <bool BACK, typename T>
int head_pairs(cudaError_t *e)
{
    static std::mutex mu;
    static int most[64];
    int dev = 0;
    *e = cudaGetDevice(&dev);
    if (*e != cudaSuccess) return 0;
    std::lock_guard<std::mutex> lock(mu);
    int &m = most[dev & 63];
    if (m) return m;
    *e = cudaFuncSetAttribute(k_head<BACK, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeadSmem);
    if (*e != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = (unsigned)current_device_sms();
    cfg.blockDim = kHeadThreads;
    cfg.dynamicSmemBytes = kHeadSmem;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 2;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    int n = 0;
    *e = cudaOccupancyMaxActiveClusters(&n, k_head<BACK, T>, &cfg);
    if (*e == cudaSuccess && n < 1) *e = cudaErrorLaunchOutOfResources;
    if (*e != cudaSuccess) return 0;
    return m = n;
}

// Tiles of 256 x 128, 256 x 256 or 256 x 512 (two accumulators) for a launch's jobs.  The wider the tile, the more products
// an operand block serves (48 bytes per cycle and SM at the full MMA rate for 512 columns, 64 for 256) and the more work
// the ring holds: 2048 x 32000 x 2048 takes 180 us forward and 560 backward with 512 columns throughout, 218 and 682 with 256,
// 402 and 1185 with 128.  The narrower, the more tiles there are to deal out: 64 x 8000 x 512 takes 19.1 and 48.6 us with 512
// columns, 11.8 and 31.0 with 256, 11.0 and 31.4 with 128, and 5 x 1000 x 256 15.8 and 36.7, 9.7 and 23.2, 8.9 and 19.6.
// Which is best follows from the cycles a tile takes (512 per contraction step and 256
// columns, some 3000 to empty an accumulator; 1.25 and 1.6 times that for the lost operand reuse of 256 and 128 columns)
// dealt to the pairs of CTAs.
void choose_columns(HeadParams &p, int pairs)
{
    double best = 0.0;
    int take = kTile;
    for (int wide = kTile / 2; wide <= 2 * kTile; wide *= 2) {
        double total = 0.0, longest = 0.0;
        long long tiles = 0;
        for (int i = 0; i < p.n_jobs; ++i) {
            const HeadJob &j = p.job[i];
            const int w = wide > kTile && j.columns <= kTile ? kTile : wide;
            const long long t = (long long)j.m_tiles * ((j.columns + w - 1) / w) * j.splits;
            const double part = (double)w / kTile, loss = w > kTile ? 1.0 : w == kTile ? 1.25 : 1.6;
            const double time = loss * part * (512.0 * j.split_steps + 3000.0);
            total += t * time;
            tiles += t;
            if (time > longest) longest = time;
        }
        // one job's tiles come in rounds, several jobs' fill one another's gaps
        const double rounds = p.n_jobs == 1 ? (double)((tiles + pairs - 1) / pairs) * longest : total / pairs;
        const double cost = rounds > longest ? rounds : longest;
        if (wide < kTile || cost <= best) best = cost, take = wide;
    }
    for (int i = 0; i < p.n_jobs; ++i) {
        HeadJob &j = p.job[i];
        const int w = take > kTile && j.columns <= kTile ? kTile : take;
        j.halves = w > kTile ? 2 : 1;
        j.cols = w < kTile ? w : kTile;
        j.n_tiles = (int)((j.columns + w - 1) / w);
    }
}

template <bool BACK, typename T>
cudaError_t launch_tiles(HeadParams &p, int *counter, cudaStream_t s)
{
    cudaError_t e = cudaSuccess;
    const int most = head_pairs<BACK, T>(&e);
    if (e != cudaSuccess) return e;
    choose_columns(p, most);
    auto length = [](const HeadJob &j) { return (long long)j.split_steps * j.halves * j.cols; };  // longest tiles first
    for (int a = 0; a < p.n_jobs; ++a)
        for (int b = a + 1; b < p.n_jobs; ++b)
            if (length(p.job[b]) > length(p.job[a])) std::swap(p.job[a], p.job[b]);
    long long tiles = 0;
    int halves = 1;
    for (int i = 0; i < p.n_jobs; ++i) {
        tiles += (long long)p.job[i].m_tiles * p.job[i].n_tiles * p.job[i].splits;
        if (p.job[i].halves > halves) halves = p.job[i].halves;
    }
    p.stages = kRingBlocks / (1 + halves);
    if (tiles > INT_MAX / 2) return cudaErrorInvalidValue;
    p.tiles = (int)tiles;
    p.parts = p.job[0].n_tiles * p.job[0].halves;
    p.next_tile = counter;
    const unsigned pairs = (unsigned)(tiles < most ? tiles : most);
    return launch_chained(k_head<BACK, T>, 2 * pairs, kHeadThreads, kHeadSmem, s, 2, p);
}

constexpr double kTruncationBf16 = 0.26, kTruncationF16 = 0.27;
constexpr int kBand = 16;
cudaError_t set_job(HeadJob &j, int kind, int dtype, const void *a, bool a_mn, long long ar, long long ac, long long as,
                    const void *b, bool b_mn, long long br, long long bc, long long bs, long long m, long long n, long long k)
{
    std::memset(&j, 0, sizeof j);
    j.kind = kind;
    j.a_mn = a_mn;
    j.b_mn = b_mn;
    j.k_steps = (int)((k + kStepK - 1) / kStepK);
    j.m_tiles = tiles_of(m);
    j.columns = n;  // cut into tiles by choose_columns()
    j.band = j.m_tiles < kBand ? j.m_tiles : kBand;
    j.splits = 1;
    j.split_steps = j.k_steps;
    const cudaError_t e = encode(&j.a, dtype, a, ar, ac, as);
    return e == cudaSuccess ? encode(&j.b, dtype, b, br, bc, bs) : e;
}

cudaError_t targets(const HeadCall &c, const HeadLayout &L)
{
    if (!c.k) return cudaSuccess;
    const unsigned grid = (unsigned)((c.n + kPrepWarps - 1) / kPrepWarps);
    int *oi = (int *)(c.workspace + L.index);
    float *oq = (float *)(c.workspace + L.q), *oe = (float *)(c.workspace + L.entropy);
    const float inv_t = 1.0f / c.temperature;
    int wide = 1;
    while (wide < c.k) wide *= 2;
    auto go = [&](auto t) {
        typedef decltype(t) T;
        return launch_chained(k_head_targets<T>, grid, 32 * kPrepWarps, (size_t)wide * kPrepWarps * 8, c.s, 1, c.top_index,
                              (long long)c.is, (const T *)c.top_logit, (long long)c.ls, (int)c.n, (int)c.k, wide, (long long)c.v,
                              inv_t, oi, oq, oe);
    };
    return c.top_dtype == RSDGC_F32 ? go(float{}) : c.top_dtype == RSDGC_BF16 ? go(__nv_bfloat16{}) : go(__half{});
}

void common_params(HeadParams &p, const HeadCall &c, const HeadLayout &L)
{
    p.n = (int)c.n;
    p.vocab_total = c.v;
    // The tensor core truncates its running sum, so that a step of 16 terms takes a part of 2^-24 off it, towards zero.  What a
    // whole sum loses depends on how it grows: per step and in 2^-24 of the final value 0.21 to 0.27 (bfloat16) or 0.22 to 0.28
    // (binary16) for terms of random signs, at every width from 256 to 2^20; 0.3 to 0.9 where the terms lean to one sign, 0.5
    // to 1.8 where all have one; 0.05 to 0.2 where most comes from the last eighth of the columns.  The exponent's factor puts
    // back what random signs lose (root mean square over 4096 bfloat16 columns 4.5e-6 of z without it, 2.2e-6 with it; leaning
    // 5.8e-6 and 1.8e-6), less than the other forms lose except for the last, where the factor is most of what is left (0.95e-6
    // without it, 3.0e-6 with it).  All of it lies within the products' bound, 2^-23 of |h| |W| per step.
    const double steps = (double)((c.d + 15) / 16), lost = c.dtype == RSDGC_BF16 ? kTruncationBf16 : kTruncationF16;
    p.c2 = (float)(1.4426950408889634 / c.temperature * (1.0 + lost * steps * 0x1p-24));
    p.labels = c.labels;
    p.k = (int)c.k;
    p.target_index = (const int *)(c.workspace + L.index);
    p.target_q = (const float *)(c.workspace + L.q);
    p.entropy = (const float *)(c.workspace + L.entropy);
    p.temperature = c.temperature;
}

int head_forward(const HeadCall &c, float *loss, float *lse)
{
    int rc = call_check(c);
    if (rc) return rc;
    if (c.n == 0) return RSDGC_OK;
    if (!loss) return RSDGC_ERR_INVALID;
    if (!pointer_aligned(loss, 4) || !pointer_aligned(lse, 4)) return RSDGC_ERR_ALIGNMENT;
    const HeadLayout L = head_layout(c.n, c.v, c.d, c.k ? c.k : 1);
    HeadParams p;
    std::memset(&p, 0, sizeof p);
    cudaError_t e = operators_ready();
    if (e == cudaSuccess) e = operator_status_ptr(&p.status);
    p.polls = operator_polls();
    common_params(p, c, L);
    p.n_jobs = 1;
    p.partial = (float2 *)(c.workspace + L.partial);
    p.target_z = (float *)(c.workspace + L.target_z);
    if (e == cudaSuccess)
        e = set_job(p.job[0], kForward, c.dtype, c.hidden, false, c.n, c.d, c.hs, c.weight, false, c.v, c.d, c.ws, c.n, c.v,
                    c.d);
    p.job[0].vocab = (int)c.v;
    if (e == cudaSuccess) e = targets(c, L);
    if (e == cudaSuccess)
        e = c.dtype == RSDGC_BF16 ? launch_tiles<false, __nv_bfloat16>(p, nullptr, c.s)
                                  : launch_tiles<false, __half>(p, nullptr, c.s);
    if (e == cudaSuccess)
        e = launch_chained(k_head_join, (unsigned)((c.n + kJoinRows - 1) / kJoinRows), 256, 0, c.s, 1, (const float2 *)p.partial,
                           p.parts, (int)c.n, c.labels, (long long)c.v, p.target_index, p.target_q,
                           (const float *)p.target_z, p.entropy, (int)c.k, 1.0f / c.temperature, p.c2 * 0.6931471805599453f, loss, lse);
    return operator_result(e);
}

struct HeadGrads {
    void *dh, *dw;
    long long dh_stride, dw_stride;
    int dw_dtype;
};

// Launch i computes piece i's dz and, from the piece before it, dh and dW: three products whose tiles share a queue,
// longest contraction first, so that the multiprocessors end together.  dh goes to binary32 sums unless one piece in one
// part is all there is: stored by the first piece, added to by the others (one bulk reduction per element and launch).
template <typename T>
cudaError_t backward_pieces(const HeadCall &c, const HeadLayout &L, HeadParams &p, const HeadGrads &g)
{
    const int planes = (int)L.planes;
    int parts = 1;  // of dh
    float *sum = (float *)(c.workspace + L.dh_sum);
    int *counter = (int *)(c.workspace + L.counter);
    for (int64_t i = 0; i <= L.pieces; ++i) {
        cudaError_t e = cudaSuccess;
        p.n_jobs = 0;
        auto rows = [&](int64_t at) { return c.v - at * L.piece < L.piece ? c.v - at * L.piece : L.piece; };
        auto weight = [&](int64_t at) { return (const unsigned char *)c.weight + at * L.piece * c.ws * 2; };
        auto buffer = [&](int64_t at) { return c.workspace + L.dz[at & 1]; };
        if (i < L.pieces) {
            HeadJob &j = p.job[p.n_jobs++];
            e = set_job(j, kLogitGrad, c.dtype, c.hidden, false, c.n, c.d, c.hs, weight(i), false, rows(i), c.d, c.ws, c.n,
                        rows(i), c.d);
            j.v0 = i * L.piece;
            j.vocab = (int)rows(i);
            j.plane = planes > 1 ? (int)c.n : 0;
            if (e == cudaSuccess) e = set_output(j, kOut16, c.dtype, buffer(i), c.n, L.piece, L.piece, planes);
        }
        if (i > 0 && e == cudaSuccess) {
            const int64_t at = i - 1, v = rows(at);
            const void *dz = buffer(at);
            // the tiles of dz are whole: zeros beyond the vocabulary, so the contraction may run over whole steps
            HeadJob &j = p.job[p.n_jobs++];
            e = set_job(j, kHiddenGrad, c.dtype, dz, false, planes * c.n, L.piece, L.piece, weight(at), true, v, c.d, c.ws, c.n, c.d, v);
            j.plane = planes > 1 ? (int)c.n : 0;
            j.split_steps = (j.k_steps + (int)L.splits - 1) / (int)L.splits;
            j.splits = (j.k_steps + j.split_steps - 1) / j.split_steps;
            if (at == 0) parts = planes * j.splits;  // the other pieces are no longer: they have no more parts
            if (e == cudaSuccess)
                e = L.pieces == 1 && parts == 1
                        ? set_output(j, kOut16, c.dtype, g.dh, c.n, c.d, g.dh_stride)
                        : set_output(j, at == 0 ? kOutF32 : kOutAddF32, c.dtype, sum, c.n, L.dh_pitch, L.dh_pitch, parts);
            if (e == cudaSuccess) {
                HeadJob &w = p.job[p.n_jobs++];
                e = set_job(w, kWeightGrad, c.dtype, dz, true, planes * c.n, L.piece, L.piece, c.hidden, true, c.n, c.d, c.hs, v, c.d,
                            c.n);
                if (planes > 1) {  // the tokens twice; what lies beyond them in a plane meets the zeros beyond them in h
                    w.plane = (int)c.n;
                    w.plane_steps = w.k_steps;
                    w.k_steps = w.split_steps = 2 * w.k_steps;
                }
                const bool wide = g.dw_dtype == RSDGC_F32;
                if (e == cudaSuccess)
                    e = set_output(w, wide ? kOutF32 : kOut16, c.dtype,
                                   (unsigned char *)g.dw + at * L.piece * g.dw_stride * (wide ? 4 : 2), v, c.d, g.dw_stride);
            }
        }
        if (e != cudaSuccess) return e;
        // the first launch has tiles of one length and deals them out in rounds; it clears the others' counters
        p.clear = counter;
        p.n_clear = i == 0 ? (int)L.pieces : 0;
        e = launch_tiles<true, T>(p, i == 0 ? nullptr : counter + i - 1, c.s);
        if (e != cudaSuccess) return e;
    }
    if (L.pieces == 1 && parts == 1) return cudaSuccess;
    const unsigned wide = (unsigned)((c.d + 1023) / 1024);
    cudaError_t e = cudaSuccess;
    for (int64_t row = 0; row < c.n && e == cudaSuccess; row += 32768) {  // rows of a grid
        const unsigned rows = (unsigned)(c.n - row < 32768 ? c.n - row : 32768);
        e = launch_chained(k_head_hidden_sum<T>, dim3(wide, rows), 256, 0, c.s, 1, (const float *)sum + row * L.dh_pitch,
                           (long long)L.dh_pitch, parts, (int)c.n, (int)c.d, (T *)g.dh + row * g.dh_stride, g.dh_stride);
    }
    return e;
}

int head_backward(const HeadCall &c, const float *lse, const float *grad, void *dh, int64_t dh_stride, void *dw,
                  int64_t dw_stride, int32_t dw_dtype)
{
    int rc = call_check(c);
    if (rc) return rc;
    if (!dw || dw_stride < c.d || (dw_dtype != c.dtype && dw_dtype != RSDGC_F32)) return RSDGC_ERR_INVALID;
    if (!pointer_aligned(dw, dtype_bytes(dw_dtype))) return RSDGC_ERR_ALIGNMENT;
    cudaError_t e = cudaSuccess;
    if (c.n == 0) {  // sums over nothing
        const size_t b = (size_t)dtype_bytes(dw_dtype);
        e = cudaMemset2DAsync(dw, (size_t)dw_stride * b, 0, (size_t)c.d * b, (size_t)c.v, c.s);
        return operator_result(e);
    }
    if (!lse || !grad || !dh || dh_stride < c.d) return RSDGC_ERR_INVALID;
    if (!pointer_aligned(lse, 4) || !pointer_aligned(grad, 4) || !pointer_aligned(dh, 2)) return RSDGC_ERR_ALIGNMENT;
    const HeadLayout L = head_layout(c.n, c.v, c.d, c.k ? c.k : 1);
    HeadParams p;
    std::memset(&p, 0, sizeof p);
    e = operators_ready();
    if (e == cudaSuccess) e = operator_status_ptr(&p.status);
    p.polls = operator_polls();
    common_params(p, c, L);
    p.lse = lse;
    p.grad = grad;
    if (e == cudaSuccess) e = targets(c, L);
    p.scale = (const float *)(c.workspace + L.scale);
    if (e == cudaSuccess)
        e = launch_chained(k_head_scale, 1, 1024, 0, c.s, 1, grad, c.labels, p.entropy, (int)c.n, (long long)c.v,
                           c.temperature, (float *)(c.workspace + L.scale));
    if (e == cudaSuccess) {
        const HeadGrads g = {dh, dw, dh_stride, dw_stride, dw_dtype};
        e = c.dtype == RSDGC_BF16 ? backward_pieces<__nv_bfloat16>(c, L, p, g) : backward_pieces<__half>(c, L, p, g);
    }
    return operator_result(e);
}

}  // namespace
}  // namespace rsdgc

using namespace rsdgc;

extern "C" int64_t rsdgc_head_workspace_bytes(int64_t n_tokens, int64_t vocab, int64_t width, int64_t n_targets)
{
    const int rc = head_check(n_tokens, vocab, width, n_targets);
    return rc ? rc : head_bytes(n_tokens, vocab, width, n_targets);
}

extern "C" int64_t rsdgc_head_forward_workspace_bytes(int64_t n_tokens, int64_t vocab, int64_t width, int64_t n_targets)
{
    const int rc = head_check(n_tokens, vocab, width, n_targets);
    return rc ? rc : head_layout(n_tokens, vocab, width, n_targets).forward_bytes;
}

extern "C" int rsdgc_head_loss_forward(const void *hidden_dev, int64_t hidden_stride, const void *weight_dev,
                                       int64_t weight_stride, const int64_t *labels_dev, float *loss_dev, float *lse_dev,
                                       int64_t n_tokens, int64_t vocab, int64_t width, int32_t dtype, void *workspace_dev,
                                       void *stream)
{
    OperatorRange range("rsdgc_head_loss_forward");
    const HeadCall c = {hidden_dev, weight_dev, hidden_stride, weight_stride, (const long long *)labels_dev, nullptr, nullptr,
                        0, 0, 0, 0, 1.0f, n_tokens, vocab, width, dtype, (unsigned char *)workspace_dev, (cudaStream_t)stream};
    return head_forward(c, loss_dev, lse_dev);
}

extern "C" int rsdgc_head_loss_backward(const void *hidden_dev, int64_t hidden_stride, const void *weight_dev,
                                        int64_t weight_stride, const int64_t *labels_dev, const float *lse_dev,
                                        const float *grad_loss_dev, void *dhidden_dev, int64_t dhidden_stride,
                                        void *dweight_dev, int64_t dweight_stride, int32_t dweight_dtype, int64_t n_tokens,
                                        int64_t vocab, int64_t width, int32_t dtype, void *workspace_dev, void *stream)
{
    OperatorRange range("rsdgc_head_loss_backward");
    const HeadCall c = {hidden_dev, weight_dev, hidden_stride, weight_stride, (const long long *)labels_dev, nullptr, nullptr,
                        0, 0, 0, 0, 1.0f, n_tokens, vocab, width, dtype, (unsigned char *)workspace_dev, (cudaStream_t)stream};
    return head_backward(c, lse_dev, grad_loss_dev, dhidden_dev, dhidden_stride, dweight_dev, dweight_stride, dweight_dtype);
}

extern "C" int rsdgc_head_distill_forward(const void *hidden_dev, int64_t hidden_stride, const void *weight_dev,
                                          int64_t weight_stride, const int64_t *top_index_dev, int64_t top_index_stride,
                                          const void *top_logit_dev, int64_t top_logit_stride, int32_t top_dtype,
                                          int64_t n_targets, float temperature, float *loss_dev, float *lse_dev,
                                          int64_t n_tokens, int64_t vocab, int64_t width, int32_t dtype,
                                          void *workspace_dev, void *stream)
{
    if (n_targets < 1) return RSDGC_ERR_INVALID;
    OperatorRange range("rsdgc_head_distill_forward");
    const HeadCall c = {hidden_dev, weight_dev, hidden_stride, weight_stride, nullptr, (const long long *)top_index_dev,
                        top_logit_dev, top_index_stride, top_logit_stride, top_dtype, n_targets, temperature, n_tokens, vocab,
                        width, dtype, (unsigned char *)workspace_dev, (cudaStream_t)stream};
    return head_forward(c, loss_dev, lse_dev);
}

extern "C" int rsdgc_head_distill_backward(const void *hidden_dev, int64_t hidden_stride, const void *weight_dev,
                                           int64_t weight_stride, const int64_t *top_index_dev, int64_t top_index_stride,
                                           const void *top_logit_dev, int64_t top_logit_stride, int32_t top_dtype,
                                           int64_t n_targets, float temperature, const float *lse_dev,
                                           const float *grad_loss_dev, void *dhidden_dev, int64_t dhidden_stride,
                                           void *dweight_dev, int64_t dweight_stride, int32_t dweight_dtype,
                                           int64_t n_tokens, int64_t vocab, int64_t width, int32_t dtype,
                                           void *workspace_dev, void *stream)
{
    if (n_targets < 1) return RSDGC_ERR_INVALID;
    OperatorRange range("rsdgc_head_distill_backward");
    const HeadCall c = {hidden_dev, weight_dev, hidden_stride, weight_stride, nullptr, (const long long *)top_index_dev,
                        top_logit_dev, top_index_stride, top_logit_stride, top_dtype, n_targets, temperature, n_tokens, vocab,
                        width, dtype, (unsigned char *)workspace_dev, (cudaStream_t)stream};
    return head_backward(c, lse_dev, grad_loss_dev, dhidden_dev, dhidden_stride, dweight_dev, dweight_stride, dweight_dtype);
}
