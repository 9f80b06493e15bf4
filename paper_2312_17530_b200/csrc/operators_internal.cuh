// Declarations shared by the language-model operators (layer norm, vocabulary head): element types,
// launch helpers and the device status word that calls without a plan report into.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "rsdgc_internal.cuh"

namespace rsdgc {

inline bool known_dtype(int t) { return t == RSDGC_F32 || t == RSDGC_BF16 || t == RSDGC_F16; }
inline int dtype_bytes(int t) { return t == RSDGC_F32 ? 4 : 2; }
inline bool pointer_aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// ---- element access: every type is widened to binary32 exactly, narrowed by one rounding (to nearest even)
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// Two binary32 operations per instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    return x;
}

// ---- mbarriers and bulk copies, by shared-memory address
__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)  // multiples of 16
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(__cvta_generic_to_global(src)), "r"(bytes), "r"(bar)
                 : "memory");
}

// Polls of a wait before it gives up.  operator_polls(): the limit of the launches to come, lower only in self-tests; what
// waits for a kernel's own copies and MMAs in flight always has the full one.
constexpr unsigned kOperatorPolls = 1u << 20;
unsigned operator_polls();

// Bounds-checked build: every index that an operator's kernel forms into an operand, a result, the workspace or a ring is
// tested; a failure is noted in the source file's own word (operators' kernels do not all know the status word, which
// rsdgc_operator_status() joins these to) and the access is skipped.  In the normal build the test is not compiled.
#ifdef RSDGC_DEBUG
static __device__ unsigned int debug_operator_bounds;
__device__ __forceinline__ bool debug_operator_in_bounds(bool ok)
{
    if (!ok) atomicOr(&debug_operator_bounds, RSDGC_STATUS_BOUNDS);
    return ok;
}
#define RSDGC_IN_BOUNDS(cond) debug_operator_in_bounds(cond)
// Reads and clears the word of the source file that it is expanded in.
#define RSDGC_DEFINE_DEBUG_BOUNDS(name)                                                                       \
    cudaError_t name(unsigned int *seen)                                                                      \
    {                                                                                                         \
        const unsigned int none = 0;                                                                          \
        cudaError_t e = cudaMemcpyFromSymbol(seen, debug_operator_bounds, sizeof none);                       \
        if (e == cudaSuccess && *seen) e = cudaMemcpyToSymbol(debug_operator_bounds, &none, sizeof none);     \
        return e;                                                                                             \
    }
cudaError_t head_debug_bounds(unsigned int *seen);
cudaError_t layer_norm_debug_bounds(unsigned int *seen);
#else
#define RSDGC_IN_BOUNDS(cond) true
#define RSDGC_DEFINE_DEBUG_BOUNDS(name)
#endif

// The status word of calls that take no plan: one per device, raised by the kernels, read and cleared by
// rsdgc_operator_status().  *out is its device address on the current device.
cudaError_t operator_status_ptr(unsigned int **out);

// Every entry point's first step: on a device's first call loads the kernels of the entry point that promises to allocate
// nothing, before the operators' own kernels use up the room that the driver has set aside for code.
cudaError_t operators_ready();

// Multiprocessors of the current device, asked once per device.
int current_device_sms();

// NVTX range around an entry point (nothing without RSDGC_NVTX).
struct OperatorRange {
    explicit OperatorRange(const char *name);
    ~OperatorRange();
};
// The entry point's return value for the launches' outcome.
int operator_result(cudaError_t e);

// Launches `kernel` so that its prologue may overlap the end of the previous kernel in the stream; the kernel
// calls grid_dependency_wait() before it touches anything another kernel writes.
template <typename... Params, typename... Args>
inline cudaError_t launch_chained(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t s,
                                  int cluster, Args... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    int n = 0;
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n++].val.programmaticStreamSerializationAllowed = 1;
    if (cluster > 1) {
        at[n].id = cudaLaunchAttributeClusterDimension;
        at[n].val.clusterDim.x = (unsigned)cluster;
        at[n].val.clusterDim.y = 1;
        at[n++].val.clusterDim.z = 1;
    }
    cfg.attrs = at;
    cfg.numAttrs = (unsigned)n;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
    if (e == cudaSuccess) count_launch(1);
    return e;
}

}  // namespace rsdgc
