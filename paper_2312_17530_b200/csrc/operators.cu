// What the language-model operators share on the host: the per-device status word, NVTX ranges, results.
#include <atomic>
#include <mutex>

#include "operators_internal.cuh"

#ifdef RSDGC_NVTX
#include <nvtx3/nvToolsExt.h>
#endif

namespace rsdgc {

namespace {
constexpr int kMaxDevices = 64;
__device__ unsigned int g_operator_status;
std::atomic<unsigned> g_polls{kOperatorPolls};

// Clears the bits that were read, and no others.
__global__ void k_operator_status_clear(unsigned int *status, unsigned int seen) { atomicAnd(status, ~seen); }

// The wait of the self-test: a barrier armed for bytes that nothing will deliver, with nothing in flight.
__global__ void k_selftest_operator_wait(unsigned int *status, unsigned int polls)
{
    __shared__ __align__(8) unsigned long long bar;
    barrier_init(smem_addr(&bar), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    barrier_expect(smem_addr(&bar), 16);
    bool here = false;
    for (unsigned i = 0; i < polls && !here; ++i) here = barrier_try(smem_addr(&bar), 0);
    if (!here) atomicOr(status, RSDGC_STATUS_TIMEOUT);
    asm volatile("mbarrier.inval.shared::cta.b64 [%0];" ::"r"(smem_addr(&bar)) : "memory");
}
}  // namespace

unsigned operator_polls() { return g_polls.load(std::memory_order_relaxed); }

cudaError_t operator_status_ptr(unsigned int **out)
{
    static std::mutex mu;
    static void *ptrs[kMaxDevices] = {};
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(mu);
    if (!ptrs[dev]) {
        void *p = nullptr;
        e = cudaGetSymbolAddress(&p, g_operator_status);
        if (e != cudaSuccess) return e;
        ptrs[dev] = p;
    }
    *out = static_cast<unsigned int *>(ptrs[dev]);
    return cudaSuccess;
}

cudaError_t operators_ready()
{
    static std::atomic<uint64_t> ready{0};
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    if (ready.load(std::memory_order_acquire) >> dev & 1) return cudaSuccess;
    e = load_noalloc_kernels();
    if (e == cudaSuccess) ready.fetch_or(1ull << dev, std::memory_order_release);
    return e;
}

int current_device_sms()
{
    static std::mutex mu;
    static int sms[kMaxDevices] = {};
    int dev = -1;
    // without a device the sizes of a B200 are assumed, so that workspaces can be sized on the host
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) {
        (void)cudaGetLastError();
        return 148;
    }
    std::lock_guard<std::mutex> lock(mu);
    if (!sms[dev] && cudaDeviceGetAttribute(&sms[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return 148;
    }
    return sms[dev];
}

#ifdef RSDGC_NVTX
OperatorRange::OperatorRange(const char *name) { nvtxRangePushA(name); }
OperatorRange::~OperatorRange() { nvtxRangePop(); }
#else
OperatorRange::OperatorRange(const char *) {}
OperatorRange::~OperatorRange() {}
#endif

int operator_result(cudaError_t e)
{
    if (e == cudaSuccess) return RSDGC_OK;
    (void)cudaGetLastError();
    set_last_cuda_error((int)e);
    return RSDGC_ERR_CUDA;
}

}  // namespace rsdgc

using namespace rsdgc;

extern "C" int rsdgc_selftest_operator_polls(int32_t polls)
{
    if (polls < 0 || polls > (int32_t)kOperatorPolls) return RSDGC_ERR_INVALID;
    g_polls.store(polls ? (unsigned)polls : kOperatorPolls, std::memory_order_relaxed);
    return RSDGC_OK;
}

extern "C" int rsdgc_operator_status(void *stream, uint32_t *flags_host)
{
    if (!flags_host) return RSDGC_ERR_INVALID;
    unsigned int *p = nullptr;
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e = operator_status_ptr(&p);
    unsigned int seen = 0;
    if (e == cudaSuccess) e = cudaMemcpyAsync(&seen, p, sizeof(unsigned int), cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    // Kernels on other streams may raise bits meanwhile: only what this call reports is cleared.
    if (e == cudaSuccess && seen) {
        k_operator_status_clear<<<1, 1, 0, s>>>(p, seen);
        e = cudaGetLastError();
        count_launch(1);
        if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    }
#ifdef RSDGC_DEBUG
    unsigned int more[2] = {0, 0};
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = head_debug_bounds(&more[0]);
    if (e == cudaSuccess) e = layer_norm_debug_bounds(&more[1]);
    seen |= more[0] | more[1];
#endif
    if (e == cudaSuccess) *flags_host = seen;
    return operator_result(e);
}

extern "C" int rsdgc_selftest_operator_wait(int32_t polls, void *stream)
{
    if (polls < 1 || polls > (int32_t)kOperatorPolls) return RSDGC_ERR_INVALID;
    unsigned int *p = nullptr;
    cudaError_t e = operator_status_ptr(&p);
    if (e == cudaSuccess) {
        k_selftest_operator_wait<<<1, 1, 0, (cudaStream_t)stream>>>(p, (unsigned)polls);
        e = cudaGetLastError();
        count_launch(1);
    }
    return operator_result(e);
}
