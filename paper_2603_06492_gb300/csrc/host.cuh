// Host side shared by the translation units of the library: errors, launches,
// checks of arguments and of the device, driver entry points.
#pragma once

#include <atomic>
#include <cstdarg>
#include <cstdio>
#include <mutex>
#include <type_traits>
#include <utility>
#include <vector>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/noble.h"
#include "common.cuh"
#include "profile.cuh"

namespace noble {

inline thread_local char g_last_error[512] = "";
inline std::atomic<uint64_t> g_launches{0};

inline noble_status fail(noble_status s, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
    va_end(ap);
    return s;
}

inline noble_status check_launch(const char *what)
{
    g_launches.fetch_add(1, std::memory_order_relaxed);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(NOBLE_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
    return NOBLE_OK;
}

// Kernels launched so far by the current entry-point call on this thread.
inline thread_local int g_call_kernels = 0;

// Launch through `f`, bracketed by profiling events when profiling is on.
template <class F>
noble_status run(cudaStream_t st, const KernelInfo &ki, F &&f)
{
    const int slot = Profiler::get().begin(st);
    f();
    Profiler::get().end(slot, st, ki);
    ++g_call_kernels;
    return check_launch(ki.name);
}

// Programmatic dependent launch: a kernel after the first of a call may start
// while the previous one still runs, on the SMs it leaves free; it waits for it
// (griddep_wait) before reading anything an earlier kernel of the call wrote,
// and every such grid waits at least once, so its completion implies its
// predecessors'.  The first kernel of a call, and the first after a memset, is
// launched normally and sees all prior work in the stream -- except the CosNet
// kernels, which wait for their predecessor grid in every thread before any
// global read, so that their set-up may overlap the previous kernel whatever it
// is, and let their own dependent start only after that.
constexpr bool kProgrammaticLaunch = true;
inline bool pdl_ok() { return kProgrammaticLaunch && g_call_kernels > 0; }

// On clusters of `cluster` CTAs along x (1: none, or the kernel's own).
template <class... KArgs, class... Args>
void launch_cluster(void (*kern)(KArgs...), dim3 grid, int cluster, dim3 block, size_t smem, cudaStream_t st, bool pdl,
                    Args &&...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = cluster, attr[n].val.clusterDim.y = 1, attr[n++].val.clusterDim.z = 1;
    }
    if (pdl) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    cudaLaunchKernelEx(&cfg, kern, std::forward<Args>(args)...);
}
template <class... KArgs, class... Args>
void launch_maybe_pdl(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool pdl,
                      Args &&...args)
{
    launch_cluster(kern, grid, 1, block, smem, st, pdl, std::forward<Args>(args)...);
}

// cudaMemsetAsync on the stream; the next kernel is then launched normally.
inline cudaError_t memset_async(void *p, int v, size_t n, cudaStream_t st)
{
    g_call_kernels = 0;
    return cudaMemsetAsync(p, v, n, st);
}

#define NOBLE_TRY(expr)                              \
    do {                                             \
        noble_status _s = (expr);                    \
        if (_s != NOBLE_OK) return _s;               \
    } while (0)

inline noble_status check_ptr(const void *p, const char *name, bool nullable)
{
    if (!p) return nullable ? NOBLE_OK : fail(NOBLE_ERR_INVALID_ARG, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) % 16) return fail(NOBLE_ERR_MISALIGNED, "%s is not 16-byte aligned", name);
    return NOBLE_OK;
}

inline noble_status check_device()
{
    static int cached[64];  // 0 unknown, 1 ok, 2 bad
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) {
        cudaGetLastError();
        return fail(NOBLE_ERR_NO_DEVICE, "no current CUDA device");
    }
    if (dev < 64 && cached[dev] == 1) return NOBLE_OK;
    int major = 0, minor = 0;
    cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
    cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev);
    cudaGetLastError();
    if (major != 10 || minor != 3) {
        if (dev < 64) cached[dev] = 2;
        return fail(NOBLE_ERR_NO_DEVICE, "device %d is sm_%d%d; this library is built for sm_103a", dev, major, minor);
    }
    if (dev < 64) cached[dev] = 1;
    return NOBLE_OK;
}

inline int num_sms()
{
    static int cache[64];
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && cache[dev]) return cache[dev];
    int n = 0;
    cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    cudaGetLastError();
    if (n <= 0) n = 1;
    if (dev >= 0 && dev < 64) cache[dev] = n;
    return n;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_fn()
{
    static EncodeTiledFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) !=
                cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<EncodeTiledFn>(p);
    }();
    return fn;
}

// The current CUDA context (NULL if none or the driver call is unavailable).
typedef CUresult (*CtxGetCurrentFn)(CUcontext *);
inline CUcontext current_context()
{
    static CtxGetCurrentFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuCtxGetCurrent", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<CtxGetCurrentFn>(p);
    }();
    CUcontext c = nullptr;
    if (!fn || fn(&c) != CUDA_SUCCESS) return nullptr;
    return c;
}

// Device address of a __device__ variable in the current context.  The
// host-side name of a __device__ variable is only a stand-in, so the address
// is looked up with the device current; it is cached per context (a new
// context after a device reset loads the module at another address).
template <class T>
void *symbol_address(const T &symbol)
{
    static std::mutex mu;
    static std::vector<std::pair<CUcontext, void *>> cache;
    const CUcontext ctx = current_context();
    std::lock_guard<std::mutex> g(mu);
    if (ctx)
        for (auto &e : cache)
            if (e.first == ctx) return e.second;
    void *p = nullptr;
    if (cudaGetSymbolAddress(&p, symbol) != cudaSuccess || !p) {
        cudaGetLastError();
        return nullptr;
    }
    // the lookup may have created the primary context: key on it
    const CUcontext now = ctx ? ctx : current_context();
    if (now) cache.emplace_back(now, p);
    return p;
}

// Device address of this device's status word (noble_api.cu).
uint32_t *status_ptr();

}  // namespace noble
