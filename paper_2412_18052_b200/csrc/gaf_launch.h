// Launch plumbing shared by the translation units of the C ABI: attributes and launch plans kept per device, programmatic
// launches, the driver's tensor-map encoder, small checks.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <mutex>

#include "../../include/gaf.h"

namespace {

constexpr int kMaxDevices = 64;

struct DeviceInfo {
    int dev = 0;
    int sms = 0;
    int l2_bytes = 0;
    int smem_per_sm = 0;                // shared memory of one SM
    int smem_per_cta_max = 0;           // opt-in limit of one CTA
};

// What is worked out once per device and kept for the life of the process: the device's attributes and, per
// kernel instantiation, its launch plan (occupancy, shared-memory attributes, grid).  A call then costs
// argument checks and the launch itself: at a million elements the driver queries were a third of the call.
// Device memory is not involved; the tables are guarded by one mutex on their slow path only.
std::mutex g_plan_mutex;

// Runs `make(slot)` once per (table slot, device); afterwards the slot is read without the lock.
template <typename Plan, typename Make>
int plan_once(Plan &slot, std::atomic<int> &ready, Make &&make) {
    if (ready.load(std::memory_order_acquire)) return GAF_OK;
    std::lock_guard<std::mutex> lock(g_plan_mutex);
    if (ready.load(std::memory_order_relaxed)) return GAF_OK;
    if (int rc = make(slot)) return rc;             // nothing is remembered about a failure
    ready.store(1, std::memory_order_release);
    return GAF_OK;
}

struct DeviceSlot { DeviceInfo info; std::atomic<int> ready{0}; };
DeviceSlot g_devices[kMaxDevices];

// Attributes of the current device.
bool device_info(DeviceInfo *out) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return false;
    DeviceSlot &slot = g_devices[dev];
    const int rc = plan_once(slot.info, slot.ready, [dev](DeviceInfo &d) {
        d.dev = dev;
        if (cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return GAF_ERR_CUDA;
        if (cudaDeviceGetAttribute(&d.l2_bytes, cudaDevAttrL2CacheSize, dev) != cudaSuccess) return GAF_ERR_CUDA;
        if (cudaDeviceGetAttribute(&d.smem_per_sm, cudaDevAttrMaxSharedMemoryPerMultiprocessor, dev) != cudaSuccess)
            return GAF_ERR_CUDA;
        if (cudaDeviceGetAttribute(&d.smem_per_cta_max, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev) != cudaSuccess)
            return GAF_ERR_CUDA;
        return d.sms > 0 ? GAF_OK : GAF_ERR_CUDA;
    });
    if (rc != GAF_OK) return false;
    *out = slot.info;
    return true;
}

// One slot per device for a kernel instantiation: `static PerDevice<Plan> table;` inside a function template
// gives every instantiation its own table.
template <typename Plan>
struct PerDevice {
    Plan plan[kMaxDevices];
    std::atomic<int> ready[kMaxDevices];
    PerDevice() { for (auto &r : ready) r.store(0, std::memory_order_relaxed); }
};
struct DynSmemPlan { int dyn = 0; };    // "the dynamic shared memory limit of this kernel has been raised"

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t elem_bytes(int dtype) { return dtype == GAF_F32 ? 4 : 2; }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// Launch `kernel` as a programmatic dependent of the launch before it on the stream: its blocks may be
// placed while that grid winds down; the kernel itself waits (griddepcontrol.wait) for that grid.
template <typename... KArgs, typename... Args>
cudaError_t launch_dependent_smem(void (*kernel)(KArgs...), int grid, int threads, size_t dyn_smem, cudaStream_t st,
                                  const Args &...args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = dyn_smem; cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <typename... KArgs, typename... Args>
cudaError_t launch_dependent(void (*kernel)(KArgs...), int grid, int threads, cudaStream_t st, const Args &...args) {
    return launch_dependent_smem(kernel, grid, threads, 0, st, args...);
}

// The driver's tensor-map encoder, fetched once through the runtime (the library does not link the driver).
using TensorMapEncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                       const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                       CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
TensorMapEncodeFn tensor_map_encoder() {
    static std::atomic<void *> fn{nullptr};
    static std::atomic<int> tried{0};
    if (!tried.load(std::memory_order_acquire)) {
        std::lock_guard<std::mutex> lock(g_plan_mutex);
        if (!tried.load(std::memory_order_relaxed)) {
            void *p = nullptr;
            cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
            if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
                q != cudaDriverEntryPointSuccess)
                p = nullptr;
            cudaGetLastError();
            fn.store(p, std::memory_order_relaxed);
            tried.store(1, std::memory_order_release);
        }
    }
    return reinterpret_cast<TensorMapEncodeFn>(fn.load(std::memory_order_relaxed));
}

int check_workspace(const void *ws, size_t have, size_t need) {
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0 || have < need) return GAF_ERR_WORKSPACE;
    return GAF_OK;
}

}  // namespace
