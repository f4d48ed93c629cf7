// What the launchers set up or ask once on each device: kernel attributes (a shared-memory opt-in, a
// register count) belong to a device, and a process may hold contexts on several.
#pragma once

#include <cuda_runtime.h>

#include <atomic>

namespace c2kv {
namespace {

// make() on the current device: called at a device's first use and kept (threads that meet there may
// each call it; it gives the same value).  T: a small value type.
template <class T>
class PerDevice {
public:
    template <class Make>
    T get(const Make& make) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return make();
        if (state_[dev].load(std::memory_order_acquire) == kKept) return value_[dev];
        const T v = make();
        int empty = kEmpty;
        if (state_[dev].compare_exchange_strong(empty, kWriting)) {
            value_[dev] = v;
            state_[dev].store(kKept, std::memory_order_release);
        }
        return v;
    }

private:
    static constexpr int kDevices = 64;        // (beyond: made at each call)
    enum { kEmpty, kWriting, kKept };
    std::atomic<int> state_[kDevices] = {};
    T value_[kDevices] = {};
};

// SMs of the current device.
inline int device_sms() {
    static PerDevice<int> sms;
    return sms.get([] {
        int dev = 0, n = 0;
        if (cudaGetDevice(&dev) != cudaSuccess ||
            cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1)
            return 1;
        return n;
    });
}

// `kernel` may take `bytes` of dynamic shared memory on the current device (`kept`: one per kernel).
inline cudaError_t opt_in_smem(PerDevice<cudaError_t>& kept, const void* kernel, size_t bytes) {
    return kept.get([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); });
}

// Launches `kernel` so that its CTAs may be set up while the kernel before it in the stream ends: it has to
// wait (after_kernels_before) ahead of its first access to memory that others write or read.  That saves the
// device 1.5 to 2.5 us a launch and costs the host 0.5; `overlap` false: a launch like any other.
template <class Params>
inline cudaError_t launch_overlapped(void (*kernel)(Params), dim3 grid, unsigned threads, size_t smem, cudaStream_t s, const Params& params, bool overlap = true) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = &at;
    cfg.numAttrs = overlap ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, params);
}

// The kernels before this one in the stream have ended and what they wrote is visible.
__device__ __forceinline__ void after_kernels_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// An ordinary load: one that says that its memory never changes (__ldg) may be moved ahead of that wait.
template <class T>
__device__ __forceinline__ T ld_after(const T* p) {
    return *p;
}
// The same from L2, for what other SMs wrote.
__device__ __forceinline__ float ld_after_l2(const float* p) {
    float v;
    asm volatile("ld.global.cg.f32 %0, [%1];" : "=f"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_after_l2(const float4* p) {
    float4 v;
    asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
    return v;
}

}  // namespace
}  // namespace c2kv
