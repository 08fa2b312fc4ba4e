// Launch state that is kept per device, shared by the translation units that launch kernels.
#pragma once
#include <cuda_runtime.h>
#include <atomic>

namespace gleam {

// Launch state that CUDA keeps per device (function attributes, occupancy, SM count) is cached per
// device ordinal: one process may drive several GPUs, from several host threads.  The cached values
// are idempotent, so two threads that race on a first use both compute and store the same thing.
constexpr int MAX_DEVICES = 64;
struct PerDevice {
    std::atomic<int> v[MAX_DEVICES];         // 0 = not yet known on that device
    std::atomic<int>* slot() {
        int dev = -1;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return nullptr;
        return &v[dev];
    }
};

// static_bytes: statically declared shared memory of the kernel, which counts against the same
// 48 KB default limit as the dynamic part
template <class K>
inline cudaError_t ensure_smem(K kernel, size_t bytes, PerDevice& done, size_t static_bytes = 0) {
    if (bytes + static_bytes <= 48 * 1024) return cudaSuccess;
    std::atomic<int>* flag = done.slot();               // null: device ordinal outside the cache, set every time
    if (flag && flag->load(std::memory_order_acquire)) return cudaSuccess;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) return e;
    if (flag) flag->store(1, std::memory_order_release);
    return cudaSuccess;
}

// SM count of the current device, cached per device
inline cudaError_t device_sms(int* out) {
    static PerDevice cache;
    std::atomic<int>* c = cache.slot();
    if (c) { const int v = c->load(std::memory_order_acquire); if (v > 0) { *out = v; return cudaSuccess; } }
    int dev = 0;
    cudaError_t e;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if ((e = cudaDeviceGetAttribute(out, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    if (c) c->store(*out, std::memory_order_release);
    return cudaSuccess;
}

// resident blocks of `kernel` on the current device (SM count x blocks per SM), cached per device
template <class K>
inline cudaError_t resident_slots(K kernel, int threads, size_t smem, PerDevice& cache, int* out) {
    std::atomic<int>* c = cache.slot();
    if (c) { const int v = c->load(std::memory_order_acquire); if (v > 0) { *out = v; return cudaSuccess; } }
    int sms = 0, per_sm = 0;
    cudaError_t e;
    if ((e = device_sms(&sms)) != cudaSuccess) return e;
    if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem)) != cudaSuccess) return e;
    *out = sms * (per_sm > 0 ? per_sm : 1);
    if (c) c->store(*out, std::memory_order_release);
    return cudaSuccess;
}

}  // namespace gleam
