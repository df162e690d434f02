// What the host sides of the ABI share: the caller's device, alignment, pointer tables.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <cstring>

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct DeviceGuard {
    int prev = -1;
    bool ok = false, changed = false;
    explicit DeviceGuard(int dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) return;
        changed = prev != dev;
        ok = !changed || cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceGuard()
    {
        if (ok && changed) cudaSetDevice(prev);
    }
};

// Upload `n` pointers to dev[0..n) if they differ from the mirror.  The mirror is pageable host
// memory: cudaMemcpyAsync stages it before returning, so it may be overwritten by the next call.
template <typename T>
cudaError_t sync_table(T *dev, T *mirror, const T *now, int n, bool *valid, cudaStream_t stream,
                       bool *changed = nullptr)
{
    if (changed) *changed = false;
    if (*valid && std::memcmp(mirror, now, sizeof(T) * (size_t)n) == 0) return cudaSuccess;
    if (changed) *changed = true;
    std::memcpy(mirror, now, sizeof(T) * (size_t)n);
    cudaError_t err = cudaMemcpyAsync(dev, mirror, sizeof(T) * (size_t)n, cudaMemcpyHostToDevice, stream);
    *valid = (err == cudaSuccess);
    return err;
}
