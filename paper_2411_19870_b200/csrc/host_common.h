// What the host sides of the ABI share: the caller's device, alignment, pointer tables.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <cstring>
#include <initializer_list>
#include <new>
#include <vector>

#include "../../include/demo.h"

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

// The device's copy of the pointer arrays of one entry point's calls, one array behind the other.  A captured graph reads the copy that it was
// captured with for as long as it lives: from then on that one is not written again, and calls with other pointers get another.
class PointerTable {
public:
    struct List {
        const void *const *pointers;
        size_t n;
    };
    demo_status reserve(size_t n)
    {
        try {
            host_.assign(n, nullptr);
        } catch (const std::exception &) {
            return DEMO_ERR_ALLOC;
        }
        return another();
    }
    // A copy that a capturing stream would have to make is refused: the graph would copy whatever the host's array holds when it runs.
    demo_status sync(std::initializer_list<List> lists, cudaStream_t stream)
    {
        cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(stream, &capture) != cudaSuccess) return failed(DEMO_ERR_CUDA);
        const bool capturing = capture != cudaStreamCaptureStatusNone;
        bool same = valid_;
        size_t at = 0;
        for (const List &l : lists) {
            same = same && std::memcmp(host_.data() + at, l.pointers, l.n * sizeof(void *)) == 0;
            at += l.n;
        }
        if (same) {
            captured_ = captured_ || capturing;
            return DEMO_OK;
        }
        if (capturing) return DEMO_ERR_INVALID_ARG;
        if (captured_) {
            const demo_status st = another();
            if (st != DEMO_OK) return st;
        }
        valid_ = false;
        at = 0;
        for (const List &l : lists) {
            std::memcpy(host_.data() + at, l.pointers, l.n * sizeof(void *));
            at += l.n;
        }
        // (pageable memory: staged before the call returns)
        if (cudaMemcpyAsync((void *)dev_, host_.data(), at * sizeof(void *), cudaMemcpyHostToDevice, stream) != cudaSuccess) return failed(DEMO_ERR_CUDA);
        valid_ = true;
        return DEMO_OK;
    }
    void **dev() const { return dev_; }
    bool reserved() const { return dev_ != nullptr; }
    size_t bytes() const { return all_.size() * host_.size() * sizeof(void *); }
    void release()
    {
        for (void **p : all_) cudaFree((void *)p);
        all_.clear();
        dev_ = nullptr;
    }

private:
    static demo_status failed(demo_status st)
    {
        cudaGetLastError();
        return st;
    }
    demo_status another()
    {
        void **p = nullptr;
        try {
            all_.reserve(all_.size() + 1);
        } catch (const std::exception &) {
            return DEMO_ERR_ALLOC;
        }
        if (cudaMalloc((void **)&p, host_.size() * sizeof(void *)) != cudaSuccess) return failed(DEMO_ERR_ALLOC);
        all_.push_back(p);
        dev_ = p;
        valid_ = captured_ = false;
        return DEMO_OK;
    }
    std::vector<const void *> host_;
    std::vector<void **> all_;
    void **dev_ = nullptr;
    bool valid_ = false, captured_ = false;
};
