// What the host sides of the ABI share: the caller's device, alignment, pointer tables.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <cstring>
#include <exception>
#include <initializer_list>
#include <memory>
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
// captured with for as long as it lives: until then that one is not written again, and calls with other pointers get another, one that no graph
// reads any more where there is one.
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
        unsigned long long id = 0;
        cudaGraph_t graph = nullptr;
        if (cudaStreamGetCaptureInfo(stream, &capture, &id, &graph) != cudaSuccess) return failed(DEMO_ERR_CUDA);
        const bool capturing = capture != cudaStreamCaptureStatusNone;
        bool same = valid_;
        size_t at = 0;
        for (const List &l : lists) {
            same = same && std::memcmp(host_.data() + at, l.pointers, l.n * sizeof(void *)) == 0;
            at += l.n;
        }
        if (same) return capturing ? hold(graph) : DEMO_OK;
        if (capturing) return DEMO_ERR_INVALID_ARG;
        if (now_->graphs != 0) {
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
        if (cudaMemcpyAsync((void *)now_->dev, host_.data(), at * sizeof(void *), cudaMemcpyHostToDevice, stream) != cudaSuccess) return failed(DEMO_ERR_CUDA);
        valid_ = true;
        return DEMO_OK;
    }
    void **dev() const { return now_->dev; }
    bool reserved() const { return now_ != nullptr; }
    size_t bytes() const { return all_.size() * host_.size() * sizeof(void *); }
    void release()
    {
        for (const std::shared_ptr<Copy> &c : all_) cudaFree((void *)c->dev);
        all_.clear();
        now_.reset();
    }

private:
    struct Copy {
        void **dev = nullptr;
        std::atomic<int> graphs{0};  // captured graphs, and what was made from them, that read it
    };
    static demo_status failed(demo_status st)
    {
        cudaGetLastError();
        return st;
    }
    // The graph under capture reads the copy.  It gives it back, on a thread of the runtime, when it and all that was instantiated from it are gone and
    // have run; the copy's record may outlive the table.
    demo_status hold(cudaGraph_t graph)
    {
        auto *mine = new (std::nothrow) std::shared_ptr<Copy>(now_);
        if (!mine) return DEMO_ERR_ALLOC;
        ++now_->graphs;
        const cudaHostFn_t give_back = [](void *p) {
            auto *c = static_cast<std::shared_ptr<Copy> *>(p);
            --(*c)->graphs;
            delete c;
        };
        cudaUserObject_t object = nullptr;
        if (cudaUserObjectCreate(&object, mine, give_back, 1, cudaUserObjectNoDestructorSync) != cudaSuccess) {
            give_back(mine);
            return failed(DEMO_ERR_CUDA);
        }
        if (cudaGraphRetainUserObject(graph, object, 1, cudaGraphUserObjectMove) != cudaSuccess) {
            cudaUserObjectRelease(object, 1);
            return failed(DEMO_ERR_CUDA);
        }
        return DEMO_OK;
    }
    demo_status another()
    {
        for (const std::shared_ptr<Copy> &c : all_)
            if (c->graphs == 0) {
                now_ = c;
                valid_ = false;
                return DEMO_OK;
            }
        std::shared_ptr<Copy> c;
        try {
            c = std::make_shared<Copy>();
            all_.reserve(all_.size() + 1);
        } catch (const std::exception &) {
            return DEMO_ERR_ALLOC;
        }
        if (cudaMalloc((void **)&c->dev, host_.size() * sizeof(void *)) != cudaSuccess) return failed(DEMO_ERR_ALLOC);
        all_.push_back(c);
        now_ = c;
        valid_ = false;
        return DEMO_OK;
    }
    std::vector<const void *> host_;
    std::vector<std::shared_ptr<Copy>> all_;
    std::shared_ptr<Copy> now_;  // what calls use
    bool valid_ = false;
};
