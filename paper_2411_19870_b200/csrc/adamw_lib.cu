// Host side of demo_adamw_* in include/demo.h.
#include <cmath>
#include <cstring>
#include <exception>
#include <new>
#include <vector>

#include "../../include/demo.h"
#include "adamw.h"
#include "host_common.h"
#include "launch.cuh"

struct demo_adamw_ctx {
    demo_adamw_config cfg;
    int device = 0, n_tensors = 0;
    DemoLaunch launch;
    long long n_pieces = 0, launches = 0;
    AdamwEntry *d_entries = nullptr;
    void **d_ptrs = nullptr;  // [4][n_tensors]: gradients, both moments, parameters
    std::vector<void *> ptrs;
    bool valid = false;
    unsigned *d_done = nullptr;
};

namespace {

void release(demo_adamw_ctx *c)
{
    if (!c) return;
    cudaFree(c->d_entries);
    cudaFree((void *)c->d_ptrs);
    cudaFree(c->d_done);
    delete c;
}

demo_status build(demo_adamw_ctx *c, const int64_t *numels)
{
    const size_t T = (size_t)c->n_tensors;
    std::vector<AdamwEntry> entries(T);
    for (size_t t = 0; t < T; ++t) {
        entries[t].piece_begin = c->n_pieces;
        entries[t].n = numels[t];
        c->n_pieces += (numels[t] + ADAMW_PIECE - 1) / ADAMW_PIECE;
    }
    c->ptrs.assign(4 * T, nullptr);
    if (cudaMalloc(&c->d_entries, T * sizeof(AdamwEntry)) != cudaSuccess || cudaMalloc((void **)&c->d_ptrs, 4 * T * sizeof(void *)) != cudaSuccess ||
        cudaMalloc(&c->d_done, sizeof(unsigned)) != cudaSuccess)
        return DEMO_ERR_ALLOC;
    if (cudaMemcpy(c->d_entries, entries.data(), T * sizeof(AdamwEntry), cudaMemcpyHostToDevice) != cudaSuccess ||
        cudaMemset(c->d_done, 0, sizeof(unsigned)) != cudaSuccess ||
        cudaStreamSynchronize(nullptr) != cudaSuccess)  // (the first step may be on a stream that does not wait for this one)
        return DEMO_ERR_CUDA;
    return DEMO_OK;
}

}  // namespace

extern "C" {

demo_status demo_adamw_init(demo_adamw_ctx **out, const demo_adamw_config *cfg, const int64_t *numels, int32_t n_tensors, int32_t cuda_device)
{
    if (out) *out = nullptr;
    if (!out || !cfg || !numels || n_tensors < 1 || cuda_device < 0) return DEMO_ERR_INVALID_ARG;
    if (!(cfg->beta1 >= 0 && cfg->beta1 < 1) || !(cfg->beta2 >= 0 && cfg->beta2 < 1)) return DEMO_ERR_INVALID_ARG;
    if (!std::isfinite(cfg->eps) || cfg->eps < 0 || !std::isfinite(cfg->lr) || !std::isfinite(cfg->weight_decay)) return DEMO_ERR_INVALID_ARG;
    if (cfg->grad_dtype != DEMO_F32 && cfg->grad_dtype != DEMO_BF16) return DEMO_ERR_UNSUPPORTED;
    if (n_tensors > (1 << 20)) return DEMO_ERR_UNSUPPORTED;
    for (int t = 0; t < n_tensors; ++t)
        if (numels[t] < 1 || numels[t] > (1LL << 40)) return DEMO_ERR_SHAPE;
    int n_dev = 0;
    if (cudaGetDeviceCount(&n_dev) != cudaSuccess || cuda_device >= n_dev) {
        cudaGetLastError();
        return DEMO_ERR_CUDA;
    }
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return DEMO_ERR_CUDA;
    demo_adamw_ctx *c = new (std::nothrow) demo_adamw_ctx();
    if (!c) return DEMO_ERR_ALLOC;
    c->cfg = *cfg;
    c->device = cuda_device;
    c->n_tensors = n_tensors;
    demo_status st = DEMO_OK;
    if (cudaDeviceGetAttribute(&c->launch.sm_count, cudaDevAttrMultiProcessorCount, cuda_device) != cudaSuccess) st = DEMO_ERR_CUDA;
    if (st == DEMO_OK) {
        try {
            st = build(c, numels);
        } catch (const std::exception &) {
            st = DEMO_ERR_ALLOC;
        }
    }
    if (st != DEMO_OK) {
        cudaGetLastError();
        release(c);
        return st;
    }
    *out = c;
    return DEMO_OK;
}

demo_status demo_adamw_step(demo_adamw_ctx *ctx, const void *const *grads, float *const *exp_avg, float *const *exp_avg_sq, float *const *params,
                            int64_t *step, void *cuda_stream)
{
    if (!ctx || !grads || !exp_avg || !exp_avg_sq || !params || !step || (reinterpret_cast<uintptr_t>(step) & 7u)) return DEMO_ERR_INVALID_ARG;
    const size_t T = (size_t)ctx->n_tensors, bytes = T * sizeof(void *);
    const void *lists[4] = {grads, exp_avg, exp_avg_sq, params};
    bool same = ctx->valid;
    for (int l = 0; l < 4; ++l) {
        const void *const *p = static_cast<const void *const *>(lists[l]);
        for (size_t t = 0; t < T; ++t)
            if (!p[t] || !aligned16(p[t])) return DEMO_ERR_INVALID_ARG;
        same = same && std::memcmp(ctx->ptrs.data() + l * T, p, bytes) == 0;
    }
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return DEMO_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (!same) {
        // (a captured graph would copy whatever the host array holds when it runs)
        cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(stream, &capture) != cudaSuccess) {
            cudaGetLastError();
            return DEMO_ERR_CUDA;
        }
        if (capture != cudaStreamCaptureStatusNone) return DEMO_ERR_INVALID_ARG;
        for (int l = 0; l < 4; ++l) std::memcpy(ctx->ptrs.data() + l * T, lists[l], bytes);
        ctx->valid = cudaMemcpyAsync((void *)ctx->d_ptrs, ctx->ptrs.data(), 4 * bytes, cudaMemcpyHostToDevice, stream) == cudaSuccess;
        if (!ctx->valid) {
            cudaGetLastError();
            return DEMO_ERR_CUDA;
        }
    }
    AdamwArgs a{};
    a.entries = ctx->d_entries;
    a.n_entries = ctx->n_tensors;
    a.n_pieces = ctx->n_pieces;
    a.g = ctx->d_ptrs;
    a.m = reinterpret_cast<float *const *>(ctx->d_ptrs + T);
    a.v = reinterpret_cast<float *const *>(ctx->d_ptrs + 2 * T);
    a.x = reinterpret_cast<float *const *>(ctx->d_ptrs + 3 * T);
    a.step = reinterpret_cast<long long *>(step);
    a.done = ctx->d_done;
    a.beta1 = ctx->cfg.beta1;
    a.beta2 = ctx->cfg.beta2;
    a.eps = ctx->cfg.eps;
    a.lr = ctx->cfg.lr;
    a.wd = ctx->cfg.weight_decay;
    a.grad_bf16 = ctx->cfg.grad_dtype == DEMO_BF16;
    if (adamw_launch(a, ctx->launch, stream) != cudaSuccess) {
        cudaGetLastError();
        return DEMO_ERR_CUDA;
    }
    ctx->launches += 1;
    return DEMO_OK;
}

demo_status demo_adamw_set_lr(demo_adamw_ctx *ctx, float lr)
{
    if (!ctx || !std::isfinite(lr)) return DEMO_ERR_INVALID_ARG;
    ctx->cfg.lr = lr;
    return DEMO_OK;
}

int64_t demo_adamw_launch_count(const demo_adamw_ctx *ctx) { return ctx ? ctx->launches : 0; }

void demo_adamw_free(demo_adamw_ctx *ctx)
{
    if (!ctx) return;
    DeviceGuard guard(ctx->device);
    release(ctx);
}

}  // extern "C"
