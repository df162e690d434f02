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
    PointerTable table;  // gradients, both moments, parameters
    unsigned *d_done = nullptr;
};

namespace {

void release(demo_adamw_ctx *c)
{
    if (!c) return;
    cudaFree(c->d_entries);
    c->table.release();
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
    if (cudaMalloc(&c->d_entries, T * sizeof(AdamwEntry)) != cudaSuccess || c->table.reserve(4 * T) != DEMO_OK ||
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
    const size_t T = (size_t)ctx->n_tensors;
    const PointerTable::List lists[4] = {{grads, T},
                                         {reinterpret_cast<const void *const *>(exp_avg), T},
                                         {reinterpret_cast<const void *const *>(exp_avg_sq), T},
                                         {reinterpret_cast<const void *const *>(params), T}};
    for (const PointerTable::List &l : lists)
        for (size_t t = 0; t < T; ++t)
            if (!l.pointers[t] || !aligned16(l.pointers[t])) return DEMO_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return DEMO_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const demo_status st = ctx->table.sync({lists[0], lists[1], lists[2], lists[3]}, stream);
    if (st != DEMO_OK) return st;
    void **const d_ptrs = ctx->table.dev();
    AdamwArgs a{};
    a.entries = ctx->d_entries;
    a.n_entries = ctx->n_tensors;
    a.n_pieces = ctx->n_pieces;
    a.g = d_ptrs;
    a.m = reinterpret_cast<float *const *>(d_ptrs + T);
    a.v = reinterpret_cast<float *const *>(d_ptrs + 2 * T);
    a.x = reinterpret_cast<float *const *>(d_ptrs + 3 * T);
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
