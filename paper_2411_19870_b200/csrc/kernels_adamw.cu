// AdamW for the tensors beside the orthogonalised ones: all of them in one launch.
//   m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2;  x <- x (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// Bound by memory: 26 (bf16 gradients) or 28 bytes an element, each once.  A CTA's piece of 2048 elements is eight elements a thread,
// all its loads under way together.  t is on the device, so that a captured step counts on; the last CTA moves it on.
#include <cuda_bf16.h>

#include "adamw.h"
#include "demo_internal.h"
#include "launch.cuh"

namespace {

constexpr int THREADS = 256;
constexpr int VECS = ADAMW_PIECE / (4 * THREADS);

struct Rates {
    float b1, c1, b2, c2, step, root, keep, eps;
};
__device__ __forceinline__ void update(const Rates &r, float g, float &m, float &v, float &x)
{
    m = fmaf(r.b1, m, r.c1 * g);
    v = fmaf(r.b2, v, r.c2 * g * g);
    x = fmaf(x, r.keep, -r.step * m / fmaf(sqrtf(v), r.root, r.eps));
}

template <bool BF16>
__global__ void __launch_bounds__(THREADS) adamw_kernel(AdamwArgs a)
{
    const StreamOrder order(1);
    __shared__ double shared_t[2];
    order.begin();
    if (threadIdx.x == 0) {
        const double t = (double)(*static_cast<volatile long long *>(a.step) + 1);
        shared_t[0] = 1.0 - pow(a.beta1, t);
        shared_t[1] = 1.0 - pow(a.beta2, t);
    }
    __syncthreads();
    Rates r;
    r.b1 = (float)a.beta1;
    r.c1 = (float)(1.0 - a.beta1);
    r.b2 = (float)a.beta2;
    r.c2 = (float)(1.0 - a.beta2);
    r.step = (float)((double)a.lr / shared_t[0]);
    r.root = (float)(1.0 / sqrt(shared_t[1]));
    r.keep = (float)(1.0 - (double)a.lr * (double)a.wd);
    r.eps = a.eps;
    for (long long p = blockIdx.x; p < a.n_pieces; p += gridDim.x) {
        const int e = demo_find_warp(0, a.n_entries, [&](int i) { return a.entries[i].piece_begin <= p; });
        const long long at = (p - a.entries[e].piece_begin) * ADAMW_PIECE, n = a.entries[e].n;
        const int len = (int)(n - at < ADAMW_PIECE ? n - at : ADAMW_PIECE);
        const void *gp = a.g[e];
        float *mp = a.m[e] + at, *vp = a.v[e] + at, *xp = a.x[e] + at;
        float4 m[VECS], v[VECS], x[VECS];
        float g[VECS][4];
#pragma unroll
        for (int k = 0; k < VECS; ++k) {
            const int i = (k * THREADS + threadIdx.x) * 4;
            if (i + 3 < len) {
                if (BF16) {
                    const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(gp) + at + i);
                    g[k][0] = __uint_as_float(w.x << 16);
                    g[k][1] = __uint_as_float(w.x & 0xffff0000u);
                    g[k][2] = __uint_as_float(w.y << 16);
                    g[k][3] = __uint_as_float(w.y & 0xffff0000u);
                } else {
                    const float4 w = *reinterpret_cast<const float4 *>(static_cast<const float *>(gp) + at + i);
                    g[k][0] = w.x, g[k][1] = w.y, g[k][2] = w.z, g[k][3] = w.w;
                }
                m[k] = *reinterpret_cast<const float4 *>(mp + i);
                v[k] = *reinterpret_cast<const float4 *>(vp + i);
                x[k] = *reinterpret_cast<const float4 *>(xp + i);
            }
        }
#pragma unroll
        for (int k = 0; k < VECS; ++k) {
            const int i = (k * THREADS + threadIdx.x) * 4;
            if (i + 3 < len) {
                update(r, g[k][0], m[k].x, v[k].x, x[k].x);
                update(r, g[k][1], m[k].y, v[k].y, x[k].y);
                update(r, g[k][2], m[k].z, v[k].z, x[k].z);
                update(r, g[k][3], m[k].w, v[k].w, x[k].w);
                *reinterpret_cast<float4 *>(mp + i) = m[k];
                *reinterpret_cast<float4 *>(vp + i) = v[k];
                *reinterpret_cast<float4 *>(xp + i) = x[k];
            }
        }
        const int rest = (len & ~3) + threadIdx.x;
        if (rest < len) {
            const float gv = BF16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(gp)[at + rest]) : static_cast<const float *>(gp)[at + rest];
            float mv = mp[rest], vv = vp[rest], xv = xp[rest];
            update(r, gv, mv, vv, xv);
            mp[rest] = mv;
            vp[rest] = vv;
            xp[rest] = xv;
        }
    }
    // every CTA has read t before the last one moves it on
    if (threadIdx.x == 0 && atomicInc(a.done, gridDim.x - 1) == gridDim.x - 1) *a.step += 1;
}

}  // namespace

cudaError_t adamw_launch(const AdamwArgs &a, DemoLaunch &dev, cudaStream_t stream)
{
    const void *kernel = a.grad_bf16 ? reinterpret_cast<const void *>(adamw_kernel<true>) : reinterpret_cast<const void *>(adamw_kernel<false>);
    int per_sm = 1;
    const cudaError_t err = demo_resident_ctas(dev, kernel, THREADS, 0, &per_sm);
    if (err != cudaSuccess) return err;
    const long long most = (long long)dev.sm_count * per_sm;
    AdamwArgs args = a;
    void *params[] = {&args};
    return demo_launch_kernel(kernel, a.n_pieces < most ? a.n_pieces : most, THREADS, 0, stream, params);
}
