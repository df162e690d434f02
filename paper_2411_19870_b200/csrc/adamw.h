// Internal declarations of the AdamW step (adamw_lib.cu, kernels_adamw.cu).  Nothing here is part of the public ABI.
#pragma once

#include <cuda_runtime.h>

struct DemoLaunch;  // launch.cuh

struct AdamwEntry {
    long long piece_begin;  // index of this tensor's first piece
    long long n;            // elements
};
struct AdamwArgs {
    const AdamwEntry *entries;  // device
    int n_entries;
    long long n_pieces;
    const void *const *g;  // device arrays of the caller's pointers
    float *const *m, *const *v, *const *x;
    long long *step;        // device: steps made so far; one more when the kernel ends
    unsigned *done;         // device: CTAs that are through, zero between launches
    double beta1, beta2;
    float eps, lr, wd;
    int grad_bf16;
};
constexpr int ADAMW_PIECE = 2048;

cudaError_t adamw_launch(const AdamwArgs &a, DemoLaunch &dev, cudaStream_t stream);
