// Internal declarations of the orthogonalised update (muon_lib.cu, kernels_muon.cu).  Nothing here is part of the public ABI.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <vector>

#include "../../include/demo.h"

struct DemoLaunch;  // launch.cuh

// demo_lib.cu.  Which of `n` matrices each of the context's tensors is, -1 for 1-D tensors.  SHAPE when its 2-D tensors are not these;
// UNSUPPORTED, INVALID_ARG.
demo_status demo_decode_places(const demo_ctx *ctx, int device, const demo_tensor_desc *matrices, int n, std::vector<int> *place);
// R of the 2-D tensors to to[t], which lie in the `momentum_bytes` bytes at `momentum`; 1-D tensors to[t] updated as in demo_decode_apply.
demo_status demo_decode_momentum(demo_ctx *ctx, const void *const *payloads, int32_t n_payloads, float *const *to, float *momentum,
                                 size_t momentum_bytes, cudaStream_t stream);

// One matrix.  The kernels work on X with `m` <= `n`: a tensor with more rows than columns is held transposed.  X lies in the workspace
// scaled by the power of two `S`, as hi + lo (two fp16 matrices of `ldx` elements a row), twice: an iteration reads one and writes the other.
// Gram matrix A = D + E: d holds its diagonal, E (fp16, `lde` elements a row) the rest; F and beta are the polynomial of A, split the same way.
struct MuonMat {
    int m, n;
    int ldx, lde;
    int transposed;    // 1: X is the tensor's transpose
    int precise;       // 1: products take the lo parts, too
    int tensor;        // position in the caller's pointer arrays
    int piece_begin;   // its first piece of the norm in the group, and how many
    int n_pieces;
    int maps;          // index of its first tensor map (MUON_MAPS of them)
    float S, inv_S;
    float step_scale;  // of the update: x <- x - lr (step_scale O + wd x)
    uint16_t *xhi[2], *xlo[2];
    uint16_t *ehi, *elo, *fhi, *flo;
    float *d, *beta;
};
// Tensor maps of a matrix (boxes of 64 x 64 fp16 elements, 128-byte swizzle).
enum { MUON_MAP_X0 = 0, MUON_MAP_X1 = 1, MUON_MAP_XLO0 = 2, MUON_MAP_XLO1 = 3, MUON_MAP_E = 4, MUON_MAP_ELO = 5, MUON_MAP_F = 6, MUON_MAP_FLO = 7, MUON_MAPS = 8 };
constexpr int MUON_MAP_BYTES = 128;

// E and F lie in the workspace 256 times as large: entries of 1/m and less, and their lo parts, stay in fp16's normal range (of rank one,
// 96 rows: error 1.6e-4 without).  Entries of up to 255 remain possible: singular values up to about 3 within the iterations.
constexpr float MUON_EF_SCALE = 256.f, MUON_EF_INV = 1.f / 256.f;

constexpr int MUON_PIECE = 8192;     // elements of a piece of the norm
constexpr int MUON_PACK_TILE = 64;   // side of the tiles in which X is laid out

struct MuonTile {
    int mat;
    short i, j;  // tile row and column
};

// What the update is formed from and what becomes of it.
enum { MUON_FROM_STEP = 0, MUON_FROM_INPUT = 1 };   // u = g + mu m' (or m'), m' = mu m + g; or u = the input itself
enum { MUON_TO_PARAMS = 0, MUON_TO_OUTPUT = 1 };
struct MuonArgs {
    const MuonMat *mats;   // device
    const char *maps;      // device, all matrices' tensor maps
    const void *const *in; // device array of the caller's gradients / inputs, by tensor
    float *const *mom;     // device array (MUON_FROM_STEP)
    void *const *out;      // device array: parameters (fp32) or outputs
    double *partials;      // device: a sum of squares for each piece
    int from, to;
    int in_bf16, out_bf16;
    int nesterov;
    float mu, eps, lr, wd;
    float a, b, c;
    int *status;
};

enum { MUON_GRAM = 0, MUON_POLY = 1, MUON_UPDATE = 2, MUON_FINAL = 3 };

// Momentum update and the pieces' sums of squares; pieces [0, n_pieces) of the matrices [first, first + n).
cudaError_t muon_launch_norm(const MuonArgs &a, int first_mat, int n_mats, int n_pieces, DemoLaunch &dev, cudaStream_t stream);
// X = S u / (||u|| + eps), as hi + lo.
cudaError_t muon_launch_pack(const MuonArgs &a, const MuonTile *tiles, int n_tiles, DemoLaunch &dev, cudaStream_t stream);
// One product of every listed tile.  pair: tiles of 256 x 256 by clusters of two CTAs; otherwise 128 x 128 by one.
cudaError_t muon_launch_product(int phase, bool pair, int parity, const MuonArgs &a, const MuonTile *tiles, int n_tiles, DemoLaunch &dev, cudaStream_t stream);
