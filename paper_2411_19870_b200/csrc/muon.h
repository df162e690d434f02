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

// One matrix.  The kernels work on X with `m` <= `n`: a tensor with more rows than columns is held transposed.  In the workspace, scaled by
// the power of two `S`, X is fp16 (twice: a product reads one and writes the other; lo parts only for `precise` matrices), rows of `ldx`
// elements, and x32, fp32.  Beside it are two or three symmetric matrices, A = X X^T and polynomials of it, each as its diagonal (fp32) and
// the rest: fp16, rows of `lde` elements, and fp32.  Only tiles on and above the diagonal exist.
// The fp32 copies lie in blocks of 32 x 32 as the epilogues' lanes hold them: eight groups of four columns, in each 32 rows of four elements.
constexpr int MUON_SYMMETRIC = 3;
struct MuonMat {
    int m, n;
    int ldx, lde;      // multiples of 64
    int transposed;    // 1: X is the tensor's transpose
    int precise;       // 1: products take the lo parts, too
    int tile;          // side of the products' tiles
    int twos;          // 1: the first two iterations in one
    int tensor;        // position in the caller's pointer arrays
    int piece_begin;   // its first piece of the norm in the group, and how many
    int n_pieces;
    int maps;          // index of its first tensor map (MUON_MAPS of them)
    float S, inv_S;
    float step_scale;  // of the update: x <- x - lr (step_scale O + wd x)
    int symmetric;     // how many symmetric matrices
    uint16_t *xhi[2], *xlo[2];
    uint16_t *ehi[MUON_SYMMETRIC], *elo[MUON_SYMMETRIC];
    float *x32, *e32[MUON_SYMMETRIC], *diag[MUON_SYMMETRIC];
    int *rest[2];      // of both X, by row, in MUON_REST: what the squares of the fp16 values leave out (not `precise` ones)
    // GRAM's sum over K is cut into `splits` parts of `split_steps` steps, which lie in `parts` until the last of them adds them up
    int splits, split_steps;
    int arrived;       // index of its first counter: one for each tile, CTA and warp of the epilogue
    float *parts;
};
// Tensor maps of a matrix (X twice, its lo parts, the symmetric matrices, theirs), three of each: boxes of 128 rows x 64 columns, of two times
// 64 x 64 side by side, both with 128-byte swizzle, and what an epilogue's warp writes: 32 x 64, or, in tiles of 128, 32 x 32 with 64-byte
// swizzle.  An operand is, for tiles of 256, 128 rows by 64 of K: the first where its rows run along K, the second where its columns do; for
// tiles of 128, 64 rows by 128 of K: the other way round.
enum { MUON_MAP_X = 0, MUON_MAP_XLO = 2, MUON_MAP_E = 4, MUON_MAP_ELO = 4 + MUON_SYMMETRIC, MUON_MAP_KINDS = 4 + 2 * MUON_SYMMETRIC };
constexpr int MUON_MAP_TWO = MUON_MAP_KINDS, MUON_MAP_OUT = 2 * MUON_MAP_KINDS, MUON_MAPS = 3 * MUON_MAP_KINDS;
constexpr int MUON_MAP_BYTES = 128;

// Off the diagonal, symmetric matrices lie in the workspace 256 times as large: entries of 1/m and less, and their lo parts, stay in fp16's normal range (of rank one,
// 96 rows: error 1.6e-4 without).  Entries of up to 255 remain possible: singular values up to about 3 within the iterations.
constexpr float MUON_EF_SCALE = 256.f, MUON_EF_INV = 1.f / 256.f;

// The diagonal of X X^T takes the squares of X's fp32 values: where one entry of a row outweighs the others, the rounding of its fp16 value, which
// elsewhere averages out, is that of the result (heavy-tailed 830 x 3320: entries off by up to 1.6e-3 of it, instead of 3e-4).  What is missing is
// summed up in whole multiples of 2^-36, in any order to the same bits: 2^-10 of the squares at most, below 2^31 multiples for singular values up
// to 5, beyond what MUON_EF_SCALE admits.
constexpr float MUON_REST = 68719476736.f, MUON_REST_INV = 1.f / 68719476736.f;

constexpr int MUON_PACK_TILE = 64;   // side of the tiles in which X is laid out

struct MuonTile {
    int mat;
    short i, j;  // tile row and column
};

// The products of all matrices are one list of tasks, a tile each; workers draw them in order, so a task may wait for what earlier ones
// write: `need` completions of its matrix's (each warp of an epilogue is one).
enum { MUON_GRAM = 0, MUON_POLY = 1, MUON_MUL = 2, MUON_UPDATE = 3, MUON_FINAL = 4 };
struct MuonTask {
    int product;
    short i, j;
    int part;
};
struct alignas(16) MuonProduct {  // what the tasks of one product of one matrix share
    int phase, mat;
    unsigned need;
    int steps;               // of muon_k_step(tile)
    int splits;              // GRAM: parts of the sum over K; `steps` are a part's
    int left, right, out;    // tensor maps of the operands and of the result
    int left_lo, right_lo, out_lo;
    int blocks;              // of x32 / e32 in a row of them
    int m, width;            // of the result
    int tensor, transposed;
    const float *src;        // fp32: POLY, MUL: the left factor; UPDATE, FINAL: X
    const float *src2;       // MUL: the right factor; GRAM: the parts
    float *dst;              // fp32 result, NULL: not needed
    const float *vec;        // POLY, MUL: the left factor's diagonal; UPDATE, FINAL: the polynomial's
    union {
        const float *vec2;   // MUL: the right factor's diagonal
        int *rest;           // GRAM: of the X that is read, zero afterwards; UPDATE: of the one that is written
    };
    float *diag;             // the result's diagonal
    float scale, step_scale; // GRAM: of A off the diagonal; FINAL: of O, of the update
    int last_steps;          // the last part's
    int arrived;             // GRAM: see MuonMat; tile (i, j)'s are those of tile j (j + 1) / 2 + i
};
static_assert(sizeof(MuonProduct) == 128, "read as eight 16-byte pieces");

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
    unsigned *ready;       // device: pieces of each matrix that are summed up, zero between launches
    float2 *scales;        // device: of each matrix, S / (||u|| + eps) in two factors
    unsigned *done;        // device: completions of each matrix's tasks
    unsigned *next_task;   // device
    unsigned *gave_up;     // device: not 0 once a wait of this launch has run out
    unsigned *arrived;     // device: parts of a sum that are there
    int piece;             // elements of a piece of the norm
    int from, to;
    int in_bf16, out_bf16;
    int nesterov;
    float mu, eps, lr, wd;
    float a, b, c;
    long long wait_cycles; // limit of each wait of the products
    int *status;           // DEMO_DEV_TIMEOUT once a wait of any launch has run out, until the host has asked
};

// Momentum update and the pieces' sums of squares; pieces [0, n_pieces) of the matrices [first, first + n).
cudaError_t muon_launch_norm(const MuonArgs &a, int first_mat, int n_mats, int n_pieces, DemoLaunch &dev, cudaStream_t stream);
// X = S u / (||u|| + eps), as hi + lo; clears the counters of the matrices [first_mat, first_mat + n_mats), n_arrived of their parts' from
// `arrived` on, the next task and the word that tells that a CTA has given up.
cudaError_t muon_launch_pack(const MuonArgs &a, const MuonTile *tiles, int n_tiles, int first_mat, int n_mats, int arrived, int n_arrived, DemoLaunch &dev,
                             cudaStream_t stream);
// All products, by pairs of CTAs.  precise: tiles of 128, of hi and lo parts.
cudaError_t muon_launch_products(int tile, bool precise, const MuonArgs &a, const MuonProduct *products, const MuonTask *tasks, int n_tasks, int workers, DemoLaunch &dev, cudaStream_t stream);
// Warps of an epilogue; each is a completion of a task in both CTAs.  (When they were chosen: sixteen for tiles of 128, too, 256 x 512 116 us
// instead of 107; eight of 32 columns for tiles of 256, the 300M-class layers 11.2 ms instead of 10.9.)
constexpr int muon_k_step(int tile) { return 16384 / tile; }
constexpr int muon_epilogue_warps(int tile) { return tile == 256 ? 16 : 8; }

// How a set would be worked on by a device of `sm_count` SMs; needs none (for tests).  Of each group seven numbers: 1 where products take the lo parts, the
// tiles' side, matrices, tasks, tasks that can be in work at once, workers, 1 where its first matrix does the first two iterations in one.  Returns how many groups there are, -1 on failure.
extern "C" int demo_muon_plan(const demo_muon_config *cfg, const demo_tensor_desc *tensors, int n_tensors, int sm_count, int *groups, int most_groups);
