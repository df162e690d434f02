// Orthogonalised updates: Newton-Schulz iterations on whole weight matrices, on the tensor cores.
//
//   X_0 = u / (||u||_F + eps);  A = X X^T;  X <- a X + (b A + c A^2) X
//
// as three products an iteration, the tasks of one persistent kernel:
//   GRAM    A = X X^T                        symmetric: the tiles on and above the diagonal
//   POLY    B = a + b A + c A^2, from A^2     symmetric, too
//   UPDATE  X <- B X
// Wide matrices do the first two iterations in one: the second's A is A B^2, a polynomial of the first's, and X <- (B' B) X is multiplied once,
//   GRAM, POLY, MUL T = A B, MUL A' = T B, POLY B', MUL Q = B' B, UPDATE
// which for n = 4 m takes 17 m^3 instead of 26 and reads and writes X once.
// Operands are fp16 (11 bits, accumulated in fp32), and what would lose accuracy in them is kept out of them:
//   * the linear term, on which small singular values live alone (they grow by a = 3.4 an iteration, rounding noise with them), and all
//     other sums outside the products are formed from fp32 copies;
//   * the diagonals of symmetric matrices, of order one in the last iterations, where a X and (b A + c A^2) X nearly cancel, never pass
//     through fp16: with P = D + E, Q = D' + E', P Q = D D' + D E' + E D' + E E', and only E E' is a product on the tensor cores; and that
//     of X X^T is the one of X's fp32 values (muon.h, MUON_REST).
// Relative error of the result against 64 bits, 1024 x 4096: Gaussian 3e-4, of rank 1, 32 and 128 9e-4, 6e-4 and 9e-4; 400 x 1200 5e-4 and 1.4e-3,
// 1.2e-3, 1.7e-3 (plain bf16 operands, 1024 x 4096: Gaussian 1.3e-2, of rank 1 and 32 1.2 and 0.2; fp16: 1.7e-3, 0.15 and 0.03).  Equal entries are
// rounded alike, which nothing averages out: all entries equal, 512 x 512 1.1e-2, 1111 x 3001 2.2e-2.  The error grows as matrices shrink, so those of up to 384 rows take the lo parts of the products' operands, too.  More iterations in one would multiply less (all
// five 29 m^3 for n = 4 m instead of 56), but their B' B is rounded to 11 bits after the last one that could take noise away: [1, 2, 2] has up to
// five times the error where the rank is low, [5] an error of 0.15.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "demo_internal.h"
#include "fast_common.cuh"
#include "launch.cuh"
#include "muon.h"

namespace {

using namespace fastk;

// ---- momentum, norm, layout ---------------------------------------------------------------------------------------------------

__device__ __forceinline__ float load_in(const void *p, long long i, int bf16)
{
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]) : static_cast<const float *>(p)[i];
}

constexpr int NORM_THREADS = 256;

// The matrix whose pieces hold `piece`: the last with piece_begin <= piece.
__device__ __forceinline__ int find_mat(const MuonMat *mats, int first, int n, int piece)
{
    int lo = first, hi = first + n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (mats[mid].piece_begin <= piece)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double v, double *scratch)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_down_sync(0xffffffffu, v, d);
    __syncthreads();  // (scratch may still be read from the sum before)
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0;
#pragma unroll
    for (int w = 0; w < NORM_THREADS / 32; ++w) s += scratch[w];
    return s;
}

// Sums of squares in 64 bits: gradients of 1e-20 and of 1e+20 have a norm, too.
__global__ void __launch_bounds__(NORM_THREADS) muon_norm_kernel(MuonArgs a, int first_mat, int n_mats)
{
    const StreamOrder order(1);
    __shared__ double scratch[NORM_THREADS / 32];
    const int e = find_mat(a.mats, first_mat, n_mats, blockIdx.x);
    const MuonMat &mat = a.mats[e];
    const long long n = (long long)mat.m * mat.n, at = (long long)(blockIdx.x - mat.piece_begin) * a.piece;
    order.begin();
    const void *in = a.in[mat.tensor];
    float *mom = a.from == MUON_FROM_STEP ? a.mom[mat.tensor] : nullptr;
    double sum = 0;
    auto one = [&](float g, float &m) {
        if (mom) {
            m = fmaf(a.mu, m, g);
            g = a.nesterov ? fmaf(a.mu, m, g) : m;
        }
        sum += (double)g * (double)g;
    };
    const int len = (int)(n - at < a.piece ? n - at : a.piece);
    if (at == 0 && !mat.precise)
        for (int i = threadIdx.x; i < mat.m; i += NORM_THREADS) mat.rest[0][i] = mat.rest[1][i] = 0;
#pragma unroll 4
    for (int i = threadIdx.x * 4; i + 3 < len; i += NORM_THREADS * 4) {
        float g[4];
        if (a.in_bf16) {
            const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(in) + at + i);
            g[0] = __uint_as_float(v.x << 16);
            g[1] = __uint_as_float(v.x & 0xffff0000u);
            g[2] = __uint_as_float(v.y << 16);
            g[3] = __uint_as_float(v.y & 0xffff0000u);
        } else {
            const float4 v = *reinterpret_cast<const float4 *>(static_cast<const float *>(in) + at + i);
            g[0] = v.x, g[1] = v.y, g[2] = v.z, g[3] = v.w;
        }
        float4 m = make_float4(0.f, 0.f, 0.f, 0.f);
        if (mom) m = *reinterpret_cast<const float4 *>(mom + at + i);
        one(g[0], m.x);
        one(g[1], m.y);
        one(g[2], m.z);
        one(g[3], m.w);
        if (mom) *reinterpret_cast<float4 *>(mom + at + i) = m;
    }
    const int rest = (len & ~3) + threadIdx.x;
    if (rest < len) {
        const float g = load_in(in, at + rest, a.in_bf16);
        float m = mom ? mom[at + rest] : 0.f;
        one(g, m);
        if (mom) mom[at + rest] = m;
    }
    const double s = block_sum(sum, scratch);
    // the matrix's last piece to be ready adds them all up, in one order whichever it is
    __shared__ int last;
    if (threadIdx.x == 0) {
        a.partials[blockIdx.x] = s;
        __threadfence();
        last = atomicInc(a.ready + e, (unsigned)mat.n_pieces - 1u) == (unsigned)mat.n_pieces - 1u;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0;
    for (int p = threadIdx.x; p < mat.n_pieces; p += NORM_THREADS) sum += __ldcg(a.partials + mat.piece_begin + p);
    const double norm = sqrt(block_sum(sum, scratch));
    if (threadIdx.x == 0) {
        const double all = norm + (double)a.eps, scale = all > 0 ? (double)mat.S / all : 1;
        // in two factors, so that neither leaves the range of fp32 where the norm is near its ends
        const float scale1 = (float)exp2(floor(0.5 * log2(scale)));
        a.scales[e] = make_float2(scale1, (float)(scale / (double)scale1));
    }
}

// x^2 - h^2, and a sum of them as MuonMat's `rest` holds it
__device__ __forceinline__ float add_rest(float sum, float x, float h) { return fmaf(x - h, x + h, sum); }
__device__ __forceinline__ int rest_units(float sum, float inv_S) { return __float2int_rn(sum * inv_S * inv_S * MUON_REST); }

__device__ __forceinline__ float2 unpack2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }
__device__ __forceinline__ uint32_t pack2(float x, float y)
{
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Tiles of 128 read pad columns along K: those of the other matrices of the workspace beside four elements (i, j ..) of X are set to zero.
__device__ __forceinline__ void clear_pads(const MuonMat &mat, int i, int j)
{
    if (j + 4 > mat.n)
        for (int l = max(j, mat.n); l < j + 4; ++l) {
            mat.xhi[1][(size_t)i * mat.ldx + l] = 0;
            mat.xlo[1][(size_t)i * mat.ldx + l] = 0;
        }
    if (j < 64)  // (sixteen threads a row)
        for (int l = mat.m + j / 4; l < mat.lde; l += 16)
            for (int e = 0; e < mat.symmetric; ++e) {
                mat.ehi[e][(size_t)i * mat.lde + l] = 0;
                mat.elo[e][(size_t)i * mat.lde + l] = 0;
            }
}

// Tiles of 64 x 64 elements of X, `each` one after the other to a CTA: the first one's look-ups, three loads that wait for one another, serve the
// others, too (67 million elements, 142 us one tile a CTA, 123 four, 134 eight).
__global__ void __launch_bounds__(NORM_THREADS) muon_pack_kernel(MuonArgs a, const MuonTile *tiles, int n_tiles, int each, int first_mat, int n_mats, int arrived, int n_arrived)
{
    const StreamOrder order(1);
    constexpr int T = MUON_PACK_TILE;
    __shared__ float tile[T][T + 1];
    const int x = (threadIdx.x & 15) * 4, y = threadIdx.x >> 4;  // four elements of a row, sixteen rows at a time
    constexpr int ROWS = NORM_THREADS / 16;
    order.begin();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.next_task = *a.gave_up = 0;
    for (int k = blockIdx.x * NORM_THREADS + threadIdx.x; k < n_mats; k += gridDim.x * NORM_THREADS) a.done[first_mat + k] = 0;
    for (int k = blockIdx.x * NORM_THREADS + threadIdx.x; k < n_arrived; k += gridDim.x * NORM_THREADS) a.arrived[arrived + k] = 0;
    for (int n = blockIdx.x * each, end = min(n_tiles, n + each); n < end; ++n) {
        const MuonTile t = tiles[n];
        const MuonMat &mat = a.mats[t.mat];
        const int transposed = mat.transposed, rows = transposed ? mat.n : mat.m, cols = transposed ? mat.m : mat.n;
        // tile row i0, column j0 of X; of the tensor, the other way round where X is its transpose
        const int i0 = t.i * T, j0 = t.j * T;
        const int r0 = transposed ? j0 : i0, c0 = transposed ? i0 : j0;
        const void *in = a.in[mat.tensor];
        const float *mom = a.from == MUON_FROM_STEP ? a.mom[mat.tensor] : nullptr;
        float u[T / ROWS][4];
        const bool whole = (cols & 3) == 0;
#pragma unroll
        for (int k = 0; k < T / ROWS; ++k) {
            const int r = r0 + y + k * ROWS, c = c0 + x;
            const long long at = (long long)r * cols + c;
            float m[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int l = 0; l < 4; ++l) u[k][l] = 0.f;
            if (r < rows) {
                if (whole && c < cols) {
                    if (a.in_bf16) {
                        const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(in) + at);
                        u[k][0] = __uint_as_float(v.x << 16);
                        u[k][1] = __uint_as_float(v.x & 0xffff0000u);
                        u[k][2] = __uint_as_float(v.y << 16);
                        u[k][3] = __uint_as_float(v.y & 0xffff0000u);
                    } else {
                        const float4 v = *reinterpret_cast<const float4 *>(static_cast<const float *>(in) + at);
                        u[k][0] = v.x, u[k][1] = v.y, u[k][2] = v.z, u[k][3] = v.w;
                    }
                    if (mom) {
                        const float4 v = *reinterpret_cast<const float4 *>(mom + at);
                        m[0] = v.x, m[1] = v.y, m[2] = v.z, m[3] = v.w;
                    }
                } else if (!whole) {
#pragma unroll
                    for (int l = 0; l < 4; ++l)
                        if (c + l < cols) {
                            u[k][l] = load_in(in, at + l, a.in_bf16);
                            if (mom) m[l] = mom[at + l];
                        }
                }
                if (mom) {
#pragma unroll
                    for (int l = 0; l < 4; ++l) u[k][l] = a.nesterov ? fmaf(a.mu, m[l], u[k][l]) : m[l];
                }
            }
        }
        const float2 scale = a.scales[t.mat];
#pragma unroll
        for (int k = 0; k < T / ROWS; ++k)
#pragma unroll
            for (int l = 0; l < 4; ++l) u[k][l] = u[k][l] * scale.x * scale.y;
        if (transposed) {
#pragma unroll
            for (int k = 0; k < T / ROWS; ++k)
#pragma unroll
                for (int l = 0; l < 4; ++l) tile[x + l][y + k * ROWS] = u[k][l];
        } else {
#pragma unroll
            for (int k = 0; k < T / ROWS; ++k)
#pragma unroll
                for (int l = 0; l < 4; ++l) tile[y + k * ROWS][x + l] = u[k][l];
        }
        __syncthreads();
        float rest[T / ROWS];
#pragma unroll
        for (int k = 0; k < T / ROWS; ++k) {
            const int i = y + k * ROWS;
            rest[k] = 0.f;
            if (i0 + i < mat.m) {  // (j < ldx, a multiple of the tile's side)
                const size_t at = (size_t)(i0 + i) * mat.ldx + j0 + x;
                float w[4];
#pragma unroll
                for (int l = 0; l < 4; ++l) w[l] = tile[i][x + l];
                *reinterpret_cast<uint2 *>(mat.xhi[0] + at) = make_uint2(pack2(w[0], w[1]), pack2(w[2], w[3]));
                if (mat.tile == 128) clear_pads(mat, i0 + i, j0 + x);
                if (mat.precise) {
#pragma unroll
                    for (int l = 0; l < 4; ++l) w[l] -= __half2float(__float2half_rn(w[l]));
                    *reinterpret_cast<uint2 *>(mat.xlo[0] + at) = make_uint2(pack2(w[0], w[1]), pack2(w[2], w[3]));
                } else {
#pragma unroll
                    for (int l = 0; l < 4; ++l) rest[k] = add_rest(rest[k], w[l], __half2float(__float2half_rn(w[l])));
                }
            }
            // block k of the tile's four, a warp for each of its groups of four columns
            const int lane = threadIdx.x & 31, quad = threadIdx.x >> 5, bi = k >> 1, bj = k & 1;
            if (i0 + 32 * bi < mat.m) {
                const float *from = &tile[32 * bi + lane][32 * bj + 4 * quad];
                float *to = mat.x32 + ((size_t)(i0 / 32 + bi) * (mat.ldx / 32) + j0 / 32 + bj) * 1024 + quad * 128 + lane * 4;
                *reinterpret_cast<float4 *>(to) = make_float4(from[0], from[1], from[2], from[3]);
            }
        }
        if (!mat.precise) {
            // the sums of four rows over sixteen lanes: the first exchanges leave a lane half of the rows each, five shuffles instead of sixteen
            // (67 million elements 123 us instead of 180)
            static_assert(T / ROWS == 4, "");
            const int lane = threadIdx.x & 31;
            const bool b8 = lane & 8, b4 = lane & 4;
            const float r0 = (b8 ? rest[2] : rest[0]) + __shfl_xor_sync(0xffffffffu, b8 ? rest[0] : rest[2], 8);
            const float r1 = (b8 ? rest[3] : rest[1]) + __shfl_xor_sync(0xffffffffu, b8 ? rest[1] : rest[3], 8);
            float r = (b4 ? r1 : r0) + __shfl_xor_sync(0xffffffffu, b4 ? r0 : r1, 4);
            r += __shfl_xor_sync(0xffffffffu, r, 2);
            r += __shfl_xor_sync(0xffffffffu, r, 1);
            const int i = i0 + y + (2 * b8 + b4) * ROWS;
            if ((lane & 3) == 0 && i < mat.m) atomicAdd(mat.rest[0] + i, rest_units(r, mat.inv_S));
        }
        __syncthreads();  // (the next tile comes into the same place)
    }
}

// ---- products -----------------------------------------------------------------------------------------------------------------

constexpr int MMA = 1, SCHEDULER = 2, LOAD_RIGHT = 3, FIRST_EPI = 4;  // warps; warp 0 loads the left operand
constexpr int TMEM_COLS = 512;
template <int TILE>
struct Shape {
    static constexpr int EPI_WARPS = muon_epilogue_warps(TILE), THREADS = 32 * (FIRST_EPI + EPI_WARPS);
    // a CTA's rows of both operands of a step of K, as many steps as there is room for beside 4 KB for each warp of the epilogue
    static constexpr int ROWS = TILE / 2, K = muon_k_step(TILE), OPERAND = ROWS * K * 2, STAGE = 2 * OPERAND, STAGES = (224 * 1024 - EPI_WARPS * 4096) / STAGE;
    static constexpr int SMEM = STAGES * STAGE + EPI_WARPS * 4096 + 1024;
};

__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// Shared-memory matrix descriptor of a 128-byte swizzled operand: start address, leading and stride byte offsets, version 1, layout 2.
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr, uint32_t lbo, uint32_t sbo)
{
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | (uint64_t)((lbo >> 4) & 0x3FFFu) << 16 | (uint64_t)((sbo >> 4) & 0x3FFFu) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}

__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
                 "r"(accumulate)
                 : "memory");
}
// Arrives at `bar` of both CTAs of the pair once the MMAs issued so far are done.
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// One operand of a step (MUON_MAPS), one copy: a loading warp takes 340 cycles for one and what belongs to it, whatever its size.  The loads of
// both CTAs are counted by the barrier of the first.
__device__ __forceinline__ void load_2d(uint32_t dst, const void *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x),
                 "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void load_3d(uint32_t dst, const void *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(0),
                 "r"(y), "r"(x / 64), "r"(bar)
                 : "memory");
}
template <int TILE>
__device__ __forceinline__ void load_operand(uint32_t dst, const char *map, bool columns, int at, int k, uint32_t bar)
{
    if ((TILE == 256) != columns)
        load_2d(dst, map, columns ? at : k, columns ? k : at, bar);
    else
        load_3d(dst, map + MUON_MAP_TWO * MUON_MAP_BYTES, columns ? at : k, columns ? k : at, bar);
}
// (release at the scope of the CTA even where the barrier is another CTA's: one of the cluster's would wait for this warp's stores to memory)
__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void arrive_cluster(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void arrive_release_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool wait_local(uint32_t bar, unsigned parity, const MuonArgs &a) { return mbar_wait_bounded(bar, parity, a.wait_cycles); }
// One lane of a warp that runs converged.  The loading and the MMA warp loop with all their lanes and leave only the instructions themselves to
// one: operands formed in divergent code cost each MMA and each copy 100 to 200 cycles on their way to uniform registers (a step of a 256 tile
// 581 cycles instead of 512, which is what the products take; 256 x 512 159 us instead of 136).
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ bool all_of(bool ok) { return __all_sync(0xffffffffu, ok); }
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
// Whether a phase is complete, without the pause that a try_wait may take (4 us).
__device__ __forceinline__ bool mbar_test(uint32_t bar, unsigned parity)
{
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// as wait_local, seeing what another CTA of the cluster did before its arrival
__device__ __forceinline__ bool wait_cluster(uint32_t bar, unsigned parity, const MuonArgs &a)
{
    const long long t0 = clock64();
    for (;;) {
        unsigned ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity)
            : "memory");
        if (ok) return true;
        if (clock64() - t0 > a.wait_cycles) return false;
    }
}

// ---- epilogues: a warp's block is 32 rows, a lane's row, by 16 columns ---------------------------------------------------------

// 16 consecutive fp32 columns of this thread's tensor-memory lane.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&v)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
          "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(taddr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// 32 x 32 results on their way to the caller's tensor pass through shared memory, from a row a lane to pieces of eight columns: four lanes then
// cover 32 columns of a row.  16-byte quads are stored where neither the rows' writes, nor the pieces' reads, nor reads down the columns meet
// in a bank.
__device__ __forceinline__ int quad_at(int row, int quad) { return row * 32 + ((quad ^ (row & 7) ^ ((row >> 3) << 1)) << 2); }
__device__ __forceinline__ void read_piece(const float *st, int row, int q, float (&v)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(st + quad_at(row, 2 * q)), b = *reinterpret_cast<const float4 *>(st + quad_at(row, 2 * q + 1));
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
// rows 8 q .. 8 q + 7 of one column
__device__ __forceinline__ void read_column(const float *st, int col, int q, float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = st[quad_at(8 * q + k, col >> 2) + (col & 3)];
}

// Eight neighbouring results (of a tensor row, from column c on) to the caller's tensor.  x: the parameters there, loaded beforehand where
// `whole` says that they can be in 16-byte pieces.
__device__ __forceinline__ bool whole_piece(const MuonArgs &a, int c, int cols)
{
    return cols - c >= 8 && (a.to == MUON_TO_OUTPUT && a.out_bf16 ? (cols & 7) == 0 : (cols & 3) == 0);
}
__device__ __forceinline__ void deliver(const MuonArgs &a, void *out, size_t at, int left, bool whole, const float (&o)[8], float keep, const float4 (&old)[2])
{
    if (a.to == MUON_TO_PARAMS) {  // o = -lr s O
        float *x = static_cast<float *>(out) + at;
        if (whole) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
                reinterpret_cast<float4 *>(x)[q] = make_float4(fmaf(old[q].x, keep, o[4 * q]), fmaf(old[q].y, keep, o[4 * q + 1]), fmaf(old[q].z, keep, o[4 * q + 2]),
                                                               fmaf(old[q].w, keep, o[4 * q + 3]));
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left) x[k] = fmaf(x[k], keep, o[k]);
        }
    } else if (a.out_bf16) {
        __nv_bfloat16 *p = static_cast<__nv_bfloat16 *>(out) + at;
        if (whole) {
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(o[2 * q], o[2 * q + 1]);
                w[q] = *reinterpret_cast<const uint32_t *>(&b);
            }
            *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left) p[k] = __float2bfloat16_rn(o[k]);
        }
    } else {
        float *p = static_cast<float *>(out) + at;
        if (whole) {
            reinterpret_cast<float4 *>(p)[0] = make_float4(o[0], o[1], o[2], o[3]);
            reinterpret_cast<float4 *>(p)[1] = make_float4(o[4], o[5], o[6], o[7]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left) p[k] = o[k];
        }
    }
}

// (past the L1, which may hold these addresses as they were an iteration ago)
__device__ __forceinline__ void load_block(const float *p, float4 (&x)[4])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = __ldcg(reinterpret_cast<const float4 *>(p + k * 128));
}
__device__ __forceinline__ void store_block(float *p, const float (&v)[16])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) __stcg(reinterpret_cast<float4 *>(p + k * 128), make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]));
}
__device__ __forceinline__ float part(const float4 (&x)[4], int k) { return reinterpret_cast<const float *>(x)[k]; }

struct BlockAt {
    size_t fp32;   // the lane's place in the block of the fp32 copies
    uint32_t tmem;
    int r0, j0, number, lane;  // row and column of the result; the how-manieth of the warp's blocks
    float column;  // POLY, MUL: the right factor's diagonal at column j0 + lane, lane < 16
    unsigned char *st;  // the warp's 4 KB of shared memory
};

// The fp16 values of a block into the warp's part of shared memory, from where one copy writes all of them: rows of 128 bytes, the 16-byte
// pieces of row r at piece ^ (r % 8), or, in tiles of 128, where there are two blocks and the lo parts behind the hi parts, rows of 64 bytes at
// piece ^ (r / 2 % 4).
template <int TILE, bool PRECISE>
__device__ __forceinline__ void stage_halves(const BlockAt &b, const float (&v)[16])
{
    uint32_t p[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) p[k] = pack2(v[2 * k], v[2 * k + 1]);
    auto put = [&](unsigned char *at) {
        const int swap = TILE == 256 ? b.lane & 7 : b.lane >> 1 & 3, piece = 2 * b.number;
        unsigned char *row = at + b.lane * (TILE == 256 ? 128 : 64);
        *reinterpret_cast<uint4 *>(row + ((piece ^ swap) << 4)) = make_uint4(p[0], p[1], p[2], p[3]);
        *reinterpret_cast<uint4 *>(row + (((piece + 1) ^ swap) << 4)) = make_uint4(p[4], p[5], p[6], p[7]);
    };
    put(b.st);
    if (PRECISE) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float2 h = unpack2(p[k]);
            p[k] = pack2(v[2 * k] - h.x, v[2 * k + 1] - h.y);
        }
        put(b.st + 2048);
    }
}

// The lane whose row meets the diagonal in this block takes its element out of it.
__device__ __forceinline__ float take_own(const BlockAt &b, float (&v)[16])
{
    float own = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k)
        if (b.j0 + k == b.r0 + b.lane) {
            own = v[k];
            v[k] = 0.f;
        }
    return own;
}
__device__ __forceinline__ bool on_diagonal(const BlockAt &b) { return (b.r0 ^ b.j0) < 32; }  // (both below 2^31, multiples of 32 and 16)
__device__ __forceinline__ bool has_own(const BlockAt &b) { return (unsigned)(b.r0 + b.lane - b.j0) < 16u; }

// E = A off the diagonal, d on it.  v: the products; rest: what the row's own lacks.
template <int TILE, bool PRECISE>
__device__ __forceinline__ void block_gram(const MuonProduct &t, const BlockAt &b, float (&v)[16], float rest)
{
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] *= t.scale;
    if (on_diagonal(b)) {
        const float own = take_own(b, v);
        if (has_own(b)) {
            __stcg(t.diag + b.r0 + b.lane, fmaf(own, MUON_EF_INV, rest));
            if (!PRECISE && b.r0 + b.lane < t.m) __stcg(t.rest + b.r0 + b.lane, 0);
        }
    }
    stage_halves<TILE, PRECISE>(b, v);
    store_block(t.dst + b.fp32, v);
}

// The parts of a sum, in their order.
__device__ __forceinline__ void add_parts(const float *p, int n, size_t stride, float (&v)[16])
{
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = 0.f;
#pragma unroll 2
    for (int s = 0; s < n; ++s) {
        float4 x[4];
        load_block(p + (size_t)s * stride, x);
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] += part(x, k);
    }
}

// B = a + b A + c A^2
template <int TILE, bool PRECISE>
__device__ __forceinline__ void block_poly(const MuonArgs &a, const MuonProduct &t, const BlockAt &b, const float4 (&e)[4], float di)
{
    float v[16];
    tmem_ld16(b.tmem, v);
    if (on_diagonal(b)) {
        const float own = take_own(b, v) * (MUON_EF_INV * MUON_EF_INV);
        if (has_own(b)) __stcg(t.diag + b.r0 + b.lane, a.a + fmaf(a.b, di, a.c * fmaf(di, di, own)));
    }
    const float base = fmaf(a.c, di, a.b), scale = a.c * MUON_EF_INV;
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = fmaf(fmaf(a.c, __shfl_sync(0xffffffffu, b.column, k), base), part(e, k), scale * v[k]);  // (E's own diagonal is zero)
    stage_halves<TILE, PRECISE>(b, v);
    if (t.dst) store_block(t.dst + b.fp32, v);
}

// P Q, of matrices that commute
template <int TILE, bool PRECISE>
__device__ __forceinline__ void block_mul(const MuonProduct &t, const BlockAt &b, const float4 (&e)[4], float di)
{
    float v[16];
    float4 f[4];
    load_block(t.src2 + b.fp32, f);
    tmem_ld16(b.tmem, v);
    const float dj = __shfl_sync(0xffffffffu, b.column, b.lane & 15);  // (of the lane's own element, where the block holds it)
    if (on_diagonal(b)) {
        const float own = take_own(b, v) * (MUON_EF_INV * MUON_EF_INV);
        if (has_own(b)) __stcg(t.diag + b.r0 + b.lane, fmaf(di, dj, own));
    }
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = fmaf(di, part(f, k), fmaf(part(e, k), __shfl_sync(0xffffffffu, b.column, k), v[k] * MUON_EF_INV));
    stage_halves<TILE, PRECISE>(b, v);
    if (t.dst) store_block(t.dst + b.fp32, v);
}

// X <- B X
template <int TILE, bool PRECISE>
__device__ __forceinline__ void block_update(const MuonProduct &t, const BlockAt &b, const float4 (&x)[4], float di, float &rest)
{
    float v[16];
    tmem_ld16(b.tmem, v);
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = fmaf(di, part(x, k), v[k] * MUON_EF_INV);
    if (!PRECISE) {
        if (t.width - b.j0 < 16) {  // (what is outside the matrix is no part of it)
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (k >= t.width - b.j0) v[k] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < 16; k += 2) {
            const float2 h = unpack2(pack2(v[k], v[k + 1]));
            rest = add_rest(add_rest(rest, v[k], h.x), v[k + 1], h.y);
        }
    }
    stage_halves<TILE, PRECISE>(b, v);
    store_block(t.dst + b.fp32, v);
}

// The same, the last time: to the caller's tensor, 32 columns at a time where the warp has them.  more: another 16 columns follow.
__device__ __forceinline__ void block_final(const MuonArgs &a, const MuonProduct &t, const BlockAt &b, const float4 (&x)[4], float di, bool more)
{
    const bool params = a.to == MUON_TO_PARAMS;
    const float scale = params ? -a.lr * t.step_scale : t.scale, keep = 1.f - a.lr * a.wd;
    void *out = a.out[t.tensor];
    float *st = reinterpret_cast<float *>(b.st);
    const int half = b.number & 1;
    {
        float v[16];
        tmem_ld16(b.tmem, v);
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = fmaf(di, part(x, k), v[k] * MUON_EF_INV) * scale;
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<float4 *>(st + quad_at(b.lane, 4 * half + k)) = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
    }
    if (!half && more) return;
    __syncwarp();
    // the lane's pieces of the tensor: rows 8 i + lane / 4, eight columns; of X, where it is the transpose, the other way round
    const int j0 = b.j0 - 16 * half, wide = 16 * (half + 1), sub = b.lane >> 2, q = b.lane & 3;
    const int r0 = t.transposed ? j0 : b.r0, c = (t.transposed ? b.r0 : j0) + 8 * q;
    const int rows = min(t.transposed ? t.width : t.m, r0 + (t.transposed ? wide : 32)), cols = t.transposed ? t.m : t.width;
    const bool mine = c < cols && (t.transposed || 8 * q < wide), whole = whole_piece(a, c, cols);
    float4 old[4][2];
    if (params && whole && mine) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + 8 * i + sub;
            if (r < rows) {
                const float4 *from = reinterpret_cast<const float4 *>(static_cast<const float *>(out) + (size_t)r * cols + c);
                old[i][0] = from[0];
                old[i][1] = from[1];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 8 * i + sub;
        if (!mine || r >= rows) continue;
        float v[8];
        if (t.transposed)
            read_column(st, 8 * i + sub, q, v);
        else
            read_piece(st, 8 * i + sub, q, v);
        deliver(a, out, (size_t)r * cols + c, cols - c, whole, v, keep, old[i]);
    }
    __syncwarp();
}

__device__ __forceinline__ unsigned load_acquire(const unsigned *p)
{
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// Until `need` completions of a matrix are there.  False when that takes too long or another CTA of this launch has given up.
__device__ __forceinline__ bool wait_task(const unsigned *done, unsigned need, const MuonArgs &a)
{
    if (load_acquire(done) >= need) return true;
    const long long t0 = clock64();
    for (unsigned n = 0; load_acquire(done) < need; ++n) {
        __nanosleep(20);
        if ((n & 1023) == 1023 && (clock64() - t0 > a.wait_cycles || *static_cast<const volatile unsigned *>(a.gave_up) != 0)) return false;
    }
    return true;
}
__device__ __forceinline__ void fence_proxy_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }

struct alignas(16) RingEntry {
    MuonProduct p;
    int i, j, end, part, k0, steps, pad[2];  // part: of a sum over K, from step k0 on
};

// All products of all iterations, by persistent workers, pairs of CTAs.  Tasks are drawn in the list's order from one counter, so
// whatever a task waits for is done already or in the hands of a worker that runs: no worker has to be resident for another to go on.
// Two warps load, one each operand, one issues the MMAs, sixteen (eight in tiles of 128) read accumulators back.  There are two accumulators, so that the
// products of a task run beside the epilogue of the one before.  A fourth kind of warp schedules: that of a worker's first CTA draws the tasks and waits until they may start, and in
// both CTAs it puts what the others need to know of one into a ring, up to four ahead (by the loading warp itself: its look-ups and waits,
// 3500 cycles a task, leave the tensor core without data).
// Symmetric matrices exist above the diagonal only: left of it a panel's operand is loaded from the rows above, as its transpose.
// A worker's tile is TILE x TILE: 256, of which each CTA's tensor memory holds half the rows, or 128, for small matrices: of its 64 rows a CTA
// then holds the left 64 columns in lanes 0 .. 63 and the right ones in lanes 64 .. 127.
template <int TILE, bool PRECISE>
__global__ void __launch_bounds__(Shape<TILE>::THREADS, 1) muon_products_kernel(MuonArgs a, const MuonProduct *products, const MuonTask *tasks, int n_tasks)
{
    const StreamOrder order(1);
    constexpr int ROWS = Shape<TILE>::ROWS, K = Shape<TILE>::K, OPERAND = Shape<TILE>::OPERAND, STAGE = Shape<TILE>::STAGE, STAGES = Shape<TILE>::STAGES, EPI_WARPS = Shape<TILE>::EPI_WARPS;
    constexpr int RING = 4, NEAR_STEPS = 512 / K;
    extern __shared__ unsigned char raw[];
    __shared__ unsigned long long bars[2 * STAGES + 4 + 5 * RING + 2];
    __shared__ RingEntry ring[RING];
    __shared__ int drawn_ring[RING];
    __shared__ uint32_t tmem_slot;
    const uint32_t raw_s = smem_u32(raw), base = (raw_s + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, t_full = empty + 8 * STAGES, t_empty = t_full + 16, r_full = t_empty + 16,
                   r_empty = r_full + 8 * RING, q_full = r_empty + 8 * RING, q_empty = q_full + 8 * RING, go_full = q_empty + 8 * RING, near_end = go_full + 8 * RING, drained = near_end + 8;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full + 8 * s, 2);  // a loading warp each of the first CTA
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(t_full + 8 * s, 1);
            mbar_init(t_empty + 8 * s, 2 * EPI_WARPS);
        }
        for (int s = 0; s < RING; ++s) {
            mbar_init(r_full + 8 * s, 1);
            mbar_init(r_empty + 8 * s, EPI_WARPS + (rank == 0 ? 3 : 2));  // the epilogues, the loading warps and the first CTA's MMA warp
            mbar_init(q_full + 8 * s, 1);
            mbar_init(q_empty + 8 * s, 1);
            mbar_init(go_full + 8 * s, 1);
        }
        mbar_init(near_end, 1);
        mbar_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    order.begin();
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    cluster_sync();
    tc_after();
    const uint32_t tmem = tmem_slot;
    bool ok = true;
    int slot = 0;  // of the ring
    unsigned turn = 0;
    auto next_slot = [&] {
        if (++slot == RING) slot = 0, turn ^= 1;
    };

    if (warp == SCHEDULER) {
        if (lane == 0) {
            int last_product = -1;
            unsigned near_turn = 0;
            unsigned drawn = rank == 0 ? atomicAdd(a.next_task, 1u) : 0u;
            for (;;) {
                int t;
                if (rank == 0) {
                    t = drawn < (unsigned)n_tasks ? (int)drawn : -1;
                    // the second CTA looks the task up, too, while this one waits for what the task needs
                    ok = wait_cluster(q_empty + 8 * slot, turn ^ 1, a);
                    if (!ok) break;
                    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_rank(smem_u32(drawn_ring + slot), 1)), "r"(t) : "memory");
                    arrive_release_cluster(map_to_rank(q_full + 8 * slot, 1));
                } else {
                    ok = wait_cluster(q_full + 8 * slot, turn, a);
                    if (!ok) break;
                    t = *static_cast<volatile int *>(drawn_ring + slot);
                }
                MuonTask tk{0, 0, 0, 0};
                if (t >= 0) tk = tasks[t];
                uint4 words[8];
                {
                    const uint4 *from = reinterpret_cast<const uint4 *>(products + tk.product);
#pragma unroll
                    for (int k = 0; k < 8; ++k) words[k] = __ldg(from + k);
                }
                const MuonProduct &p = *reinterpret_cast<const MuonProduct *>(words);
                if (t >= 0 && tk.product != last_product) {
                    last_product = tk.product;
                    for (int lo = 0; lo < (PRECISE ? 2 : 1); ++lo) {
                        const char *l = a.maps + (size_t)(lo ? p.left_lo : p.left) * MUON_MAP_BYTES, *r = a.maps + (size_t)(lo ? p.right_lo : p.right) * MUON_MAP_BYTES;
                        if (TILE == 256 || p.phase != MUON_GRAM) {
                            tmap_acquire(l);
                            tmap_acquire(r);
                        }
                        if (TILE == 128 || p.phase != MUON_GRAM) {
                            tmap_acquire(l + MUON_MAP_TWO * MUON_MAP_BYTES);
                            tmap_acquire(r + MUON_MAP_TWO * MUON_MAP_BYTES);
                        }
                        if (p.phase != MUON_FINAL) tmap_acquire(a.maps + (size_t)(lo ? p.out_lo : p.out) * MUON_MAP_BYTES);
                    }
                }
                if (rank == 0) {
                    ok = t < 0 || wait_task(a.done + p.mat, p.need, a);
                    if (!ok) break;
                    arrive_release_cluster(map_to_rank(go_full + 8 * slot, 1));
                } else {
                    ok = wait_cluster(go_full + 8 * slot, turn, a);
                    if (!ok) break;
                    // The slot is free behind this wait only: where tasks have one step, the first CTA gets as far as the slot's next task before any of
                    // this one's data is needed, and a barrier that is completed twice looks as if it had never been.
                    arrive_cluster(map_to_rank(q_empty + 8 * slot, 0));
                }
                fence_proxy_async_global();  // what other tasks wrote is read by this CTA's copies
                ok = wait_local(r_empty + 8 * slot, turn ^ 1, a);
                if (!ok) break;
                {
                    uint4 *to = reinterpret_cast<uint4 *>(ring + slot);
#pragma unroll
                    for (int k = 0; k < 8; ++k) to[k] = words[k];
                    to[8] = make_uint4((unsigned)(int)tk.i, (unsigned)(int)tk.j, t < 0 ? 1u : 0u, (unsigned)tk.part);
                    to[9] = make_uint4((unsigned)(tk.part * p.steps), (unsigned)(tk.part == p.splits - 1 ? p.last_steps : p.steps), 0u, 0u);
                }
                arrive(r_full + 8 * slot);
                next_slot();
                if (t < 0) break;
                const int row = tk.i * TILE + (int)rank * ROWS;
                // the epilogue will read the tile of the fp32 copies
                for (int f = 0; f < (p.phase == MUON_GRAM ? 0 : p.phase == MUON_MUL ? 2 : 1); ++f)
#pragma unroll
                    for (int k = 0; k < ROWS / 32; ++k) {
                        const int b = p.blocks - tk.j * (TILE / 32);
                        const unsigned bytes = (unsigned)(b < TILE / 32 ? b : TILE / 32) * 4096u;
                        const float *at = (f ? p.src2 : p.src) + ((size_t)(row / 32 + k) * p.blocks + tk.j * (TILE / 32)) * 1024;
                        if (row + 32 * k < p.m) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(at), "r"(bytes) : "memory");
                    }
                // The next task is drawn when this one's loads are nearly through: earlier, it would only be kept from other workers.
                if (rank == 0) {
                    ok = wait_local(near_end, near_turn, a);
                    if (!ok) break;
                    near_turn ^= 1;
                    drawn = atomicAdd(a.next_task, 1u);
                }
            }
        }
    } else if (warp == 0 || warp == LOAD_RIGHT) {
        const bool left_side = warp == 0;
        const uint32_t full0 = map_to_rank(full, 0);
        const bool one = elect_one();
        int stage = 0;
        unsigned phase = 0, used = 0;
        for (;;) {
            ok = all_of(wait_local(r_full + 8 * slot, turn, a));
            if (!ok) break;
            const RingEntry &e = ring[slot];
            const int end = uniform(e.end), kind = uniform(e.p.phase), steps = uniform(e.steps), parts = PRECISE ? 2 : 1, ti = uniform(e.i), tj = uniform(e.j);
            const char *hi = a.maps + (size_t)uniform(left_side ? e.p.left : e.p.right) * MUON_MAP_BYTES;
            const char *lo = a.maps + (size_t)uniform(left_side ? e.p.left_lo : e.p.right_lo) * MUON_MAP_BYTES;
            const int k0 = uniform(e.k0);
            const int panel = (left_side ? ti : tj) * TILE, at = panel + (int)rank * ROWS;
            // from here on K's elements lie in the panel's rows
            const int rows_from = kind == MUON_GRAM ? 0 : left_side || kind <= MUON_MUL ? panel : 1 << 30;
            __syncwarp();
            if (one) arrive(r_empty + 8 * slot);
            next_slot();
            if (end) break;
            int left_steps = steps * parts;
            const int near_steps = min(left_steps, NEAR_STEPS);
            for (int k = 0; ok && k < steps; ++k)
                for (int part = 0; part < parts; ++part) {  // hi, lo
                    if (left_steps-- == near_steps && one && left_side) arrive(near_end);
                    ok = all_of(wait_local(empty + 8 * stage, phase ^ 1, a));
                    if (!ok) break;
                    if (one) {
                        if (rank == 0) mbar_expect_tx(full + 8 * stage, 2 * OPERAND);
                        load_operand<TILE>(base + stage * STAGE + (left_side ? 0 : OPERAND), part ? lo : hi, K * k < rows_from, at, K * (k0 + k), full0 + 8 * stage);
                    }
                    ++used;
                    if (++stage == STAGES) stage = 0, phase ^= 1;
                }
            if (!ok) break;
        }
        // before the CTA ends, every stage has been read (after a failure: waited for, as long as a wait lasts)
        for (int s = 0; s < STAGES && used; ++s) {
            if (used >= (unsigned)STAGES || s < stage) {
                const unsigned last = s < stage ? phase : phase ^ 1;
                if (!wait_local(empty + 8 * s, last, a)) ok = false;
            }
        }
    } else if (warp == MMA) {
        if (rank == 0) {
            const bool one = elect_one();
            int stage = 0, n_done = 0;
            unsigned phase = 0;
            for (;; ++n_done) {
                ok = all_of(wait_local(r_full + 8 * slot, turn, a));
                if (!ok) break;
                const RingEntry &e = ring[slot];
                const int end = uniform(e.end), kind = uniform(e.p.phase), steps = uniform(e.steps), parts = PRECISE ? 2 : 1, ti = uniform(e.i), tj = uniform(e.j);
                const int left_rows = kind == MUON_GRAM ? 0 : ti * TILE, right_rows = kind == MUON_GRAM ? 0 : kind <= MUON_MUL ? tj * TILE : 1 << 30;
                __syncwarp();
                if (one) arrive(r_empty + 8 * slot);
                next_slot();
                if (end) break;
                const int acc = n_done & 1;
                ok = all_of(wait_cluster(t_empty + 8 * acc, ((n_done >> 1) & 1) ^ 1, a));
                if (!ok) break;
                tc_after();
                const uint32_t d = tmem + acc * 256;
                // K-major: groups of 8 rows 1024 bytes apart, 16 elements of K 32 bytes further in the row, the next 64 of K 8192 bytes further.
                // MN-major: blocks of 64 columns 8192 bytes apart, groups of 8 rows of K 1024.
                auto multiply = [&](uint64_t da, uint64_t db, uint32_t idesc, bool a_mn, bool b_mn, uint32_t accumulate) {
#pragma unroll
                    for (int kk = 0; kk < K / 16; ++kk) {
                        const uint32_t rows = (32 * (kk & 3) + 8192 * (kk >> 2)) >> 4, columns = (2048 * kk) >> 4;
                        mma_f16(d, da + (a_mn ? columns : rows), db + (b_mn ? columns : rows), idesc, kk ? 1u : accumulate);
                    }
                };
                for (int k = 0; k < steps; ++k) {
                    const bool a_mn = K * k < left_rows, b_mn = K * k < right_rows;
                    const uint32_t idesc = (1u << 4) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(TILE >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
                    const uint64_t a_at = operand_desc(0, a_mn ? 8192 : 16, 1024), b_at = operand_desc(0, b_mn ? 8192 : 16, 1024);
                    const uint32_t at = (base + stage * STAGE) >> 4;  // (below 2^14)
                    const uint64_t da = a_at + at, db = b_at + at + (OPERAND >> 4);
                    ok = all_of(wait_local(full + 8 * stage, phase, a));
                    if (!ok) break;
                    tc_after();
                    const int hi = stage;
                    if (one) multiply(da, db, idesc, a_mn, b_mn, k ? 1u : 0u);
                    if (++stage == STAGES) stage = 0, phase ^= 1;
                    if (parts > 1) {  // the next stage holds the lo parts
                        ok = all_of(wait_local(full + 8 * stage, phase, a));
                        if (!ok) break;
                        tc_after();
                        const uint32_t at_lo = (base + stage * STAGE) >> 4;
                        if (one) {
                            multiply(da, b_at + at_lo + (OPERAND >> 4), idesc, a_mn, b_mn, 1u);
                            multiply(a_at + at_lo, db, idesc, a_mn, b_mn, 1u);
                            mma_commit(empty + 8 * hi);
                            mma_commit(empty + 8 * stage);
                        }
                        if (++stage == STAGES) stage = 0, phase ^= 1;
                    } else if (one) {
                        mma_commit(empty + 8 * hi);
                    }
                }
                if (!ok) break;
                if (one) mma_commit(t_full + 8 * acc);
            }
            if (!ok) {  // what was issued ends before the tensor memory is freed
                if (one)
                    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(drained) : "memory");
                mbar_wait_bounded(drained, 0);
            }
        }
    } else {
        // a warp reads the lanes 32 (warp % 4) .. + 31; those of a quarter share its columns
        constexpr int BLOCKS = TILE == 256 ? 4 : 2;
        const int q = warp & 3, share = (warp - FIRST_EPI) >> 2;
        const int warp_row = (int)rank * ROWS + 32 * (TILE == 256 ? q : q & 1), warp_column = share * (16 * BLOCKS) + (TILE == 256 ? 0 : 64 * (q >> 1));
        const uint32_t t_empty0 = map_to_rank(t_empty, 0);
        unsigned char *st = raw + (base - raw_s) + STAGES * STAGE + (warp - FIRST_EPI) * 4096;
        unsigned *told = nullptr;  // the counter that is still to be told of this warp's last task
        // The copies are written; with them and this warp's other stores the completion is told.  It waits for memory, so that it comes when
        // the next task's first loads are under way, unless there is no next task yet.
        auto tell = [&] {
            if (lane == 0 && told) {
                asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
                fence_proxy_async_global();
                asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(told), "r"(1u) : "memory");
            }
            told = nullptr;
            __syncwarp();
        };
        for (int n_done = 0;; ++n_done) {
            if (!__all_sync(0xffffffffu, mbar_test(r_full + 8 * slot, turn))) tell();
            ok = wait_local(r_full + 8 * slot, turn, a);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const MuonProduct &t = ring[slot].p;  // (the slot is free again when the task is done)
            const uint32_t slot_empty = r_empty + 8 * slot;
            const int ti = ring[slot].i, tj = ring[slot].j, part_no = ring[slot].part;
            if (ring[slot].end) break;
            next_slot();
            const int r0 = ti * TILE + warp_row, first = tj * TILE + warp_column;
            int blocks = r0 < t.m && first < t.width ? min((t.width - first + 15) / 16, BLOCKS) : 0;
            const int acc = n_done & 1;
            auto place = [&](int b) { return ((size_t)(r0 / 32) * t.blocks + (first + 16 * b) / 32) * 1024 + ((first + 16 * b) & 16) * 32 + lane * 4; };
            float4 x[4], next[4];
            float row = 0.f, next_column = 0.f;
            if (blocks > 0 && t.phase != MUON_GRAM) {
                if (t.phase <= MUON_MUL) next_column = __ldcg(t.vec2 + first + (lane & 15));
                load_block(t.src + place(0), next);
                row = __ldcg(t.vec + r0 + lane);
            }
            if (!PRECISE && t.phase == MUON_GRAM && ti == tj && r0 + lane < t.m) row = (float)__ldcg(t.rest + r0 + lane) * MUON_REST_INV;
            if (t.phase == MUON_FINAL && a.to == MUON_TO_PARAMS) {  // the parameters' rows on their way to L2
                const int rows = t.transposed ? t.width : t.m, cols = t.transposed ? t.m : t.width;
                for (int b = 0; b < 16 * blocks; b += 32) {
                    const int r = (t.transposed ? first + b : r0) + lane, c = t.transposed ? r0 : first + b;
                    if (r < rows) prefetch_l2(static_cast<const float *>(a.out[t.tensor]) + (size_t)r * cols + c);
                }
            }
            tell();
            ok = wait_local(t_full + 8 * acc, (n_done >> 1) & 1, a);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_after();
            // A part of a sum over K goes to memory; the warp whose part is the last to come adds all of them up, in their order, and goes on.
            // (Sums in pieces are also the more exact: tensor cores truncate, 2^-24 of the sum for every 16 elements in one direction, and the
            // diagonal of 1 x 2^20 came out 0.4 % small.)
            constexpr size_t part_stride = (size_t)TILE * TILE;
            const float *parts = nullptr;
            bool mine = true;  // the task's results are this warp's to write
            if (t.phase == MUON_GRAM && t.splits > 1) {
                const int tile = tj * (tj + 1) / 2 + ti, place = ((int)rank * EPI_WARPS + warp - FIRST_EPI);
                float *all = const_cast<float *>(t.src2) + (size_t)tile * t.splits * part_stride + (size_t)place * (BLOCKS * 512) + lane * 4;
                parts = all;
                for (int b = 0; b < blocks; ++b) {
                    float v[16];
                    tmem_ld16(tmem + acc * 256 + share * (16 * BLOCKS) + 16 * b + ((uint32_t)(q * 32) << 16), v);
                    store_block(all + (size_t)part_no * part_stride + b * 512, v);
                }
                __syncwarp();
                unsigned before = 0;
                if (lane == 0) {
                    unsigned *count = a.arrived + t.arrived + tile * (2 * EPI_WARPS) + place;
                    __threadfence();
                    before = atomicAdd(count, 1u);
                    __threadfence();
                    if (before == (unsigned)t.splits - 1u) atomicExch(count, 0u);  // for the next iteration
                }
                mine = __shfl_sync(0xffffffffu, before, 0) == (unsigned)t.splits - 1u;
                __syncwarp();  // (what the first lane's fence lets it see, the others see, too: a shuffle alone orders no memory)
                if (!mine) blocks = 0;
            }
            auto each_block = [&](auto use) {
#pragma unroll 1
                for (int b = 0; b < blocks; ++b) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[k] = next[k];
                    const float column = next_column;
                    if (t.phase != MUON_GRAM && b + 1 < blocks) {
                        load_block(t.src + place(b + 1), next);
                        if (t.phase <= MUON_MUL) next_column = __ldcg(t.vec2 + first + 16 * (b + 1) + (lane & 15));
                    }
                    use(BlockAt{place(b), tmem + acc * 256 + share * (16 * BLOCKS) + 16 * b + ((uint32_t)(q * 32) << 16), r0, first + 16 * b, b, lane, column, st});
                }
            };
            if (t.phase == MUON_GRAM)
                each_block([&](const BlockAt &b) {
                    float v[16];
                    if (t.splits == 1) {
                        tmem_ld16(b.tmem, v);
                    } else {
                        add_parts(parts + b.number * 512, t.splits, part_stride, v);
                    }
                    block_gram<TILE, PRECISE>(t, b, v, row);
                });
            else if (t.phase == MUON_POLY)
                each_block([&](const BlockAt &b) { block_poly<TILE, PRECISE>(a, t, b, x, row); });
            else if (t.phase == MUON_MUL)
                each_block([&](const BlockAt &b) { block_mul<TILE, PRECISE>(t, b, x, row); });
            else if (t.phase == MUON_UPDATE) {
                float rest = 0.f;
                each_block([&](const BlockAt &b) { block_update<TILE, PRECISE>(t, b, x, row, rest); });
                if (!PRECISE && blocks > 0 && r0 + lane < t.m) atomicAdd(t.rest + r0 + lane, rest_units(rest, t.scale));
            } else
                each_block([&](const BlockAt &b) { block_final(a, t, b, x, row, b.number + 1 < blocks); });
            if (blocks > 0 && t.phase != MUON_FINAL) {
                // (pad rows and columns: the copy leaves out what lies outside the matrix)
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    tma_store_2d(a.maps + (size_t)t.out * MUON_MAP_BYTES, first, r0, smem_u32(st));
                    if (PRECISE) tma_store_2d(a.maps + (size_t)t.out_lo * MUON_MAP_BYTES, first, r0, smem_u32(st + 2048));
                    tma_store_commit();
                }
            }
            tc_before();
            __syncwarp();
            if (lane == 0) arrive_cluster(t_empty0 + 8 * acc);
            if (t.phase != MUON_FINAL && mine) told = a.done + t.mat;
            __syncwarp();
            if (lane == 0) arrive(slot_empty);
        }
        tell();
    }
    if (!ok) {
        atomicExch(a.gave_up, 1u);
        atomicExch(a.status, DEMO_DEV_TIMEOUT);
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    cluster_sync();
    if (warp == 0) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    }
}

template <int TILE, bool PRECISE>
cudaError_t launch_products(const MuonArgs &a, const MuonProduct *products, const MuonTask *tasks, int n_tasks, int workers, DemoLaunch &dev, cudaStream_t stream)
{
    const void *kernel = reinterpret_cast<const void *>(muon_products_kernel<TILE, PRECISE>);
    cudaError_t err = demo_allow_smem(dev, kernel);
    if (err != cudaSuccess) return err;
    MuonArgs args = a;
    void *params[] = {&args, &products, &tasks, &n_tasks};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)workers * 2u);
    cfg.blockDim = dim3(Shape<TILE>::THREADS);
    cfg.dynamicSmemBytes = Shape<TILE>::SMEM;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelExC(&cfg, kernel, params);
}

}  // namespace

cudaError_t muon_launch_norm(const MuonArgs &a, int first_mat, int n_mats, int n_pieces, DemoLaunch &, cudaStream_t stream)
{
    MuonArgs args = a;
    void *params[] = {&args, &first_mat, &n_mats};
    return demo_launch_kernel(reinterpret_cast<const void *>(muon_norm_kernel), n_pieces, NORM_THREADS, 0, stream, params);
}

cudaError_t muon_launch_pack(const MuonArgs &a, const MuonTile *tiles, int n_tiles, int first_mat, int n_mats, int arrived, int n_arrived, DemoLaunch &dev,
                             cudaStream_t stream)
{
    MuonArgs args = a;
    int each = n_tiles >= 32 * dev.sm_count ? 4 : 1;
    void *params[] = {&args, &tiles, &n_tiles, &each, &first_mat, &n_mats, &arrived, &n_arrived};
    return demo_launch_kernel(reinterpret_cast<const void *>(muon_pack_kernel), (n_tiles + each - 1) / each, NORM_THREADS, 0, stream, params);
}

cudaError_t muon_launch_products(int tile, bool precise, const MuonArgs &a, const MuonProduct *products, const MuonTask *tasks, int n_tasks, int workers, DemoLaunch &dev, cudaStream_t stream)
{
    if (precise) return launch_products<128, true>(a, products, tasks, n_tasks, workers, dev, stream);
    return tile == 256 ? launch_products<256, false>(a, products, tasks, n_tasks, workers, dev, stream)
                       : launch_products<128, false>(a, products, tasks, n_tasks, workers, dev, stream);
}
