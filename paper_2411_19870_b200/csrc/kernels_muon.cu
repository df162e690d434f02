// Orthogonalised updates: Newton-Schulz iterations on whole weight matrices, on the tensor cores.
//
//   X_0 = u / (||u||_F + eps);  A = X X^T;  X <- a X + (b A + c A^2) X
//
// as three products an iteration, each over all matrices of a group:
//   GRAM    A = X X^T        symmetric: the tiles on and above the diagonal, mirrored
//   POLY    A^2 -> F, beta   symmetric, too
//   UPDATE  F X  -> X
// Operands are fp16 (11 bits, accumulated in fp32), and what would lose accuracy in them is kept out of them:
//   * the linear term a X, on which small singular values live alone (they grow by a = 3.4 an iteration, rounding noise with them),
//     is formed from X = hi + lo, 22 bits;
//   * the diagonal of A, of order one in the last iterations, where a X and (b A + c A^2) X nearly cancel, never passes through fp16:
//     A = D + E, A^2 = D^2 + D E + E D + E^2, so F = offdiag((b + c (d_i + d_j)) E + c E^2) and X <- (a + beta_i) X + F X with
//     beta_i = b d_i + c (d_i^2 + (E^2)_ii) in fp32.
// Relative error of the result against 64 bits, Gaussian 1024 x 1024: 6e-4 (plain fp16 operands 1.6e-3, bf16 1.2e-2); of rank one:
// 5e-4 (0.15 and 1.2).  It grows as matrices shrink, so those of up to 256 rows take the lo parts of the products' operands, too.
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
    const long long n = (long long)mat.m * mat.n, at = (long long)(blockIdx.x - mat.piece_begin) * MUON_PIECE;
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
    const int len = (int)(n - at < MUON_PIECE ? n - at : MUON_PIECE);
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
    if (threadIdx.x == 0) a.partials[blockIdx.x] = s;
}

__device__ __forceinline__ void split(float v, __half &hi, __half &lo)
{
    hi = __float2half_rn(v);
    lo = __float2half_rn(v - __half2float(hi));
}

// A tile of 64 x 64 elements of X.  The pieces' sums are added in one order by every CTA.
__global__ void __launch_bounds__(NORM_THREADS) muon_pack_kernel(MuonArgs a, const MuonTile *tiles)
{
    const StreamOrder order(1);
    constexpr int T = MUON_PACK_TILE;
    __shared__ double scratch[NORM_THREADS / 32];
    __shared__ float tile[T][T + 1];
    const MuonTile t = tiles[blockIdx.x];
    const MuonMat &mat = a.mats[t.mat];
    order.begin();
    double sum = 0;
    for (int p = threadIdx.x; p < mat.n_pieces; p += NORM_THREADS) sum += a.partials[mat.piece_begin + p];
    const double norm = sqrt(block_sum(sum, scratch));
    const double all = norm + (double)a.eps, scale_d = all > 0 ? (double)mat.S / all : 1;
    // in two factors, so that neither leaves the range of fp32 where the norm is near its ends
    const float scale1 = (float)exp2(floor(0.5 * log2(scale_d))), scale2 = (float)(scale_d / (double)scale1);
    const void *in = a.in[mat.tensor];
    const float *mom = a.from == MUON_FROM_STEP ? a.mom[mat.tensor] : nullptr;
    const int rows = mat.transposed ? mat.n : mat.m, cols = mat.transposed ? mat.m : mat.n;
    // tile row i0, column j0 of X; of the tensor, the other way round where X is its transpose
    const int i0 = t.i * T, j0 = t.j * T;
    const int r0 = mat.transposed ? j0 : i0, c0 = mat.transposed ? i0 : j0;
    const int x = threadIdx.x & (T - 1);
#pragma unroll 4
    for (int y = threadIdx.x / T; y < T; y += NORM_THREADS / T) {
        const int r = r0 + y, c = c0 + x;
        float u = 0.f;
        if (r < rows && c < cols) {
            const long long at = (long long)r * cols + c;
            u = load_in(in, at, a.in_bf16);
            if (mom) {
                const float m = mom[at];
                u = a.nesterov ? fmaf(a.mu, m, u) : m;
            }
        }
        tile[y][x] = u * scale1 * scale2;
    }
    __syncthreads();
#pragma unroll 4
    for (int y = threadIdx.x / T; y < T; y += NORM_THREADS / T) {
        const int i = i0 + y, j = j0 + x;
        if (i < mat.m && j < mat.ldx) {
            __half hi, lo;
            split(mat.transposed ? tile[x][y] : tile[y][x], hi, lo);
            const size_t at = (size_t)i * mat.ldx + j;
            reinterpret_cast<__half *>(mat.xhi[0])[at] = hi;
            reinterpret_cast<__half *>(mat.xlo[0])[at] = lo;
        }
    }
}

// ---- products -----------------------------------------------------------------------------------------------------------------

constexpr int EPI_WARPS = 8;
constexpr int THREADS = 64 + 32 * EPI_WARPS;  // producer warp, MMA warp, epilogue
constexpr int OPERAND = 16384;                // 128 rows (K-major) or 64 x 128 (MN-major) fp16 elements of one step of K = 64
constexpr int STAGE = 2 * OPERAND;
constexpr int STAGES = 6;
constexpr int TMEM_COLS = 512;
constexpr int SMEM = STAGES * STAGE + 1024;

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

template <int CG>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(idesc), "r"(accumulate)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(idesc), "r"(accumulate)
                     : "memory");
}
// Arrives at `bar` (of both CTAs of a pair) once the MMAs issued so far are done.
template <int CG>
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// A box of 64 x 64 elements; a pair's loads are counted by the barrier of its first CTA.
template <int CG>
__device__ __forceinline__ void load_box(uint32_t dst, const void *map, int x, int y, uint32_t bar)
{
    if constexpr (CG == 1)
        tma_load_2d(dst, map, x, y, bar);
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
                     "r"(x), "r"(y), "r"(bar)
                     : "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t bar, bool remote)
{
    if (remote)
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// as mbar_wait_bounded, seeing what another CTA of the cluster did before its arrival
__device__ __forceinline__ bool wait_cluster(uint32_t bar, unsigned parity)
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
        if (clock64() - t0 > WAIT_LIMIT_CYCLES) return false;
    }
}

__device__ __forceinline__ float2 unpack2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }
__device__ __forceinline__ uint32_t pack2(float x, float y)
{
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// 32 consecutive fp16 values of a row (its start a multiple of 64 bytes) to and from fp32.
__device__ __forceinline__ void load_row32(const uint16_t *p, float (&v)[32])
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint4 w = reinterpret_cast<const uint4 *>(p)[q];
        const float2 a = unpack2(w.x), b = unpack2(w.y), c = unpack2(w.z), d = unpack2(w.w);
        v[8 * q] = a.x, v[8 * q + 1] = a.y, v[8 * q + 2] = b.x, v[8 * q + 3] = b.y;
        v[8 * q + 4] = c.x, v[8 * q + 5] = c.y, v[8 * q + 6] = d.x, v[8 * q + 7] = d.y;
    }
}
__device__ __forceinline__ void store_row32(uint16_t *p, const float (&v)[32])
{
#pragma unroll
    for (int q = 0; q < 4; ++q)
        reinterpret_cast<uint4 *>(p)[q] = make_uint4(pack2(v[8 * q], v[8 * q + 1]), pack2(v[8 * q + 2], v[8 * q + 3]), pack2(v[8 * q + 4], v[8 * q + 5]),
                                                     pack2(v[8 * q + 6], v[8 * q + 7]));
}
__device__ __forceinline__ void keep_rest(float (&v)[32])  // v - fp16(v)
{
#pragma unroll
    for (int k = 0; k < 32; ++k) v[k] -= __half2float(__float2half_rn(v[k]));
}

// A row piece (row i, columns j0 .. j0 + 31) of a symmetric result, into its place and, off the diagonal tiles, mirrored: there a warp's
// 32 rows are 32 neighbouring columns.
__device__ __forceinline__ void store_symmetric(const MuonMat &mat, uint16_t *hi, uint16_t *lo, float (&v)[32], int i, int j0, bool mirror)
{
    const size_t at = (size_t)i * mat.lde + j0;
    if (mirror) {
#pragma unroll
        for (int k = 0; k < 32; ++k)
            if (j0 + k < mat.m) {
                __half h, l;
                split(v[k], h, l);
                const size_t to = (size_t)(j0 + k) * mat.lde + i;
                reinterpret_cast<__half *>(hi)[to] = h;
                if (mat.precise) reinterpret_cast<__half *>(lo)[to] = l;
            }
    }
    store_row32(hi + at, v);
    if (mat.precise) {
        keep_rest(v);
        store_row32(lo + at, v);
    }
}

template <int PHASE>
__device__ __forceinline__ void epilogue(const MuonArgs &a, const MuonMat &mat, float (&v)[32], int i, int j0, bool mirror, int parity)
{
    if (i >= mat.m) return;
    if constexpr (PHASE == MUON_GRAM) {
        if (j0 >= mat.m) return;
        const float s = mat.inv_S * mat.inv_S * MUON_EF_SCALE;
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            v[k] *= s;
            if (j0 + k == i) {
                mat.d[i] = v[k] * MUON_EF_INV;
                v[k] = 0.f;
            }
        }
        store_symmetric(mat, mat.ehi, mat.elo, v, i, j0, mirror);
    } else if constexpr (PHASE == MUON_POLY) {
        if (j0 >= mat.m) return;
        const size_t at = (size_t)i * mat.lde + j0;
        float e[32];
        load_row32(mat.ehi + at, e);
        if (mat.precise) {
            float l[32];
            load_row32(mat.elo + at, l);
#pragma unroll
            for (int k = 0; k < 32; ++k) e[k] += l[k];
        }
        const float di = mat.d[i], base = fmaf(a.c, di, a.b);
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            const float dj = j0 + k < mat.m ? mat.d[j0 + k] : 0.f;
            const float f = fmaf(fmaf(a.c, dj, base), e[k], a.c * MUON_EF_INV * v[k]);
            if (j0 + k == i) mat.beta[i] = fmaf(a.b, di, a.c * fmaf(di, di, v[k] * (MUON_EF_INV * MUON_EF_INV)));
            v[k] = j0 + k == i ? 0.f : f;
        }
        store_symmetric(mat, mat.fhi, mat.flo, v, i, j0, mirror);
    } else {
        if (j0 >= mat.n) return;
        const size_t at = (size_t)i * mat.ldx + j0;
        const float lin = a.a + mat.beta[i];
        {
            float x[32];
            load_row32(mat.xlo[parity] + at, x);
            float h[32];
            load_row32(mat.xhi[parity] + at, h);
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] = fmaf(lin, h[k] + x[k], v[k] * MUON_EF_INV);
        }
        if constexpr (PHASE == MUON_UPDATE) {
            store_row32(mat.xhi[parity ^ 1] + at, v);
            keep_rest(v);
            store_row32(mat.xlo[parity ^ 1] + at, v);
        } else {
            const bool params = a.to == MUON_TO_PARAMS;
            const float keep = 1.f - a.lr * a.wd, scale = params ? -a.lr * mat.step_scale * mat.inv_S : mat.inv_S;
            const int cols = mat.transposed ? mat.m : mat.n;
            const size_t to = mat.transposed ? (size_t)j0 * cols + i : (size_t)i * cols + j0;
            const int step = mat.transposed ? cols : 1;
            void *out = a.out[mat.tensor];
            const bool whole = !mat.transposed && cols % 8 == 0 && j0 + 32 <= cols;
            if (params) {
                float *x = static_cast<float *>(out) + to;
                if (whole) {
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        float4 w = reinterpret_cast<float4 *>(x)[q];
                        w.x = fmaf(w.x, keep, v[4 * q] * scale);
                        w.y = fmaf(w.y, keep, v[4 * q + 1] * scale);
                        w.z = fmaf(w.z, keep, v[4 * q + 2] * scale);
                        w.w = fmaf(w.w, keep, v[4 * q + 3] * scale);
                        reinterpret_cast<float4 *>(x)[q] = w;
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (j0 + k < mat.n) x[(size_t)k * step] = fmaf(x[(size_t)k * step], keep, v[k] * scale);
                }
            } else if (a.out_bf16) {
                __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(out) + to;
                if (whole) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t w[4];
#pragma unroll
                        for (int p = 0; p < 4; ++p) {
                            const __nv_bfloat162 b = __floats2bfloat162_rn(v[8 * q + 2 * p] * scale, v[8 * q + 2 * p + 1] * scale);
                            w[p] = *reinterpret_cast<const uint32_t *>(&b);
                        }
                        reinterpret_cast<uint4 *>(o)[q] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (j0 + k < mat.n) o[(size_t)k * step] = __float2bfloat16_rn(v[k] * scale);
                }
            } else {
                float *o = static_cast<float *>(out) + to;
#pragma unroll
                for (int k = 0; k < 32; ++k)
                    if (j0 + k < mat.n) o[(size_t)k * step] = v[k] * scale;
            }
        }
    }
}

// Persistent CTAs (CG = 2: pairs) over the tiles.  One warp loads, one issues the MMAs, eight read accumulators back: two of them, so that
// the products of a tile run beside the epilogue of the one before.
template <int PHASE, int CG>
__global__ void __launch_bounds__(THREADS, 1) muon_product_kernel(MuonArgs a, const MuonTile *tiles, int n_tiles, int parity)
{
    const StreamOrder order(1);
    constexpr int TILE = 128 * CG;  // of both sides
    constexpr bool B_MN = PHASE >= MUON_UPDATE;  // X as K x N: its rows run along K
    constexpr uint32_t IDESC = (1u << 4) | ((uint32_t)B_MN << 16) | ((uint32_t)(TILE >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
    extern __shared__ unsigned char raw[];
    __shared__ unsigned long long bars[2 * STAGES + 4 + 1];
    __shared__ uint32_t tmem_slot;
    const uint32_t raw_s = smem_u32(raw), base = (raw_s + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0u;
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, t_full = empty + 8 * STAGES, t_empty = t_full + 16, drained = t_empty + 16;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(t_full + 8 * s, 1);
            mbar_init(t_empty + 8 * s, CG * EPI_WARPS);
        }
        mbar_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    order.begin();
    if (warp == 0) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    tc_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    tc_after();
    const uint32_t tmem = tmem_slot;
    const int stride = gridDim.x / CG, start = blockIdx.x / CG;
    bool ok = true;

    if (warp == 0) {
        if (lane == 0) {
            const uint32_t full0 = CG == 2 ? map_to_rank(full, 0) : full;
            int stage = 0, last_mat = -1;
            unsigned phase = 0, used = 0;
            for (int t = start; ok && t < n_tiles; t += stride) {
                const MuonTile tl = tiles[t];
                const MuonMat &mat = a.mats[tl.mat];
                const char *maps = a.maps + (size_t)mat.maps * MUON_MAP_BYTES;
                // left operand (and its lo part), right operand
                const int left = PHASE == MUON_GRAM ? MUON_MAP_X0 + parity : PHASE == MUON_POLY ? MUON_MAP_E : MUON_MAP_F;
                const int right = PHASE == MUON_POLY ? MUON_MAP_E : MUON_MAP_X0 + parity;
                const int left_lo = PHASE == MUON_GRAM ? MUON_MAP_XLO0 + parity : left + 1;
                const int right_lo = PHASE == MUON_POLY ? MUON_MAP_ELO : MUON_MAP_XLO0 + parity;
                if (tl.mat != last_mat) {
                    tmap_acquire(maps + left * MUON_MAP_BYTES);
                    tmap_acquire(maps + right * MUON_MAP_BYTES);
                    if (mat.precise) {
                        tmap_acquire(maps + left_lo * MUON_MAP_BYTES);
                        tmap_acquire(maps + right_lo * MUON_MAP_BYTES);
                    }
                    last_mat = tl.mat;
                }
                const int K = PHASE == MUON_GRAM ? mat.n : mat.m, steps = (K + 63) / 64, parts = mat.precise ? 3 : 1;
                const int row = tl.i * TILE + (int)rank * 128, col = tl.j * TILE + (int)rank * 128;
                for (int part = 0; ok && part < parts; ++part) {  // hi hi, hi lo, lo hi
                    const char *ml = maps + (part == 2 ? left_lo : left) * MUON_MAP_BYTES, *mr = maps + (part == 1 ? right_lo : right) * MUON_MAP_BYTES;
                    for (int k = 0; k < steps; ++k) {
                        ok = CG == 2 ? wait_cluster(empty + 8 * stage, phase ^ 1) : mbar_wait_bounded(empty + 8 * stage, phase ^ 1);
                        if (!ok) break;
                        const uint32_t bar = full0 + 8 * stage, A = base + stage * STAGE, B = A + OPERAND;
                        if (rank == 0) mbar_expect_tx(full + 8 * stage, CG * STAGE);
                        load_box<CG>(A, ml, 64 * k, row, bar);
                        load_box<CG>(A + OPERAND / 2, ml, 64 * k, row + 64, bar);
                        if (B_MN) {
                            load_box<CG>(B, mr, col, 64 * k, bar);
                            load_box<CG>(B + OPERAND / 2, mr, col + 64, 64 * k, bar);
                        } else {
                            load_box<CG>(B, mr, 64 * k, col, bar);
                            load_box<CG>(B + OPERAND / 2, mr, 64 * k, col + 64, bar);
                        }
                        ++used;
                        if (++stage == STAGES) stage = 0, phase ^= 1;
                    }
                }
            }
            // before the CTA ends, every stage has been read (after a failure: waited for, as long as a wait lasts)
            for (int s = 0; s < STAGES && used; ++s) {
                if (used >= (unsigned)STAGES || s < stage) {
                    const unsigned last = s < stage ? phase : phase ^ 1;
                    if (!(CG == 2 ? wait_cluster(empty + 8 * s, last) : mbar_wait_bounded(empty + 8 * s, last))) ok = false;
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            int stage = 0, n_done = 0;
            unsigned phase = 0;
            for (int t = start; ok && t < n_tiles; t += stride, ++n_done) {
                const MuonMat &mat = a.mats[tiles[t].mat];
                const int K = PHASE == MUON_GRAM ? mat.n : mat.m, steps = (K + 63) / 64 * (mat.precise ? 3 : 1);
                const int acc = n_done & 1;
                ok = CG == 2 ? wait_cluster(t_empty + 8 * acc, ((n_done >> 1) & 1) ^ 1) : mbar_wait_bounded(t_empty + 8 * acc, ((n_done >> 1) & 1) ^ 1);
                if (!ok) break;
                tc_after();
                const uint32_t d = tmem + acc * 256;
                for (int k = 0; k < steps; ++k) {
                    ok = CG == 2 ? wait_cluster(full + 8 * stage, phase) : mbar_wait_bounded(full + 8 * stage, phase);
                    if (!ok) break;
                    tc_after();
                    const uint32_t A = base + stage * STAGE;
                    // K-major: groups of 8 rows 1024 bytes apart, 16 elements of K 32 bytes further in the row.  MN-major: blocks of 64 columns
                    // 8192 bytes apart, groups of 8 rows of K 1024.
                    uint64_t da = operand_desc(A, 16, 1024), db = operand_desc(A + OPERAND, B_MN ? 8192 : 16, 1024);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) {
                        mma_f16<CG>(d, da, db, IDESC, (k | kk) != 0);
                        da += 32 >> 4;
                        db += (B_MN ? 2048 : 32) >> 4;
                    }
                    mma_commit<CG>(empty + 8 * stage);
                    if (++stage == STAGES) stage = 0, phase ^= 1;
                }
                mma_commit<CG>(t_full + 8 * acc);
            }
            if (!ok) {  // what was issued ends before the tensor memory is freed
                if constexpr (CG == 1)
                    mma_commit<1>(drained);
                else
                    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(drained) : "memory");
                mbar_wait_bounded(drained, 0);
            }
        }
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;  // a warp reads the lanes 32 (warp % 4) .. + 31; the two of a quarter share its columns
        const uint32_t t_empty0 = CG == 2 ? map_to_rank(t_empty, 0) : t_empty;
        int n_done = 0;
        for (int t = start; t < n_tiles; t += stride, ++n_done) {
            const MuonTile tl = tiles[t];
            const MuonMat &mat = a.mats[tl.mat];
            const int acc = n_done & 1;
            ok = CG == 2 ? wait_cluster(t_full + 8 * acc, (n_done >> 1) & 1) : mbar_wait_bounded(t_full + 8 * acc, (n_done >> 1) & 1);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_after();
            const int i = tl.i * TILE + (int)rank * 128 + q * 32 + lane;
            const bool mirror = PHASE <= MUON_POLY && tl.i != tl.j;
#pragma unroll 1
            for (int c = half * (TILE / 2); c < (half + 1) * (TILE / 2); c += 32) {
                float v[32];
                tmem_ld32(tmem + acc * 256 + c + ((uint32_t)(q * 32) << 16), v);
                epilogue<PHASE>(a, mat, v, i, tl.j * TILE + c, mirror, parity);
                __syncwarp();
            }
            tc_before();
            __syncwarp();
            if (lane == 0) arrive_at(t_empty0 + 8 * acc, CG == 2);
        }
    }
    if (!ok) atomicExch(a.status, DEMO_DEV_TIMEOUT);
    __syncwarp();
    // the next launch's copies read through the asynchronous proxy what these warps stored
    asm volatile("fence.proxy.async;" ::: "memory");
    tc_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    if (warp == 0) {
        tc_after();
        if constexpr (CG == 1)
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    }
}

template <int PHASE, int CG>
cudaError_t launch_product(const MuonArgs &a, const MuonTile *tiles, int n_tiles, int parity, DemoLaunch &dev, cudaStream_t stream)
{
    const void *kernel = reinterpret_cast<const void *>(muon_product_kernel<PHASE, CG>);
    cudaError_t err = demo_allow_smem(dev, kernel);
    if (err != cudaSuccess) return err;
    const int most = dev.sm_count / CG;
    const int grid = (n_tiles < most ? n_tiles : most) * CG;
    MuonArgs args = a;
    void *params[] = {&args, &tiles, &n_tiles, &parity};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CG;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = CG == 2 ? 2 : 1;
    return cudaLaunchKernelExC(&cfg, kernel, params);
}

template <int CG>
cudaError_t launch_phase(int phase, const MuonArgs &a, const MuonTile *tiles, int n_tiles, int parity, DemoLaunch &dev, cudaStream_t stream)
{
    switch (phase) {
        case MUON_GRAM: return launch_product<MUON_GRAM, CG>(a, tiles, n_tiles, parity, dev, stream);
        case MUON_POLY: return launch_product<MUON_POLY, CG>(a, tiles, n_tiles, parity, dev, stream);
        case MUON_UPDATE: return launch_product<MUON_UPDATE, CG>(a, tiles, n_tiles, parity, dev, stream);
        default: return launch_product<MUON_FINAL, CG>(a, tiles, n_tiles, parity, dev, stream);
    }
}

}  // namespace

cudaError_t muon_launch_norm(const MuonArgs &a, int first_mat, int n_mats, int n_pieces, DemoLaunch &, cudaStream_t stream)
{
    MuonArgs args = a;
    void *params[] = {&args, &first_mat, &n_mats};
    return demo_launch_kernel(reinterpret_cast<const void *>(muon_norm_kernel), n_pieces, NORM_THREADS, 0, stream, params);
}

cudaError_t muon_launch_pack(const MuonArgs &a, const MuonTile *tiles, int n_tiles, DemoLaunch &, cudaStream_t stream)
{
    MuonArgs args = a;
    void *params[] = {&args, &tiles};
    return demo_launch_kernel(reinterpret_cast<const void *>(muon_pack_kernel), n_tiles, NORM_THREADS, 0, stream, params);
}

cudaError_t muon_launch_product(int phase, bool pair, int parity, const MuonArgs &a, const MuonTile *tiles, int n_tiles, DemoLaunch &dev, cudaStream_t stream)
{
    return pair ? launch_phase<2>(phase, a, tiles, n_tiles, parity, dev, stream) : launch_phase<1>(phase, a, tiles, n_tiles, parity, dev, stream);
}
