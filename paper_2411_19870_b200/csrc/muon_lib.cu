// Host side of the orthogonalised updates in include/demo.h: plan (groups of matrices, tiles), workspace and tensor maps, launches.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <new>
#include <vector>

#include "../../include/demo.h"
#include "demo_internal.h"
#include "host_common.h"
#include "launch.cuh"
#include "muon.h"

namespace {

// Matrices that are in the workspace together: a launch for their norms, one to lay them out and one for all their products.
struct Group {
    int first_mat, n_mats, n_pieces, piece;
    int tile;              // side of the tiles
    bool precise;
    long long pack_tiles;  // first of its list
    int n_pack;
    long long tasks;
    int n_tasks, workers;
    int at_once;             // tasks that can be in work at the same time
    int waiting, n_waiting;  // those of its first matrix's second product, for the self-test
    int arrived, n_arrived;  // counters of the parts of its sums
};

enum { FROM_ORTHOGONALIZE = 0, FROM_STEP = 1, FROM_DECODE = 2, ENTRY_POINTS = 3 };

constexpr long long GROUP_ELEMENTS = 128LL << 20;  // workspace: 8 bytes for each, and up to 18 bytes for each of the square matrices beside X
constexpr size_t GROUP_BYTES = 26 * (size_t)GROUP_ELEMENTS;  // of their workspace: thin matrices take more than 26 bytes an element, up to 145 where there is one row
// Up to here the products take the lo parts, too (kernels_muon.cu): what 11 bits lose grows as matrices shrink, and small products are quick.
// (At 384 rows an error of 1.4e-3 where the rank is 128 becomes 1e-5, for 111 us instead of 93 of 384 x 768, 134 instead of 111 of fourteen of 384 x 384, 1324
// instead of 838 of sixty of 384 x 1536.  At 512 rows 1.3e-3 is left, and one matrix would take 113 us instead of 93, 24 of 512 x 512 351 instead of 260,
// 24 of 512 x 2048 1013 instead of 541.)
constexpr int PRECISE_SIDE = 384;
constexpr long long WAIT_CYCLES = 20000000000LL;  // ~10 s: what is waited for may be other workers' tasks, long ones for large matrices

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }

}  // namespace

struct demo_muon_ctx {
    demo_muon_config cfg;
    int device = 0, n_tensors = 0;
    DemoLaunch launch;
    std::vector<demo_tensor_desc> descs;
    std::vector<Group> groups;
    long long launches = 0;
    size_t bytes = 0;
    MuonMat *d_mats = nullptr;
    MuonTile *d_tiles = nullptr;
    MuonProduct *d_products = nullptr;
    MuonTask *d_tasks = nullptr;
    unsigned *d_done = nullptr;  // [n_tensors] completions; [n_tensors] pieces ready; the next task of each kind; whether it has given up
    float2 *d_scales = nullptr;
    unsigned *d_arrived = nullptr;
    char *d_maps = nullptr;
    char *d_work = nullptr;
    double *d_partials = nullptr;
    int side_partials = 0;  // where those of the precise matrices begin
    int side_workers = 0;   // workers of the precise matrices where there are others, too
    int *d_status = nullptr;
    // Where there are matrices of both kinds, the precise ones go through the iterations beside the others, on a stream of the context's own,
    // which the caller's stream waits for (five matrices of 512 rows and one of 147: 350 us, the five alone 341, the one 106).
    cudaStream_t side_stream = nullptr;
    cudaEvent_t fork = nullptr, join = nullptr;
    PointerTable tables[ENTRY_POINTS];  // inputs, outputs, and momenta where they are the caller's
    float *d_momentum = nullptr;  // reconstructed momenta of demo_muon_decode_apply, from its first call
    size_t momentum_bytes = 0;
    std::vector<float *> momentum_ptrs;
};

namespace {

void release(demo_muon_ctx *c)
{
    if (!c) return;
    cudaFree(c->d_mats);
    cudaFree(c->d_tiles);
    cudaFree(c->d_products);
    cudaFree(c->d_tasks);
    cudaFree(c->d_done);
    cudaFree(c->d_scales);
    cudaFree(c->d_arrived);
    cudaFree(c->d_maps);
    cudaFree(c->d_work);
    cudaFree(c->d_partials);
    cudaFree(c->d_status);
    cudaFree(c->d_momentum);
    if (c->fork) cudaEventDestroy(c->fork);
    if (c->join) cudaEventDestroy(c->join);
    if (c->side_stream) cudaStreamDestroy(c->side_stream);
    for (PointerTable &t : c->tables) t.release();
    delete c;
}

struct Plan {
    std::vector<MuonMat> mats;
    std::vector<MuonTile> tiles;
    std::vector<MuonProduct> products;
    std::vector<MuonTask> tasks;
    size_t work[2] = {0, 0};  // of the groups of each kind, the precise ones last
    int pieces[2] = {0, 0};
    size_t arrived = 0;
};

int ceil_div(int v, int by) { return (v + by - 1) / by; }

// Tiles of a symmetric product.
int tiles_above(const MuonMat &m)
{
    const int k = ceil_div(m.m, m.tile);
    return k * (k + 1) / 2;
}

// Workspace of one matrix from `at` on, as offsets (the base is added once it is known).  Returns its end.
size_t place(MuonMat &m, size_t at)
{
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (size_t)round_up((long long)bytes, 256);
        return reinterpret_cast<uint16_t *>(here);
    };
    const size_t x = (size_t)m.m * (size_t)m.ldx * 2, e = (size_t)m.m * (size_t)m.lde * 2, rows = (size_t)round_up(m.m, 32);
    for (int p = 0; p < 2; ++p) {
        m.xhi[p] = take(x);
        m.xlo[p] = m.precise ? take(x) : m.xhi[p];
    }
    m.x32 = reinterpret_cast<float *>(take(rows * (size_t)m.ldx * 4));
    m.parts = reinterpret_cast<float *>(m.splits > 1 ? reinterpret_cast<size_t>(take((size_t)m.splits * (size_t)tiles_above(m) * (size_t)(m.tile * m.tile) * 4)) : 0);
    for (int p = 0; p < 2; ++p) m.rest[p] = m.precise ? nullptr : reinterpret_cast<int *>(take((size_t)m.m * 4));
    for (int k = 0; k < m.symmetric; ++k) {
        m.ehi[k] = take(e);
        m.elo[k] = m.precise ? take(e) : m.ehi[k];
        m.e32[k] = m.symmetric == 2 && k == 1 ? nullptr : reinterpret_cast<float *>(take(rows * (size_t)m.lde * 4));  // (B of one iteration: not needed)
        m.diag[k] = reinterpret_cast<float *>(take((size_t)m.lde * 4));
    }
    return at;
}
void rebase(MuonMat &m, char *base)
{
    auto move = [&](auto *&p) { p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + reinterpret_cast<size_t>(p)); };
    for (int p = 0; p < 2; ++p) {
        move(m.xhi[p]);
        move(m.xlo[p]);
        if (!m.precise) move(m.rest[p]);
    }
    move(m.x32);
    move(m.parts);
    for (int k = 0; k < m.symmetric; ++k) {
        move(m.ehi[k]);
        move(m.elo[k]);
        if (m.symmetric > 2 || k == 0) move(m.e32[k]);
        move(m.diag[k]);
    }
}

// Tiles (i, j) of a grid in bands of eight rows, so that those in work together share rows and columns.
template <class Use>
void each_tile(int rows, int cols, bool upper, Use use)
{
    for (int band = 0; band < rows; band += 8)
        for (int j = upper ? band : 0; j < cols; ++j)
            for (int i = band; i < std::min(rows, band + 8); ++i)
                if (!upper || i <= j) use(i, j);
}

// The products that one matrix goes through, in order.
std::vector<MuonProduct> products_of(const MuonMat &m, int steps)
{
    std::vector<MuonProduct> list;
    int now = 0;  // the X that is read
    auto add = [&](int phase) -> MuonProduct & {
        MuonProduct t;
        std::memset(&t, 0, sizeof(t));
        const bool wide = phase >= MUON_UPDATE;
        t.phase = phase;
        t.steps = t.last_steps = ceil_div(phase == MUON_GRAM ? m.n : m.m, muon_k_step(m.tile));
        t.splits = 1;
        if (phase == MUON_GRAM && m.splits > 1) {
            t.last_steps = t.steps - (m.splits - 1) * m.split_steps;
            t.steps = m.split_steps;
            t.splits = m.splits;
            t.arrived = m.arrived;
            t.src2 = m.parts;
        }
        t.m = m.m;
        t.width = wide ? m.n : m.m;
        t.blocks = (wide ? m.ldx : m.lde) / 32;
        t.tensor = m.tensor;
        t.transposed = m.transposed;
        t.scale = phase == MUON_GRAM ? m.inv_S * m.inv_S * MUON_EF_SCALE : m.inv_S;
        t.step_scale = m.step_scale * m.inv_S;
        list.push_back(t);
        return list.back();
    };
    auto x_maps = [&](int &hi, int &lo, int which) { hi = m.maps + MUON_MAP_X + which, lo = m.maps + MUON_MAP_XLO + which; };
    auto e_maps = [&](int &hi, int &lo, int which) { hi = m.maps + MUON_MAP_E + which, lo = m.maps + MUON_MAP_ELO + which; };
    auto result = [&](MuonProduct &t, int to, bool fp32) {
        e_maps(t.out, t.out_lo, to);
        t.dst = fp32 ? m.e32[to] : nullptr;
        t.diag = m.diag[to];
    };
    auto gram = [&](int to) {
        MuonProduct &t = add(MUON_GRAM);
        x_maps(t.left, t.left_lo, now);
        x_maps(t.right, t.right_lo, now);
        t.rest = m.rest[now];
        result(t, to, true);
    };
    auto multiply = [&](int phase, int p, int q, int to, bool fp32) {
        MuonProduct &t = add(phase);
        e_maps(t.left, t.left_lo, p);
        e_maps(t.right, t.right_lo, q);
        t.src = m.e32[p];
        t.src2 = m.e32[q];
        t.vec = m.diag[p];
        t.vec2 = m.diag[q];
        result(t, to, fp32);
    };
    auto update = [&](int by, bool last) {
        MuonProduct &t = add(last ? MUON_FINAL : MUON_UPDATE);
        e_maps(t.left, t.left_lo, by);
        x_maps(t.right, t.right_lo, now);
        t.src = t.dst = m.x32;
        t.vec = m.diag[by];
        now ^= 1;
        t.rest = last ? nullptr : m.rest[now];
        x_maps(t.out, t.out_lo, now);
    };
    for (int k = 0; k < steps;) {
        // The first two only: what the products of two iterations round adds noise where the rank is low, and from the first ones the later
        // iterations take it away again.  (1024 x 2048 of rank 1, 5, 32, 128: [2, 1, 1, 1] 9e-4, 4e-4, 6e-4, 9e-4, which is what one after the other gives;
        // [1, 2, 2], which would multiply 16 % less at n = 4 m, 6e-4, 3e-3, 2e-3, 4e-3.)
        const bool two = m.twos && k == 0;
        gram(0);
        multiply(MUON_POLY, 0, 0, 1, two);
        if (two) {
            multiply(MUON_MUL, 0, 1, 2, true);   // T = A B
            multiply(MUON_MUL, 2, 1, 0, true);   // A' = T B
            multiply(MUON_POLY, 0, 0, 2, true);  // B'
            multiply(MUON_MUL, 2, 1, 0, false);  // Q = B' B
        }
        k += two ? 2 : 1;
        update(two ? 0 : 1, k == steps);
    }
    for (MuonProduct &t : list)
        for (int *map : {&t.out, &t.out_lo}) *map += MUON_MAP_OUT;
    return list;
}

// How many workers one kind of matrices has.
int workers_for(const demo_muon_ctx *c, bool precise)
{
    const int device = std::max(1, c->launch.sm_count / 2);
    return std::max(1, c->side_workers == 0 ? device : precise ? c->side_workers : device - c->side_workers);
}

// The products of the matrices mats[0 .. n), `first` the index of the first.  Matrices go through the iterations in cohorts, product by product,
// every product matrix by matrix: with two rounds of the workers' tasks in a cohort's symmetric products, a matrix's next product starts when its last
// is done.  (48 of 2048 x 2048: 9.6 ms with two rounds, 10.3 with one, 9.5 to 9.8 with three to twelve; 60 of 1024 x 1024 2.36, 2.54 and
// 2.2 to 2.35.  Less than one takes up to twice as long, and an order in which workers of a model of the device would start the tasks, with as few
// matrices under way as that takes, as long as two rounds.)  Returns how many tasks there are at once.
int add_tasks(const demo_muon_ctx *c, const MuonMat *mats, int first, int n, int side, Plan *plan)
{
    const int workers = workers_for(c, mats[0].precise);
    auto symmetric = [&](const MuonMat &m) { const long long k = ceil_div(m.m, side); return k * (k + 1) / 2; };
    long long total = 0;
    for (int e = 0; e < n; ++e) total += symmetric(mats[e]);
    const long long cohorts = std::max(1LL, total / (2LL * workers));
    long long before = 0;
    size_t most = 1;
    for (int lo = 0, hi = 0; lo < n; lo = hi) {
        const long long which = before * cohorts / total;
        for (; hi < n && (hi == lo || before * cohorts / total == which); ++hi) before += symmetric(mats[hi]);
        std::vector<std::vector<MuonProduct>> lists;
        for (int e = lo; e < hi; ++e) lists.push_back(products_of(mats[e], c->cfg.steps));
        std::vector<unsigned> completed(lists.size(), 0u);
        for (size_t k = 0, more = 1; more; ++k) {
            more = 0;
            const size_t step = plan->tasks.size();
            for (size_t e = 0; e < lists.size(); ++e) {
                if (k >= lists[e].size()) continue;
                more = 1;
                MuonProduct t = lists[e][k];
                t.mat = first + lo + (int)e;
                t.need = completed[e];
                const int product = (int)plan->products.size();
                plan->products.push_back(t);
                const size_t begin = plan->tasks.size();
                each_tile(ceil_div(t.m, side), ceil_div(t.width, side), t.phase < MUON_UPDATE, [&](int i, int j) {
                    for (int part = 0; part < t.splits; ++part) plan->tasks.push_back(MuonTask{product, (short)i, (short)j, part});
                });
                completed[e] += (unsigned)((plan->tasks.size() - begin) / (size_t)t.splits) * (unsigned)(2 * muon_epilogue_warps(side));
            }
            most = std::max(most, plan->tasks.size() - step);
        }
    }
    return (int)most;
}

// Sets the tile and the way of the iterations of every matrix.
// The first two iterations in one take 3 r + 5 products of m^3 multiplications, one after the other 6 r + 2, r = n / m, but are one product longer.
// Tiles of 256 multiply fastest (twice the products for the bytes that a CTA loads), those of 128 pass from one product to the next fastest (5
// us instead of 8.5).  Which counts for a set is estimated from both: its tasks spread over the workers, and its longest chain of products.
// Measured, us, tiles of 256 / 128, one after the other and with the first two in one where that is not the same:
//   512 x 512 170 / 94; 1024 x 1024 213 / 116, four of them 238 / 193; 2048 x 2048 314 / 299; 4096 x 4096 1380 / 1810
//   512 x 2048 206, 220 / 109, 114; 512 x 4608, five of them 349, 346 / 337, 310; 1024 x 4096 273, 286 / 212, 204, four of them 473, 460 / 552, 498;
//   768 x 8000 334, 330 / 250, 233; 2048 x 8192 697, 653 / 834, 737
void choose_shapes(demo_muon_ctx *c, std::vector<MuonMat> *all)
{
    const double workers = std::max(1, c->launch.sm_count / 2);
    // tiles: of the symmetric products of all matrices of this kind
    auto set = [&](MuonMat &m, int tile, bool twos, double tiles) {
        m.tile = m.precise ? 128 : tile;
        m.twos = twos && !m.precise && c->cfg.steps >= 2 && 2LL * m.n >= 3LL * m.m;
        m.symmetric = m.twos ? 3 : 2;
        // Sums of up to 2048 elements (8192 where the products are of 11 bits) at a time for their exactness: what the tensor core cuts off all goes
        // one way (160 of 64 x 8192, Gaussian / all entries equal: error 4.9e-5 / 5.2e-4 in 3.59 ms at 8192 at a time, 1.1e-5 / 6.4e-5 in 3.66 ms at
        // 2048; 50304 x 384 692, 722, 808 us at 8192, 4096, 2048; 60 of 400 x 32768, all equal: 1.5e-2 in 16.3 ms at 32768, 3e-3 in 14.2 ms at 8192).
        // (From m = 8192 on parts of m, at most 32768: the other products' sums are as long, and a part takes 2 m^2 bytes.)
        // And long ones in three parts of 1024 or more where half of the workers have no tile.  Not more parts than workers: their way through memory
        // costs more than they save.  (In parts for the workers' sake / not / in twice as many: 768 x 8000 234 / 254 / 259 us, 2048 x 8192 654 / 772 / 748,
        // 512 x 16000 260 / 286 / 300, 256 x 8000 165 / 171 / 165.)
        const int steps = ceil_div(m.n, muon_k_step(m.tile)), exact = ceil_div(m.n, m.precise ? 2048 : std::min(32768, std::max(8192, m.m)));
        const int parts = m.n / 1024, spread = parts > 2 && 2 * tiles <= workers ? std::min(parts, (int)(workers / tiles)) : 1;
        m.split_steps = ceil_div(steps, std::max(exact, spread));
        m.splits = ceil_div(steps, m.split_steps);
    };
    auto all_tiles = [&](int tile, bool precise) {
        double n = 0;
        for (const MuonMat &m : *all)
            if ((m.precise != 0) == precise) {
                const double k = ceil_div(m.m, precise ? 128 : tile);
                n += k * (k + 1) / 2;
            }
        return std::max(1.0, n);
    };
    struct Load {
        struct Step {
            double tiles, cost;  // of a product; us: of one of its tasks
        };
        struct Chain {
            std::vector<Step> steps;
            double handovers;  // us
        };
        double total = 0, tasks = 0;  // us: of all tasks, one after the other; how many can be in work at once
        std::vector<Chain> chains;    // of each shape: the products of one matrix, one behind the other
        // us, of w workers: of the tasks spread over them, and of the longest chain
        double time(double w) const
        {
            double chain = 0;
            for (const Chain &c : chains) {
                double one = c.handovers;
                for (const Step &s : c.steps) one += std::ceil(s.tiles / w) * s.cost;
                chain = std::max(chain, one);
            }
            return std::max(total / w, chain) + 0.3 * std::min(total / w, chain);
        }
    };
    auto load = [&](bool precise, int tile, bool twos) {
        // us: of a step of K, of a task beside its steps, from a product's last step to the next one's first
        const double step = precise ? 0.4 : tile == 256 ? 0.28 : 0.2, task = tile == 256 ? 1.5 : 1.0, handover = tile == 256 ? 8.5 : 5.0;
        Load l;
        const double square = all_tiles(tile, precise);
        const MuonMat *last = nullptr;
        double last_total = 0, last_tasks = 0;
        for (const MuonMat &m : *all) {
            if ((m.precise != 0) != precise) continue;
            if (!last || last->m != m.m || last->n != m.n) {
                MuonMat probe = m;
                set(probe, tile, twos, square);
                Load::Chain chain{{}, 0};
                last_total = last_tasks = 0;
                for (const MuonProduct &t : products_of(probe, c->cfg.steps)) {
                    const double rows = ceil_div(t.m, tile), cols = ceil_div(t.width, tile);
                    const Load::Step s{(t.phase < MUON_UPDATE ? rows * (rows + 1) / 2 : rows * cols) * t.splits, t.steps * step + task};
                    chain.steps.push_back(s);
                    chain.handovers += handover + (t.splits > 1 ? 2 : 0);
                    last_total += s.tiles * s.cost;
                    last_tasks = std::max(last_tasks, s.tiles);
                }
                l.chains.push_back(std::move(chain));
                last = &m;
            }
            l.total += last_total;
            l.tasks += last_tasks;
        }
        return l;
    };
    Load best;
    int best_tile = 0;
    bool best_twos = false;
    for (const int tile : {256, 128})
        for (const bool twos : {true, false}) {
            Load l = load(false, tile, twos);
            if (!best_tile || l.time(workers) < best.time(workers)) best = std::move(l), best_tile = tile, best_twos = twos;
        }
    const Load side = load(true, 128, false);
    if (side.total > 0 && best.total > 0) {
        // Both kinds at once, the workers divided between them so that the later of the two ends earliest, and the other early, too, where that costs
        // little: never more for the small ones than they have tasks at once.  (Those of the larger ones stay until their last task is done: were they
        // as many as the device holds, the small ones would come after them.)  Measured, us, larger / small ones alone, both, and the best of fourteen
        // divisions from 1 to 70 workers: 512 x 512 / 64 x 64 93 / 78, 99, 98; 768 x 512 / 256 x 640 and 128 x 128 95 / 105, 117, 115; four of 1024 x
        // 1024 / 256 x 512 195 / 101, 205, 207; 1024 x 1024 / thirty of 256 x 1024 117 / 287, 379, 348; eight of 512 x 512 / forty of 128 x 128 115 / 95, 181, 136.
        auto both = [&](double w) {
            const double small = side.time(w), large = best.time(workers - w);
            return std::max(small, large) + 0.1 * std::min(small, large);
        };
        double least = 0;
        for (int w = 1; w < (int)workers && (w == 1 || w <= side.tasks); w += 1 + w / 8) {
            const double t = both(w);
            if (w == 1 || t < least) least = t, c->side_workers = w;
        }
    }
    const double squares[2] = {all_tiles(best_tile, false), all_tiles(best_tile, true)};
    for (MuonMat &m : *all) set(m, best_tile, best_twos, squares[m.precise != 0]);
}

// Elements of the matrices of one kind from `at` on.
long long total_of(const std::vector<MuonMat> &all, size_t at)
{
    long long n = 0;
    for (size_t e = at; e < all.size() && all[e].precise == all[at].precise; ++e) n += (long long)all[e].m * all[e].n;
    return n;
}

demo_status make_plan(demo_muon_ctx *c, Plan *plan)
{
    std::vector<MuonMat> all((size_t)c->n_tensors);
    for (int t = 0; t < c->n_tensors; ++t) {
        MuonMat &m = all[(size_t)t];
        std::memset(&m, 0, sizeof(m));
        const long long rows = c->descs[(size_t)t].shape[0], cols = c->descs[(size_t)t].shape[1];
        m.transposed = rows > cols;
        m.m = (int)std::min(rows, cols);
        m.n = (int)std::max(rows, cols);
        m.ldx = (int)round_up(m.n, 64);
        m.lde = (int)round_up(m.m, 64);
        m.precise = m.m <= PRECISE_SIDE;
        m.tensor = t;
        // X's elements are of order one once its singular values are: then neither hi nor lo leaves the normal range of fp16
        m.S = (float)std::exp2(std::floor(0.5 * std::log2((double)m.n)));
        m.inv_S = 1.0f / m.S;
        m.step_scale = c->cfg.scale == DEMO_SCALE_RMS      ? 0.2f * std::sqrt((float)m.n)
                       : c->cfg.scale == DEMO_SCALE_ASPECT ? std::sqrt(std::max(1.0f, (float)rows / (float)cols))
                                                           : 1.0f;
    }
    choose_shapes(c, &all);
    // groups hold matrices of one kind
    std::stable_sort(all.begin(), all.end(), [](const MuonMat &x, const MuonMat &y) { return x.precise < y.precise; });
    for (size_t at = 0; at < all.size();) {
        Group g;
        std::memset(&g, 0, sizeof(g));
        g.first_mat = (int)at;
        g.tile = all[at].tile;
        g.precise = all[at].precise != 0;
        long long elements = 0, pieces = 0;
        size_t work = 0, end = at, counters = 0;
        // (32 elements for each thread of a CTA, or eight where there are few: 256 x 512 105.4 us instead of 106.7)
        g.piece = total_of(all, at) < (2LL << 20) ? 2048 : 8192;
        for (; end < all.size() && (all[end].precise != 0) == g.precise; ++end) {
            MuonMat &m = all[end];
            const long long n = (long long)m.m * m.n;
            const size_t place_end = place(m, work);
            if (end > at && (elements + n > GROUP_ELEMENTS || place_end > GROUP_BYTES)) break;
            elements += n;
            work = place_end;
            m.piece_begin = (int)pieces;
            m.n_pieces = (int)((n + g.piece - 1) / g.piece);
            pieces += m.n_pieces;
            m.maps = (int)end * MUON_MAPS;
            m.arrived = (int)(plan->arrived + counters);
            if (m.splits > 1) counters += (size_t)tiles_above(m) * (size_t)(2 * muon_epilogue_warps(m.tile));
        }
        if (pieces > (1LL << 31) - 1) return DEMO_ERR_UNSUPPORTED;
        g.n_mats = (int)(end - at);
        g.arrived = (int)plan->arrived;
        g.n_arrived = (int)counters;
        plan->arrived += counters;
        if (plan->arrived > (size_t)(1LL << 30)) return DEMO_ERR_UNSUPPORTED;
        g.n_pieces = (int)pieces;
        const int kind = g.precise;
        plan->work[kind] = std::max(plan->work[kind], work);
        plan->pieces[kind] = std::max(plan->pieces[kind], g.n_pieces);
        g.pack_tiles = (long long)plan->tiles.size();
        for (size_t e = at; e < end; ++e)
            for (int i = 0; i < ceil_div(all[e].m, MUON_PACK_TILE); ++i)
                for (int j = 0; j < ceil_div(all[e].n, MUON_PACK_TILE); ++j) plan->tiles.push_back(MuonTile{(int)e, (short)i, (short)j});
        g.n_pack = (int)((long long)plan->tiles.size() - g.pack_tiles);
        if (plan->tiles.size() > (size_t)(1LL << 30)) return DEMO_ERR_UNSUPPORTED;
        c->groups.push_back(g);
        at = end;
    }
    plan->mats = std::move(all);
    return DEMO_OK;
}

demo_status make_tasks(demo_muon_ctx *c, Plan *plan)
{
    for (Group &g : c->groups) {
        g.tasks = (long long)plan->tasks.size();
        g.at_once = add_tasks(c, plan->mats.data() + g.first_mat, g.first_mat, g.n_mats, g.tile, plan);
        g.workers = std::min(g.at_once, workers_for(c, g.precise));
        g.n_tasks = (int)((long long)plan->tasks.size() - g.tasks);
        const auto waits = [&](long long k) { const MuonProduct &p = plan->products[(size_t)plan->tasks[(size_t)(g.tasks + k)].product]; return p.mat == g.first_mat && p.phase == MUON_POLY; };
        while (!waits(g.waiting)) ++g.waiting;  // (every matrix has that product)
        while (g.waiting + g.n_waiting < g.n_tasks && waits(g.waiting + g.n_waiting)) ++g.n_waiting;
        if (plan->tasks.size() > (size_t)(1LL << 30)) return DEMO_ERR_UNSUPPORTED;
    }
    return DEMO_OK;
}

// The three maps of a matrix of fp16 elements: see MUON_MAPS.
bool encode_maps(PFN_cuTensorMapEncodeTiled encode, CUtensorMap *map, int tile, void *base, long long cols, long long rows, long long ld)
{
    auto make = [&](CUtensorMap *to, int dims, const cuuint64_t *extent, const cuuint64_t *stride, const cuuint32_t *box, CUtensorMapSwizzle swizzle) {
        const cuuint32_t ones[3] = {1, 1, 1};
        return encode(to, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)dims, base, extent, stride, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    const cuuint64_t flat[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, row[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t panel[2] = {64, 128}, block[2] = {tile == 256 ? 64u : 32u, 32};
    // blocks of 64 columns as the last axis (pad columns are read: along K they are zero, else they only reach results outside the matrix)
    const cuuint64_t cut[3] = {64, (cuuint64_t)rows, (cuuint64_t)(ld / 64)}, cut_stride[2] = {(cuuint64_t)ld * 2, 128};
    const cuuint32_t two[3] = {64, 64, 2};
    return make(map, 2, flat, row, panel, CU_TENSOR_MAP_SWIZZLE_128B) && make(map + MUON_MAP_TWO, 3, cut, cut_stride, two, CU_TENSOR_MAP_SWIZZLE_128B) &&
           make(map + MUON_MAP_OUT, 2, flat, row, block, tile == 256 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}

template <typename T>
bool alloc(demo_muon_ctx *c, T **p, size_t bytes)
{
    if (cudaMalloc((void **)p, bytes) != cudaSuccess) return false;
    c->bytes += bytes;
    return true;
}

demo_status build(demo_muon_ctx *c)
{
    Plan plan;
    demo_status st = make_plan(c, &plan);
    if (st != DEMO_OK) return st;
    PFN_cuTensorMapEncodeTiled encode = nullptr;
    {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess || !fn)
            return DEMO_ERR_UNSUPPORTED;
        encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled>(fn);
    }
    const size_t T = (size_t)c->n_tensors;
    bool ok = alloc(c, &c->d_mats, T * sizeof(MuonMat)) && alloc(c, &c->d_tiles, plan.tiles.size() * sizeof(MuonTile)) &&
              alloc(c, &c->d_done, (2 * T + 4) * sizeof(unsigned)) &&
              alloc(c, &c->d_scales, T * sizeof(float2)) && alloc(c, &c->d_arrived, (plan.arrived + 1) * sizeof(unsigned)) &&
              alloc(c, &c->d_maps, T * MUON_MAPS * MUON_MAP_BYTES) && alloc(c, &c->d_work, plan.work[0] + plan.work[1]) &&
              alloc(c, &c->d_partials, (size_t)(plan.pieces[0] + plan.pieces[1]) * sizeof(double)) && alloc(c, &c->d_status, sizeof(int));
    for (int e = 0; e < ENTRY_POINTS; ++e) ok = ok && c->tables[e].reserve((e == FROM_STEP ? 3 : 2) * T) == DEMO_OK;
    if (ok && plan.work[0] && plan.work[1])
        ok = cudaStreamCreateWithFlags(&c->side_stream, cudaStreamNonBlocking) == cudaSuccess && cudaEventCreateWithFlags(&c->fork, cudaEventDisableTiming) == cudaSuccess &&
             cudaEventCreateWithFlags(&c->join, cudaEventDisableTiming) == cudaSuccess;
    if (!ok) return DEMO_ERR_ALLOC;
    for (MuonMat &m : plan.mats) rebase(m, c->d_work + (m.precise ? plan.work[0] : 0));
    c->side_partials = plan.pieces[0];
    st = make_tasks(c, &plan);
    if (st != DEMO_OK) return st;
    if (!alloc(c, &c->d_products, plan.products.size() * sizeof(MuonProduct)) || !alloc(c, &c->d_tasks, plan.tasks.size() * sizeof(MuonTask))) return DEMO_ERR_ALLOC;
    std::vector<CUtensorMap> maps(T * MUON_MAPS);
    std::memset(maps.data(), 0, maps.size() * sizeof(CUtensorMap));
    for (MuonMat &m : plan.mats) {
        CUtensorMap *p = &maps[(size_t)m.maps];
        for (int k = 0; k < 2; ++k)
            ok = ok && encode_maps(encode, p + MUON_MAP_X + k, m.tile, m.xhi[k], m.n, m.m, m.ldx) && encode_maps(encode, p + MUON_MAP_XLO + k, m.tile, m.xlo[k], m.n, m.m, m.ldx);
        for (int k = 0; k < m.symmetric; ++k)
            ok = ok && encode_maps(encode, p + MUON_MAP_E + k, m.tile, m.ehi[k], m.m, m.m, m.lde) && encode_maps(encode, p + MUON_MAP_ELO + k, m.tile, m.elo[k], m.m, m.m, m.lde);
    }
    if (!ok) return DEMO_ERR_CUDA;
    ok = cudaMemcpy(c->d_mats, plan.mats.data(), T * sizeof(MuonMat), cudaMemcpyHostToDevice) == cudaSuccess &&
         cudaMemcpy(c->d_tiles, plan.tiles.data(), plan.tiles.size() * sizeof(MuonTile), cudaMemcpyHostToDevice) == cudaSuccess &&
         cudaMemcpy(c->d_products, plan.products.data(), plan.products.size() * sizeof(MuonProduct), cudaMemcpyHostToDevice) == cudaSuccess &&
         cudaMemcpy(c->d_tasks, plan.tasks.data(), plan.tasks.size() * sizeof(MuonTask), cudaMemcpyHostToDevice) == cudaSuccess &&
         cudaMemcpy(c->d_maps, maps.data(), maps.size() * sizeof(CUtensorMap), cudaMemcpyHostToDevice) == cudaSuccess &&
         cudaMemset(c->d_status, 0, sizeof(int)) == cudaSuccess && cudaMemset(c->d_done, 0, (2 * T + 4) * sizeof(unsigned)) == cudaSuccess &&
         cudaStreamSynchronize(nullptr) == cudaSuccess;  // (the first call may be on a stream that does not wait for this one)
    return ok ? DEMO_OK : DEMO_ERR_CUDA;
}

// What the kernels of every call take.
void fill_common(const demo_muon_ctx *c, MuonArgs *a)
{
    a->mats = c->d_mats;
    a->maps = c->d_maps;
    a->done = c->d_done;
    a->ready = c->d_done + c->n_tensors;
    a->scales = c->d_scales;
    a->arrived = c->d_arrived;
    a->wait_cycles = WAIT_CYCLES;
    a->status = c->d_status;
}

demo_status run(demo_muon_ctx *c, MuonArgs a, const PointerTable &t, cudaStream_t stream)
{
    const demo_muon_config &g = c->cfg;
    fill_common(c, &a);
    a.in = const_cast<const void *const *>(t.dev());
    a.out = t.dev() + c->n_tensors;
    a.mom = a.from == MUON_FROM_STEP ? reinterpret_cast<float *const *>(t.dev() + 2 * (size_t)c->n_tensors) : nullptr;
    a.nesterov = g.nesterov;
    a.mu = g.momentum;
    a.eps = g.eps;
    a.lr = g.lr;
    a.wd = g.weight_decay;
    a.a = g.coefficients[0];
    a.b = g.coefficients[1];
    a.c = g.coefficients[2];
    cudaError_t err = cudaSuccess;
    const bool both = c->side_stream != nullptr;
    if (both) {
        err = cudaEventRecord(c->fork, stream);
        if (err == cudaSuccess) err = cudaStreamWaitEvent(c->side_stream, c->fork, 0);
    }
    for (int kind = 1; kind >= 0; --kind)  // (the small matrices first: they take a few SMs, the others the rest)
        for (const Group &grp : c->groups) {
            if (grp.precise != (kind == 1)) continue;
            cudaStream_t on = both && kind ? c->side_stream : stream;
            a.partials = c->d_partials + (kind ? c->side_partials : 0);
            a.piece = grp.piece;
            a.next_task = c->d_done + 2 * c->n_tensors + kind;
            a.gave_up = a.next_task + 2;
            if (err == cudaSuccess) err = muon_launch_norm(a, grp.first_mat, grp.n_mats, grp.n_pieces, c->launch, on);
            if (err == cudaSuccess) err = muon_launch_pack(a, c->d_tiles + grp.pack_tiles, grp.n_pack, grp.first_mat, grp.n_mats, grp.arrived, grp.n_arrived, c->launch, on);
            if (err == cudaSuccess) err = muon_launch_products(grp.tile, grp.precise, a, c->d_products, c->d_tasks + grp.tasks, grp.n_tasks, grp.workers, c->launch, on);
            c->launches += 3;
        }
    if (both) {  // (also after a failure: a forked capture has to be joined)
        const cudaError_t joined = cudaEventRecord(c->join, c->side_stream), waited = cudaStreamWaitEvent(stream, c->join, 0);
        if (err == cudaSuccess) err = joined != cudaSuccess ? joined : waited;
    }
    if (err != cudaSuccess) {
        cudaGetLastError();
        return DEMO_ERR_CUDA;
    }
    return DEMO_OK;
}

bool usable(const void *const *p, int n)
{
    for (int t = 0; t < n; ++t)
        if (!p[t] || !aligned16(p[t])) return false;
    return true;
}

}  // namespace

extern "C" {

int demo_muon_plan(const demo_muon_config *cfg, const demo_tensor_desc *tensors, int n_tensors, int sm_count, int *groups, int most_groups)
{
    try {
        demo_muon_ctx c;
        c.cfg = *cfg;
        c.n_tensors = n_tensors;
        c.launch.sm_count = sm_count;
        c.descs.assign(tensors, tensors + n_tensors);
        Plan plan;
        if (make_plan(&c, &plan) != DEMO_OK || make_tasks(&c, &plan) != DEMO_OK) return -1;
        int n = 0;
        for (const Group &g : c.groups)
            if (n < most_groups) {
                int *to = groups + 7 * n++;
                to[0] = g.precise, to[1] = g.tile, to[2] = g.n_mats, to[3] = g.n_tasks, to[4] = g.at_once, to[5] = g.workers;
                to[6] = plan.mats[(size_t)g.first_mat].twos;
            }
        return (int)c.groups.size();
    } catch (const std::exception &) {
        return -1;
    }
}

demo_status demo_muon_init(demo_muon_ctx **out, const demo_muon_config *cfg, const demo_tensor_desc *tensors, int32_t n_tensors, int32_t cuda_device)
{
    if (out) *out = nullptr;
    if (!out || !cfg || !tensors || n_tensors < 1 || cuda_device < 0) return DEMO_ERR_INVALID_ARG;
    for (const float v : {cfg->momentum, cfg->coefficients[0], cfg->coefficients[1], cfg->coefficients[2], cfg->eps, cfg->lr, cfg->weight_decay})
        if (!std::isfinite(v)) return DEMO_ERR_INVALID_ARG;
    if (cfg->steps < 1 || cfg->steps > DEMO_MUON_MAX_STEPS || cfg->eps < 0 || (cfg->nesterov != 0 && cfg->nesterov != 1)) return DEMO_ERR_INVALID_ARG;
    if (cfg->scale != DEMO_SCALE_NONE && cfg->scale != DEMO_SCALE_ASPECT && cfg->scale != DEMO_SCALE_RMS) return DEMO_ERR_INVALID_ARG;
    if (cfg->grad_dtype != DEMO_F32 && cfg->grad_dtype != DEMO_BF16) return DEMO_ERR_UNSUPPORTED;
    if (n_tensors > DEMO_MUON_MAX_TENSORS) return DEMO_ERR_UNSUPPORTED;
    for (int t = 0; t < n_tensors; ++t) {
        const demo_tensor_desc &d = tensors[t];
        if (d.ndim != 2) return DEMO_ERR_SHAPE;
        for (int a = 0; a < 2; ++a)
            if (d.shape[a] < 1 || d.shape[a] > DEMO_MUON_MAX_EXTENT) return DEMO_ERR_SHAPE;
    }
    int n_dev = 0;
    if (cudaGetDeviceCount(&n_dev) != cudaSuccess || cuda_device >= n_dev) {
        cudaGetLastError();
        return DEMO_ERR_CUDA;
    }
    DeviceGuard guard(cuda_device);
    if (!guard.ok) return DEMO_ERR_CUDA;
    demo_muon_ctx *c = new (std::nothrow) demo_muon_ctx();
    if (!c) return DEMO_ERR_ALLOC;
    demo_status st = DEMO_OK;
    if (cudaDeviceGetAttribute(&c->launch.sm_count, cudaDevAttrMultiProcessorCount, cuda_device) != cudaSuccess) st = DEMO_ERR_CUDA;
    if (st == DEMO_OK) {
        try {
            c->cfg = *cfg;
            c->device = cuda_device;
            c->n_tensors = n_tensors;
            c->descs.assign(tensors, tensors + n_tensors);
            st = build(c);
        } catch (const std::exception &) {  // (no memory, or a list longer than a vector can be)
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

demo_status demo_orthogonalize(demo_muon_ctx *ctx, const void *const *in, int32_t in_dtype, void *const *out, int32_t out_dtype, void *cuda_stream)
{
    if (!ctx || !in || !out) return DEMO_ERR_INVALID_ARG;
    for (const int32_t d : {in_dtype, out_dtype})
        if (d != DEMO_F32 && d != DEMO_BF16) return DEMO_ERR_UNSUPPORTED;
    if (!usable(in, ctx->n_tensors) || !usable(out, ctx->n_tensors)) return DEMO_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return DEMO_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    PointerTable &t = ctx->tables[FROM_ORTHOGONALIZE];
    const size_t T = (size_t)ctx->n_tensors;
    const demo_status st = t.sync({{in, T}, {out, T}}, stream);
    if (st != DEMO_OK) return st;
    MuonArgs a{};
    a.from = MUON_FROM_INPUT;
    a.to = MUON_TO_OUTPUT;
    a.in_bf16 = in_dtype == DEMO_BF16;
    a.out_bf16 = out_dtype == DEMO_BF16;
    return run(ctx, a, t, stream);
}

demo_status demo_muon_step(demo_muon_ctx *ctx, const void *const *grads, float *const *momentum, float *const *params, void *cuda_stream)
{
    if (!ctx || !grads || !momentum || !params) return DEMO_ERR_INVALID_ARG;
    if (!usable(grads, ctx->n_tensors) || !usable(reinterpret_cast<const void *const *>(momentum), ctx->n_tensors) ||
        !usable(reinterpret_cast<const void *const *>(params), ctx->n_tensors))
        return DEMO_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return DEMO_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    PointerTable &t = ctx->tables[FROM_STEP];
    const size_t T = (size_t)ctx->n_tensors;
    const demo_status st = t.sync({{grads, T}, {reinterpret_cast<const void *const *>(params), T}, {reinterpret_cast<const void *const *>(momentum), T}}, stream);
    if (st != DEMO_OK) return st;
    MuonArgs a{};
    a.from = MUON_FROM_STEP;
    a.to = MUON_TO_PARAMS;
    a.in_bf16 = ctx->cfg.grad_dtype == DEMO_BF16;
    return run(ctx, a, t, stream);
}

demo_status demo_muon_decode_apply(demo_muon_ctx *ctx, demo_ctx *demo, const void *const *payloads, int32_t n_payloads, float *const *params, void *cuda_stream)
{
    if (!ctx || !demo || !payloads || !params) return DEMO_ERR_INVALID_ARG;
    std::vector<void *> out;
    std::vector<float *> table;
    try {
        std::vector<int> place;
        const demo_status st = demo_decode_places(demo, ctx->device, ctx->descs.data(), ctx->n_tensors, &place);
        if (st != DEMO_OK) return st;
        if (!usable(reinterpret_cast<const void *const *>(params), (int)place.size())) return DEMO_ERR_INVALID_ARG;
        DeviceGuard guard(ctx->device);
        if (!guard.ok) return DEMO_ERR_CUDA;
        cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
        if (!ctx->d_momentum) {
            cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
            if (cudaStreamIsCapturing(stream, &capture) != cudaSuccess) {
                cudaGetLastError();
                return DEMO_ERR_CUDA;
            }
            if (capture != cudaStreamCaptureStatusNone) return DEMO_ERR_INVALID_ARG;
            size_t n = 0;
            for (const demo_tensor_desc &d : ctx->descs) n += (size_t)round_up(d.shape[0] * d.shape[1], 64);
            ctx->momentum_ptrs.assign((size_t)ctx->n_tensors, nullptr);
            if (!alloc(ctx, &ctx->d_momentum, n * sizeof(float))) {
                cudaGetLastError();
                ctx->d_momentum = nullptr;
                return DEMO_ERR_ALLOC;
            }
            ctx->momentum_bytes = n * sizeof(float);
            size_t at = 0;
            for (int t = 0; t < ctx->n_tensors; ++t) {
                ctx->momentum_ptrs[(size_t)t] = ctx->d_momentum + at;
                at += (size_t)round_up(ctx->descs[(size_t)t].shape[0] * ctx->descs[(size_t)t].shape[1], 64);
            }
        }
        table.resize(place.size());
        out.resize((size_t)ctx->n_tensors);
        for (size_t i = 0; i < place.size(); ++i) {
            table[i] = place[i] < 0 ? params[i] : ctx->momentum_ptrs[(size_t)place[i]];
            if (place[i] >= 0) out[(size_t)place[i]] = params[i];
        }
        PointerTable &t = ctx->tables[FROM_DECODE];
        demo_status done = t.sync({{reinterpret_cast<const void *const *>(ctx->momentum_ptrs.data()), out.size()}, {out.data(), out.size()}}, stream);
        if (done != DEMO_OK) return done;
        done = demo_decode_momentum(demo, payloads, n_payloads, table.data(), ctx->d_momentum, ctx->momentum_bytes, stream);
        if (done != DEMO_OK) return done;
        MuonArgs a{};
        a.from = MUON_FROM_INPUT;
        a.to = MUON_TO_PARAMS;
        return run(ctx, a, t, stream);
    } catch (const std::exception &) {
        return DEMO_ERR_ALLOC;
    }
}

demo_status demo_muon_set_lr(demo_muon_ctx *ctx, float lr)
{
    if (!ctx || !std::isfinite(lr)) return DEMO_ERR_INVALID_ARG;
    ctx->cfg.lr = lr;
    return DEMO_OK;
}

size_t demo_muon_workspace_bytes(const demo_muon_ctx *ctx)
{
    size_t tables = 0;
    if (ctx)
        for (const PointerTable &t : ctx->tables) tables += t.bytes();
    return ctx ? ctx->bytes + tables : 0;
}

int64_t demo_muon_launch_count(const demo_muon_ctx *ctx) { return ctx ? ctx->launches : 0; }

demo_status demo_muon_device_status(demo_muon_ctx *ctx, void *cuda_stream)
{
    if (!ctx) return DEMO_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return DEMO_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int word = 0;
    if (cudaMemcpyAsync(&word, ctx->d_status, sizeof(int), cudaMemcpyDeviceToHost, stream) != cudaSuccess || cudaStreamSynchronize(stream) != cudaSuccess ||
        (word != 0 && (cudaMemsetAsync(ctx->d_status, 0, sizeof(int), stream) != cudaSuccess || cudaStreamSynchronize(stream) != cudaSuccess))) {
        cudaGetLastError();
        return DEMO_ERR_CUDA;
    }
    return word == 0 ? DEMO_OK : word == DEMO_DEV_TIMEOUT ? DEMO_ERR_TIMEOUT : DEMO_ERR_CUDA;
}

demo_status demo_muon_selftest_bounded_wait(demo_muon_ctx *ctx, int64_t limit_cycles, void *cuda_stream)
{
    if (!ctx || limit_cycles < 1 || limit_cycles > 2000000000LL) return DEMO_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return DEMO_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const Group &g = ctx->groups.front();
    MuonArgs a{};
    fill_common(ctx, &a);
    a.wait_cycles = limit_cycles;
    a.next_task = ctx->d_done + 2 * ctx->n_tensors;
    a.gave_up = a.next_task + 2;
    // no product is done, no task drawn
    if (cudaMemsetAsync(ctx->d_done + g.first_mat, 0, sizeof(unsigned), stream) != cudaSuccess || cudaMemsetAsync(a.next_task, 0, 4 * sizeof(unsigned), stream) != cudaSuccess ||
        muon_launch_products(g.tile, g.precise, a, ctx->d_products, ctx->d_tasks + g.tasks + g.waiting, g.n_waiting, g.workers, ctx->launch, stream) != cudaSuccess) {
        cudaGetLastError();
        return DEMO_ERR_CUDA;
    }
    ctx->launches += 1;
    return DEMO_OK;
}

void demo_muon_free(demo_muon_ctx *ctx)
{
    if (!ctx) return;
    DeviceGuard guard(ctx->device);
    release(ctx);
}

}  // extern "C"
