// Host side of the full-rank matrix step (Newton-Schulz orthogonalisation, Muon) and of the AdamW step: plans, workspace
// layout, launch batches and the sequence of products.  All device work is enqueued on the caller's stream.
#include "../../include/orthdion.h"

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <memory>
#include <mutex>
#include <new>
#include <vector>

#include "adamw.cuh"
#include "lanes.cuh"
#include "newton_schulz.cuh"

using namespace od;

namespace {
constexpr uint32_t kMuonMagic = 0x0D10B0E5u, kAdamWMagic = 0x0D10ADA3u;
constexpr int32_t kMaxSteps = 32;
constexpr size_t kScratchBudget = (size_t)1 << 30;     // per launch batch
constexpr int kPlannedLanes = 4;
constexpr int kTwoTermChunk = 1;                        // depth blocks of 64 that two-plane products sum in tensor memory
}  // namespace

struct orthdion_muon_plan {
    uint32_t magic;
    int64_t m, n;
    int64_t ld_x, ld_m, ld_g;
    double mu;
    float eta, wd, scale;
    int32_t nesterov, x_dtype, g_dtype;
    int32_t passes, passes_set;
    int32_t steps;
    double eps;
    float abc[kMaxSteps][3];
};

struct orthdion_adamw_plan {
    uint32_t magic;
    int64_t numel;
    double beta1, beta2;
    float eps, eta, wd;
    int32_t x_dtype, g_dtype;
};

namespace {

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool valid(orthdion_muon_t h) { return h && h->magic == kMuonMagic; }
inline bool valid(orthdion_adamw_t h) { return h && h->magic == kAdamWMagic; }
inline bool known(int32_t dtype) { return dtype == ORTHDION_DTYPE_F32 || dtype == ORTHDION_DTYPE_BF16; }

int check_ptr(const void* p) {
    if (!p) return ORTHDION_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(p) % 16) return ORTHDION_ERR_ALIGNMENT;
    return 0;
}

// Whether a pointer stands twice among `count`: two matrices of a call that are one would race.
bool twice(const void* const* p, int32_t count) {
    std::vector<const void*> v(p, p + count);
    std::sort(v.begin(), v.end());
    return std::adjacent_find(v.begin(), v.end()) != v.end();
}

// Two matrices that one launch can serve.  (The bytes of a plan: every field is set by value, padding cleared on creation.)
bool same_class(const orthdion_muon_plan* a, const orthdion_muon_plan* b) { return a == b || std::memcmp(a, b, sizeof(*a)) == 0; }

int terms_of(const orthdion_muon_plan* p) { return p->passes == 3 ? 2 : 1; }

// Steps per product with X.  A pair of steps makes one Gram product of X (s^2 l multiply-adds by half), A^2 twice,
// A' = Q A Q and P = Q' Q (five products of s^3 by half in all) and X = P X (s^2 l): 3 l + 5 s against 2 (3 l + s) of single
// steps, in units of s^2 by half.  The rounding of A, relative to its norm, is multiplied by up to a^2 where a pair forms A', which counts
// while some directions have grown and others have not: not in the first two steps (all singular values are small after the division by
// the norm) and not in the last two, but in between (noise and 32 strong directions, 129 x 1000, error of the result by grouping of five steps:
// 2,2,1 8.1e-3; 1,2,2 2.8e-3; singles 2.5e-3; 2,1,2 2.3e-3; 2,1,1,1 2.2e-3).  A pair in front costs a square matrix nothing and saves
// a rounding of X; one at the end pays where the matrix is longer than wide.
std::vector<int> group_steps(const orthdion_muon_plan* p) {
    std::vector<int> out;
    const int64_t s = std::min(p->m, p->n), l = std::max(p->m, p->n);
    const bool pair_last = p->steps >= 5 && 4 * l >= 5 * s;
    for (int left = p->steps; left > 0; left -= out.back())
        out.push_back((left == p->steps || (pair_last && left == 2)) ? std::min(2, left) : 1);
    return out;
}

struct Scratch {
    int64_t slot, part, x[2], sq[4];        // byte offsets inside the scratch of a batch of `count` matrices
    int64_t x_pitch, x_term, x_mat;         // in elements
    int64_t s_pitch, s_term, s_mat;
    size_t bytes;
};

Scratch scratch_layout(const orthdion_muon_plan* p, int count) {
    Scratch c{};
    const int terms = terms_of(p);
    const int64_t s = std::min(p->m, p->n);
    c.x_pitch = (int64_t)align_up(p->n, 64); c.x_term = p->m * c.x_pitch; c.x_mat = terms * c.x_term;
    c.s_pitch = (int64_t)align_up(s, 64); c.s_term = s * c.s_pitch; c.s_mat = terms * c.s_term;
    const std::vector<int> groups = group_steps(p);
    size_t off = 0;
    c.slot = 0; off += align_up(count * sizeof(ns::Slot), 256);
    c.part = off; off += align_up((size_t)count * ns::MAX_PARTS * 8, 256);
    for (int i = 0; i < 2; ++i) {
        c.x[i] = off;
        if (i == 0 || groups.size() > 1) off += align_up((size_t)count * c.x_mat * 2, 1024);
    }
    for (int i = 0; i < 4; ++i) {
        c.sq[i] = off;
        if (i < 2 || groups[0] > 1) off += align_up((size_t)count * c.s_mat * 2, 1024);
    }
    c.bytes = align_up(off, 1024);
    return c;
}

// Launch batches of a call (matrices of one class, so many that the scratch stays within the budget), in the order in which they are
// enqueued, and the lanes they run on: one chain of launches leaves multiprocessors idle at the end of each, which those of another lane fill.
// Every lane has scratch of its own.
struct Batching {
    std::vector<std::vector<int>> batches;
    std::vector<size_t> off;           // scratch offset
    int lanes = 1;                     // batch i runs on lane i % lanes
    size_t scratch = 0;
};

double cost(const orthdion_muon_plan* p, size_t count) {
    const double s = (double)std::min(p->m, p->n), l = (double)std::max(p->m, p->n);
    return (double)count * p->steps * s * s * (3 * l + s) * (p->passes == 3 ? 3 : 1);
}

Batching make_batches(const orthdion_muon_t* hs, int32_t count) {
    Batching out;
    std::vector<char> done(count, 0);
    for (int i = 0; i < count; ++i) {
        if (done[i]) continue;
        std::vector<int> cls;
        for (int j = i; j < count; ++j)
            if (!done[j] && same_class(hs[i], hs[j])) { cls.push_back(j); done[j] = 1; }
        const size_t per = scratch_layout(hs[i], 1).bytes;
        const size_t cap = std::min<size_t>(std::max<size_t>(1, kScratchBudget / per), ns::MAX_BATCH);
        const size_t nb = (cls.size() + cap - 1) / cap, bs = (cls.size() + nb - 1) / nb;
        for (size_t b = 0; b < cls.size(); b += bs) out.batches.emplace_back(cls.begin() + b, cls.begin() + std::min(cls.size(), b + bs));
    }
    // heaviest first
    std::stable_sort(out.batches.begin(), out.batches.end(),
                     [&](const auto& a, const auto& b) { return cost(hs[a[0]], a.size()) > cost(hs[b[0]], b.size()); });
    out.lanes = std::min<int>(kPlannedLanes, (int)out.batches.size());
    std::vector<size_t> most(out.lanes, 0), at(out.lanes, 0);
    for (size_t b = 0; b < out.batches.size(); ++b)
        most[b % out.lanes] = std::max(most[b % out.lanes], scratch_layout(hs[out.batches[b][0]], (int)out.batches[b].size()).bytes);
    for (int l = 0; l < out.lanes; ++l) { at[l] = out.scratch; out.scratch += most[l]; }
    for (size_t b = 0; b < out.batches.size(); ++b) out.off.push_back(at[b % out.lanes]);
    return out;
}

size_t status_bytes(int32_t count) { return align_up((size_t)count * 4, 1024); }

// A 4-d map over the images (columns, rows, planes, matrices) of a batch.
bool encode(CUtensorMap* map, const void* base, int64_t cols, int64_t rows, int terms, int count, int64_t pitch, int64_t term, int64_t mat,
            int box_rows, int box_terms) {
    TensorMapEncodeFn enc = tensor_map_encoder();
    if (!enc) { engine_error() = 1; return false; }
    const cuuint64_t dims[4] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)terms, (cuuint64_t)count};
    const cuuint64_t strides[3] = {(cuuint64_t)pitch * 2, (cuuint64_t)term * 2, (cuuint64_t)mat * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, (cuuint32_t)box_terms, 1}, ones[4] = {1, 1, 1, 1};
    const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        std::fprintf(stderr, "orthdion: cuTensorMapEncodeTiled failed (%d)\n", (int)r);
        engine_error() = 2;
        return false;
    }
    return true;
}

struct Image {
    char* base;
    int64_t rows, cols, pitch, term, mat;
};

// One batch on its way through the products.
struct Chain {
    const orthdion_muon_plan* p;
    int count, terms;
    ns::Slot* slot;
    cudaStream_t st;
};

template <bool PAIR, int BN, int TERMS, int EPI, class TABLE>
void launch_gemm(const Chain& c, ns::GemmArgs& g, const Image& a, const Image& b, const Image* out, const TABLE& table) {
    constexpr int TM = ns::tile_rows<PAIR>(), NB = ns::side_rows<PAIR, BN>();
    g.m_tiles = (g.rows + TM - 1) / TM;
    g.n_tiles = (g.cols + BN - 1) / BN;
    g.tiles = g.sym ? (TM / BN == 1 ? g.m_tiles * (g.m_tiles + 1) / 2 : g.m_tiles * (g.m_tiles + 1)) : g.m_tiles * g.n_tiles;
    g.total = g.tiles * c.count;
    if (!encode(&g.map_a, a.base, a.cols, a.rows, TERMS, c.count, a.pitch, a.term, a.mat, g.a_mn ? 64 : 128, TERMS)) return;
    if (!encode(&g.map_b, b.base, b.cols, b.rows, TERMS, c.count, b.pitch, b.term, b.mat, g.b_mn ? 64 : NB, TERMS)) return;
    if (out) {
        g.out = reinterpret_cast<__half*>(out->base);
        g.pitch = out->pitch; g.term_stride = out->term; g.mat_stride = out->mat;
    }
    const int sms = sm_count(), units = std::min(g.total, PAIR ? sms / 2 : sms);
    launch(ns::gemm_kernel<PAIR, BN, TERMS, EPI, TABLE>, dim3((unsigned)(PAIR ? 2 * units : units)), ns::THREADS, ns::SMEM_BYTES, PAIR ? 2 : 1,
           prof::S_NS_PRODUCT, c.st, table, g);
}

// Tile shape of a product.
enum TileShape { T_PAIR256, T_SINGLE128 };
TileShape tile_shape(const ns::GemmArgs& g, int count) {
    const int64_t mt = (g.rows + 255) / 256, nt = (g.cols + 255) / 256;
    const int64_t tiles = (g.sym ? mt * (mt + 1) / 2 : mt * nt) * count;
    return tiles >= sm_count() / 2 ? T_PAIR256 : T_SINGLE128;
}

template <int EPI, class TABLE>
void product(const Chain& c, ns::GemmArgs& g, const Image& a, const Image& b, const Image* out, const TABLE& table) {
    g.slot = c.slot; g.count = c.count;
    g.chunk = c.terms == 2 ? kTwoTermChunk : g.kblocks;
    const TileShape ts = tile_shape(g, c.count);
    if (c.terms == 2) {
        if (ts == T_PAIR256) launch_gemm<true, 256, 2, EPI>(c, g, a, b, out, table);
        else launch_gemm<false, 128, 2, EPI>(c, g, a, b, out, table);
    } else {
        if (ts == T_PAIR256) launch_gemm<true, 256, 1, EPI>(c, g, a, b, out, table);
        else launch_gemm<false, 128, 1, EPI>(c, g, a, b, out, table);
    }
}

int depth_blocks(int64_t k) { return (int)((k + 63) / 64); }

// out = alpha A B (+ beta C + diag I) of symmetric s x s images that commute
void square_product(const Chain& c, const Image& a, const Image& b, const Image& out, float alpha, const Image* add = nullptr, float beta = 0.f,
                    float diag = 0.f) {
    ns::GemmArgs g{};
    g.rows = g.cols = (int32_t)a.rows;
    g.kblocks = depth_blocks(a.rows);
    g.sym = 1;
    g.alpha = alpha; g.beta = beta; g.diag = diag;
    g.add = add ? reinterpret_cast<const __half*>(add->base) : nullptr;
    product<ns::EPI_IMAGE>(c, g, a, b, &out, ns::NoTable{0});
}

// A = X X^T, or X^T X of a tall matrix
void gram_product(const Chain& c, const Image& x, const Image& out, bool first) {
    const bool wide = c.p->m <= c.p->n;
    ns::GemmArgs g{};
    g.rows = g.cols = (int32_t)std::min(c.p->m, c.p->n);
    g.kblocks = depth_blocks(std::max(c.p->m, c.p->n));
    g.sym = 1;
    g.a_mn = g.b_mn = wide ? 0 : 1;
    g.alpha = 1.f / ns::UNIT;
    g.sigma_pow = first ? 2 : 0;
    product<ns::EPI_IMAGE>(c, g, x, x, &out, ns::NoTable{0});
}

// X' = P X, or X P of a tall matrix: to an image, or (out null) to the caller's matrix
void apply_product(const Chain& c, const Image& pm, const Image& x, const Image* out, bool first, const ns::Table* table, bool update) {
    const bool wide = c.p->m <= c.p->n;
    ns::GemmArgs g{};
    g.rows = (int32_t)c.p->m; g.cols = (int32_t)c.p->n;
    g.kblocks = depth_blocks(std::min(c.p->m, c.p->n));
    g.b_mn = wide ? 1 : 0;
    g.sigma_pow = first ? 1 : 0;
    const Image &a = wide ? pm : x, &b = wide ? x : pm;
    if (out) {
        g.alpha = 1.f / ns::UNIT;
        product<ns::EPI_IMAGE>(c, g, a, b, out, ns::NoTable{0});
    } else {
        g.alpha = 1.f / (ns::UNIT * ns::UNIT);
        g.update = update;
        g.x_bf16 = c.p->x_dtype == ORTHDION_DTYPE_BF16;
        g.wc = 1.f - c.p->eta * c.p->wd; g.wd = c.p->eta * c.p->scale;
        g.ld_x = c.p->ld_x;
        const int64_t whole = g.x_bf16 ? 8 : 4;
        g.x_vec = c.p->n % whole == 0 && c.p->ld_x % whole == 0;
        product<ns::EPI_FINAL>(c, g, a, b, nullptr, *table);
    }
}

void run_batch(const orthdion_muon_plan* p, const ns::Table& t, bool update, char* scratch, cudaStream_t st) {
    const Scratch sc = scratch_layout(p, t.count);
    const int terms = terms_of(p);
    ns::PrepArgs a{};
    a.rows = p->m; a.cols = p->n; a.ld_g = p->ld_g; a.ld_m = p->ld_m;
    a.g_bf16 = p->g_dtype == ORTHDION_DTYPE_BF16; a.nesterov = p->nesterov;
    a.mu = (float)p->mu; a.rest = (float)(1.0 - p->mu);
    a.eps = p->eps;
    a.terms = terms;
    a.vec = p->n % 8 == 0 && p->ld_g % 8 == 0 && (!update || p->ld_m % 4 == 0);
    a.part = reinterpret_cast<double*>(scratch + sc.part);
    a.slot = reinterpret_cast<ns::Slot*>(scratch + sc.slot);
    a.img = reinterpret_cast<__half*>(scratch + sc.x[0]);
    a.pitch = sc.x_pitch; a.term_stride = sc.x_term; a.mat_stride = sc.x_mat;
    // four chunks of 8 a thread, and no more blocks than eight per multiprocessor
    const int64_t chunks = (p->n + 7) / 8 * p->m;
    const int64_t most = std::max<int64_t>(1, 8 * sm_count() / t.count);
    a.parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>({(chunks + 1023) / 1024, most, ns::MAX_PARTS}));
    launch(ns::norm_kernel, dim3((unsigned)a.parts, (unsigned)t.count), 256, 0, 1, prof::S_NS_BUFFER, st, t, a);
    const unsigned blocks = (unsigned)std::max<int64_t>(1, std::min<int64_t>((chunks + 1023) / 1024, most));
    launch(ns::prep_kernel, dim3(blocks, (unsigned)t.count), 256, 0, 1, prof::S_NS_BUFFER, st, t, a);

    const Chain c{p, t.count, terms, a.slot, st};
    const int64_t s = std::min(p->m, p->n);
    Image x[2], sq[4];
    for (int i = 0; i < 2; ++i) x[i] = Image{scratch + sc.x[i], p->m, p->n, sc.x_pitch, sc.x_term, sc.x_mat};
    for (int i = 0; i < 4; ++i) sq[i] = Image{scratch + sc.sq[i], s, s, sc.s_pitch, sc.s_term, sc.s_mat};
    const std::vector<int> groups = group_steps(p);
    const float unit = 1.f / ns::UNIT;
    int step = 0, cur = 0;
    auto poly = [&](const Image& out) {          // Q = a I + b A + c A^2 of the next step, A in sq[0]
        const float* k = p->abc[step++];
        square_product(c, sq[0], sq[0], out, k[2] * unit, &sq[0], k[1], k[0] * ns::UNIT);
    };
    for (size_t gi = 0; gi < groups.size(); ++gi) {
        const bool first = gi == 0, last = gi + 1 == groups.size();
        gram_product(c, x[cur], sq[0], first);
        poly(sq[1]);
        if (groups[gi] == 2) {
            square_product(c, sq[1], sq[0], sq[2], unit);       // A' = Q (Q A)
            square_product(c, sq[1], sq[2], sq[0], unit);
            poly(sq[3]);
            square_product(c, sq[3], sq[1], sq[2], unit);       // P = Q' Q
        }
        apply_product(c, sq[groups[gi] == 2 ? 2 : 1], x[cur], last ? nullptr : &x[1 - cur], first, &t, update);
        cur = 1 - cur;
    }
}

int ensure_attributes() {
    static std::mutex mu;
    static signed char state[kMaxDevices] = {};   // 0 unknown, 1 ok, -1 failed
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return ORTHDION_ERR_CUDA;
    std::lock_guard<std::mutex> lock(mu);
    if (state[dev]) return state[dev] > 0 ? 0 : ORTHDION_ERR_CUDA;
    cudaError_t e = cudaSuccess;
    auto set = [&](auto* kernel) {
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ns::SMEM_BYTES);
    };
#define OD_SET(...) set(ns::gemm_kernel<__VA_ARGS__, ns::EPI_IMAGE, ns::NoTable>); set(ns::gemm_kernel<__VA_ARGS__, ns::EPI_FINAL, ns::Table>);
    OD_SET(true, 256, 1)
    OD_SET(true, 256, 2)
    OD_SET(false, 128, 1)
    OD_SET(false, 128, 2)
#undef OD_SET
    if (e != cudaSuccess) std::fprintf(stderr, "orthdion: kernel attribute setup failed on device %d: %s\n", dev, cudaGetErrorString(e));
    state[dev] = e == cudaSuccess ? 1 : -1;
    return e == cudaSuccess ? 0 : ORTHDION_ERR_CUDA;
}

// What the launches of a call came to.
int launch_outcome() {
    const int e = engine_error();
    if (!e) return ORTHDION_OK;
    if (e == LAUNCH_FAILED) std::fprintf(stderr, "orthdion: launch failed: %s\n", cudaGetErrorString(cudaGetLastError()));
    else std::fprintf(stderr, "orthdion: tensor-map set-up failed (%d)\n", e);
    return ORTHDION_ERR_CUDA;
}

// No exception leaves a C entry point: what the host heap does not hold is an error code.
template <class R, class F>
R guarded(R failed, F f) {
    try {
        return f();
    } catch (...) {
        return failed;
    }
}

// X: weights (M not null) or where the result goes
int run_call(const orthdion_muon_t* hs, int32_t count, void* const* X, float* const* M, const void* const* G, bool update, void* workspace,
             size_t workspace_bytes, void* stream) {
    if (!hs || !X || (update && !M) || !G || !workspace) return ORTHDION_ERR_NULL;
    if (count < 1) return ORTHDION_ERR_INVALID_ARG;
    for (int i = 0; i < count; ++i) {
        if (!valid(hs[i])) return ORTHDION_ERR_INVALID_ARG;
        int e;
        if ((e = check_ptr(X[i])) || (update && (e = check_ptr(M[i]))) || (e = check_ptr(G[i]))) return e;
    }
    if (twice(X, count) || (update && twice(reinterpret_cast<const void* const*>(M), count))) return ORTHDION_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(workspace) % 256) return ORTHDION_ERR_WORKSPACE;
    const Batching bt = make_batches(hs, count);
    if (workspace_bytes < status_bytes(count) + bt.scratch) return ORTHDION_ERR_WORKSPACE;
    int e = ensure_attributes();
    if (e) return e;
    char* ws = reinterpret_cast<char*>(workspace);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int lanes = std::min(bt.lanes, g_lanes.load());
    DeviceLanes* dl = lanes > 1 ? device_lanes() : nullptr;
    std::unique_lock<std::mutex> lock;
    if (dl) {
        lock = std::unique_lock<std::mutex>(dl->mu);
        cudaEventRecord(dl->fork, st);
        for (int l = 0; l < lanes; ++l) cudaStreamWaitEvent(dl->lane[l], dl->fork, 0);
    }
    engine_error() = 0;
    overlap_launches() = dl == nullptr;      // (CTAs that wait for one chain's next launch would keep the others' off the multiprocessors)
    for (size_t b = 0; b < bt.batches.size() && !engine_error(); ++b) {
        const auto& idx = bt.batches[b];
        ns::Table t{};
        t.count = (int32_t)idx.size();
        for (int k = 0; k < t.count; ++k) {
            const int i = idx[k];
            t.w[k] = ns::Mat{G[i], update ? M[i] : nullptr, X[i], reinterpret_cast<int32_t*>(ws) + i};
        }
        // (lane b % bt.lanes, whose scratch this is, is wholly on one stream)
        run_batch(hs[idx[0]], t, update, ws + status_bytes(count) + bt.off[b], dl ? dl->lane[(b % bt.lanes) % lanes] : st);
    }
    if (dl) {
        for (int l = 0; l < lanes; ++l) {
            cudaEventRecord(dl->done[l], dl->lane[l]);
            cudaStreamWaitEvent(st, dl->done[l], 0);
        }
    }
    return launch_outcome();
}

int run_adamw(const orthdion_adamw_t* hs, int32_t count, void* const* X, float* const* M, float* const* V, const void* const* G,
              int64_t* step, void* stream) {
    if (!hs || !X || !M || !V || !G) return ORTHDION_ERR_NULL;
    if (count < 1) return ORTHDION_ERR_INVALID_ARG;
    int e;
    if ((e = check_ptr(step))) return e;
    for (int i = 0; i < count; ++i) {
        if (!valid(hs[i])) return ORTHDION_ERR_INVALID_ARG;
        if ((e = check_ptr(X[i])) || (e = check_ptr(M[i])) || (e = check_ptr(V[i])) || (e = check_ptr(G[i]))) return e;
    }
    if (twice(X, count) || twice(reinterpret_cast<const void* const*>(M), count) || twice(reinterpret_cast<const void* const*>(V), count))
        return ORTHDION_ERR_INVALID_ARG;

    // one launch per pair of types and table of tensors
    std::vector<adamw::Table> launches;
    std::vector<int> types;
    for (int type = 0; type < 4; ++type) {
        adamw::Table* t = nullptr;
        int kinds = 0;
        for (int i = 0; i < count; ++i) {
            const orthdion_adamw_plan* p = hs[i];
            if ((p->x_dtype == ORTHDION_DTYPE_BF16) + 2 * (p->g_dtype == ORTHDION_DTYPE_BF16) != type) continue;
            const adamw::Kind k{std::log(p->beta1), std::log(p->beta2), (float)p->beta1, (float)(1.0 - p->beta1), (float)p->beta2, (float)(1.0 - p->beta2),
                                p->eps, p->eta, p->wd, 0.f};
            const int64_t chunks = (p->numel + adamw::CHUNK - 1) / adamw::CHUNK;
            if (chunks > (1 << 30)) return ORTHDION_ERR_INVALID_ARG;
            int kind = 0;
            if (t) while (kind < kinds && std::memcmp(&t->kind[kind], &k, sizeof(k)) != 0) ++kind;
            if (!t || t->count == adamw::MAX_TENSORS || kind == adamw::MAX_KINDS || t->chunks + chunks > (1 << 30)) {
                launches.emplace_back();
                types.push_back(type);
                t = &launches.back();
                t->count = 0; t->chunks = 0; t->step = step; t->last = 0;
                std::memset(t->kind, 0, sizeof(t->kind));
                kinds = kind = 0;
            }
            if (kind == kinds) t->kind[kinds++] = k;
            t->t[t->count++] = adamw::Tensor{X[i], M[i], V[i], G[i], p->numel, t->chunks, kind};
            t->chunks += (int32_t)chunks;
        }
    }
    launches.back().last = 1;
    engine_error() = 0;
    overlap_launches() = true;
    for (size_t i = 0; i < launches.size(); ++i) {
        adamw::Table& t = launches[i];
        t.blocks = std::min(t.chunks, 8 * sm_count());
        const dim3 grid((unsigned)t.blocks);
        cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
        switch (types[i]) {
            case 0: launch(adamw::adamw_kernel<false, false>, grid, adamw::THREADS, 0, 1, prof::S_ADAMW, st, t); break;
            case 1: launch(adamw::adamw_kernel<true, false>, grid, adamw::THREADS, 0, 1, prof::S_ADAMW, st, t); break;
            case 2: launch(adamw::adamw_kernel<false, true>, grid, adamw::THREADS, 0, 1, prof::S_ADAMW, st, t); break;
            default: launch(adamw::adamw_kernel<true, true>, grid, adamw::THREADS, 0, 1, prof::S_ADAMW, st, t); break;
        }
        if (engine_error()) break;
    }
    return launch_outcome();
}

// fp32 results show the iteration at full precision: two planes.  bf16 results: one.
void default_passes(orthdion_muon_plan* p) {
    if (!p->passes_set) p->passes = p->x_dtype == ORTHDION_DTYPE_F32 ? 3 : 1;
}

// Whether singular values in [0, 1] stay within what the images hold (entries up to 255): no value above 8 after any step, no
// entry of a I + b A + c A^2 above 128.
bool schedule_ok(int32_t steps, const float* abc) {
    double top = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double a = abc[3 * k], b = abc[3 * k + 1], c = abc[3 * k + 2];
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
        if (std::fabs(a) + std::fabs(b) * top * top + std::fabs(c) * top * top * top * top > 128.0) return false;
        double most = 0.0;
        for (int i = 0; i <= 1024; ++i) {
            const double s = top * i / 1024, s2 = s * s;
            most = std::max(most, std::fabs(s * (a + b * s2 + c * s2 * s2)));
        }
        top = std::max(1e-3, 1.01 * most);
        if (top > 8.0) return false;
    }
    return true;
}

}  // namespace

extern "C" {

int orthdion_muon_create(orthdion_muon_t* out, int64_t m, int64_t n, double mu, float eta, float wd, int32_t nesterov) {
    if (!out) return ORTHDION_ERR_NULL;
    *out = nullptr;
    if (m < 1 || n < 1 || m > (1 << 24) || n > (1 << 24) || std::min(m, n) > 32768) return ORTHDION_ERR_INVALID_ARG;
    if (!(mu >= 0.0 && mu < 1.0) || !std::isfinite(eta) || !std::isfinite(wd) || (nesterov != 0 && nesterov != 1)) return ORTHDION_ERR_INVALID_ARG;
    orthdion_muon_plan* p = new (std::nothrow) orthdion_muon_plan;
    if (!p) return ORTHDION_ERR_MEMORY;
    std::memset(static_cast<void*>(p), 0, sizeof(*p));
    p->magic = kMuonMagic;
    p->m = m; p->n = n;
    p->ld_x = p->ld_m = p->ld_g = n;
    p->mu = mu; p->eta = eta; p->wd = wd; p->scale = 1.f;
    p->nesterov = nesterov;
    p->x_dtype = p->g_dtype = ORTHDION_DTYPE_BF16;
    p->steps = 5;
    p->eps = 1e-7;
    for (int k = 0; k < p->steps; ++k) { p->abc[k][0] = 3.4445f; p->abc[k][1] = -4.7750f; p->abc[k][2] = 2.0315f; }
    default_passes(p);
    *out = p;
    return ORTHDION_OK;
}

int orthdion_muon_destroy(orthdion_muon_t h) {
    if (!valid(h)) return ORTHDION_ERR_INVALID_ARG;
    h->magic = 0;
    delete h;
    return ORTHDION_OK;
}

int orthdion_muon_set_dtypes(orthdion_muon_t h, int32_t x_dtype, int32_t g_dtype) {
    if (!valid(h) || !known(x_dtype) || !known(g_dtype)) return ORTHDION_ERR_INVALID_ARG;
    h->x_dtype = x_dtype; h->g_dtype = g_dtype;
    default_passes(h);
    return ORTHDION_OK;
}

int orthdion_muon_set_lr(orthdion_muon_t h, float eta) {
    if (!valid(h) || !std::isfinite(eta)) return ORTHDION_ERR_INVALID_ARG;
    h->eta = eta;
    return ORTHDION_OK;
}

int orthdion_muon_set_scale(orthdion_muon_t h, float scale) {
    if (!valid(h) || !std::isfinite(scale)) return ORTHDION_ERR_INVALID_ARG;
    h->scale = scale;
    return ORTHDION_OK;
}

int orthdion_muon_set_ld(orthdion_muon_t h, int64_t ld_x, int64_t ld_m, int64_t ld_g) {
    if (!valid(h)) return ORTHDION_ERR_INVALID_ARG;
    for (int64_t ld : {ld_x, ld_m, ld_g})
        if (ld < h->n || ld > ((int64_t)1 << 31)) return ORTHDION_ERR_INVALID_ARG;
    h->ld_x = ld_x; h->ld_m = ld_m; h->ld_g = ld_g;
    return ORTHDION_OK;
}

int orthdion_muon_set_schedule(orthdion_muon_t h, int32_t steps, const float* abc, double eps) {
    if (!valid(h)) return ORTHDION_ERR_INVALID_ARG;
    if (!abc) return ORTHDION_ERR_NULL;
    if (steps < 1 || steps > kMaxSteps || !(eps >= 0.0 && eps <= 1e30) || !schedule_ok(steps, abc)) return ORTHDION_ERR_INVALID_ARG;
    std::memset(h->abc, 0, sizeof(h->abc));
    std::memcpy(h->abc, abc, sizeof(float) * 3 * steps);
    h->steps = steps;
    h->eps = eps;
    return ORTHDION_OK;
}

int orthdion_muon_set_passes(orthdion_muon_t h, int32_t passes) {
    if (!valid(h) || (passes > 0 && passes != 1 && passes != 3)) return ORTHDION_ERR_INVALID_ARG;
    h->passes_set = passes > 0;
    if (passes > 0) h->passes = passes;
    default_passes(h);
    return ORTHDION_OK;
}

size_t orthdion_muon_workspace_bytes_grouped(const orthdion_muon_t* hs, int32_t count) {
    if (!hs || count < 1) return 0;
    for (int i = 0; i < count; ++i)
        if (!valid(hs[i])) return 0;
    return guarded((size_t)0, [&] {
        return status_bytes(count) + make_batches(hs, count).scratch;
    });
}

size_t orthdion_muon_workspace_bytes(orthdion_muon_t h) { return orthdion_muon_workspace_bytes_grouped(&h, 1); }

int orthdion_orthogonalize_grouped(const orthdion_muon_t* hs, int32_t count, const void* const* G, void* const* O, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    return guarded((int)ORTHDION_ERR_MEMORY, [&] { return run_call(hs, count, O, nullptr, G, false, workspace, workspace_bytes, stream); });
}

int orthdion_orthogonalize(orthdion_muon_t h, const void* G, void* O, void* workspace, size_t workspace_bytes, void* stream) {
    return orthdion_orthogonalize_grouped(&h, 1, &G, &O, workspace, workspace_bytes, stream);
}

int orthdion_muon_step_grouped(const orthdion_muon_t* hs, int32_t count, void* const* X, float* const* M, const void* const* G, void* workspace,
                               size_t workspace_bytes, void* stream) {
    return guarded((int)ORTHDION_ERR_MEMORY, [&] { return run_call(hs, count, X, M, G, true, workspace, workspace_bytes, stream); });
}

int orthdion_muon_step(orthdion_muon_t h, void* X, float* M, const void* G, void* workspace, size_t workspace_bytes, void* stream) {
    return orthdion_muon_step_grouped(&h, 1, &X, &M, &G, workspace, workspace_bytes, stream);
}

int orthdion_muon_last_status(int32_t count, const void* workspace, void* stream, int32_t* flags) {
    if (!workspace || !flags) return ORTHDION_ERR_NULL;
    if (count < 1) return ORTHDION_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (cudaMemcpyAsync(flags, workspace, (size_t)count * 4, cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) {
        std::fprintf(stderr, "orthdion: reading the status words failed: %s\n", cudaGetErrorString(cudaGetLastError()));
        return ORTHDION_ERR_CUDA;
    }
    return ORTHDION_OK;
}

int orthdion_adamw_create(orthdion_adamw_t* out, int64_t numel, double beta1, double beta2, float eps, float eta, float wd) {
    if (!out) return ORTHDION_ERR_NULL;
    *out = nullptr;
    if (numel < 1 || numel > ((int64_t)1 << 40)) return ORTHDION_ERR_INVALID_ARG;
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.f) || !std::isfinite(eps) || !std::isfinite(eta) ||
        !std::isfinite(wd))
        return ORTHDION_ERR_INVALID_ARG;
    orthdion_adamw_plan* p = new (std::nothrow) orthdion_adamw_plan();
    if (!p) return ORTHDION_ERR_MEMORY;
    p->magic = kAdamWMagic;
    p->numel = numel;
    p->beta1 = beta1; p->beta2 = beta2; p->eps = eps; p->eta = eta; p->wd = wd;
    p->x_dtype = p->g_dtype = ORTHDION_DTYPE_BF16;
    *out = p;
    return ORTHDION_OK;
}

int orthdion_adamw_destroy(orthdion_adamw_t h) {
    if (!valid(h)) return ORTHDION_ERR_INVALID_ARG;
    h->magic = 0;
    delete h;
    return ORTHDION_OK;
}

int orthdion_adamw_set_dtypes(orthdion_adamw_t h, int32_t x_dtype, int32_t g_dtype) {
    if (!valid(h) || !known(x_dtype) || !known(g_dtype)) return ORTHDION_ERR_INVALID_ARG;
    h->x_dtype = x_dtype; h->g_dtype = g_dtype;
    return ORTHDION_OK;
}

int orthdion_adamw_set_lr(orthdion_adamw_t h, float eta) {
    if (!valid(h) || !std::isfinite(eta)) return ORTHDION_ERR_INVALID_ARG;
    h->eta = eta;
    return ORTHDION_OK;
}

int orthdion_adamw_step_grouped(const orthdion_adamw_t* hs, int32_t count, void* const* X, float* const* M, float* const* V, const void* const* G,
                                int64_t* step, void* stream) {
    return guarded((int)ORTHDION_ERR_MEMORY, [&] { return run_adamw(hs, count, X, M, V, G, step, stream); });
}

int orthdion_adamw_step(orthdion_adamw_t h, void* X, float* M, float* V, const void* G, int64_t* step, void* stream) {
    return orthdion_adamw_step_grouped(&h, 1, &X, &M, &V, &G, step, stream);
}

}  // extern "C"
