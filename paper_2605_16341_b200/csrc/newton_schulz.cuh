// Newton-Schulz orthogonalisation on tcgen05: X <- a X + (b A + c A^2) X with A = X X^T (X^T X where the matrix is
// taller than wide), a few times over, from X = B / (|B| + eps).
//
// Operands.  The iterate and the products of the smaller side s live in scratch as fp16 images: row-major, 256 times
// the value (so that entries of 1 / s^1.5 are no subnormals and entries of 64 do not overflow), one plane (11 bits), or two
// planes v = t0 + t1 with t1 = fp16(v - t0) (22 bits; products t0 u0 + t0 u1 + t1 u0).  bf16 planes would cost the same and hold
// 8 bits: 8 times the error, 1 to 3 % of the result.  TMA loads swizzle 64-column boxes of an image into shared memory, which serve as
// K-major tiles (depth along the columns) or MN-major tiles (depth along the rows), so nothing is ever transposed.
//
// Sums are fp32, in tensor memory.  The tensor core truncates as it adds, which lowers a long sum of squares by about 5e-9 of it
// per term: two-plane products are summed over 64 terms at a time there, the small products first, and beyond that by the epilogue, in
// registers (256 x 512 in fp32: error of the result 1.3e-5 with 256 terms at a time, 3.1e-6 with 64; the plain form in fp32 has 2e-6).
#pragma once
#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"
#include "launch.cuh"
#include "tcgen05.cuh"

namespace od {
namespace ns {

using namespace od::tc;

constexpr float UNIT = 256.f;            // images hold UNIT times the value
constexpr int MAX_BATCH = 64;            // matrices of one launch (its table: 2 KB of kernel parameters)
constexpr int MAX_PARTS = 512;           // partial sums of squares of one matrix

// The caller's buffers of one matrix.
struct Mat {
    const void* G;
    float* M;          // momentum; null: B = G
    void* X;           // weights to update, or where the result goes
    int32_t* status;
};
struct Table {
    int32_t count, pad;
    Mat w[MAX_BATCH];
};
// What the launches of a batch hand on, per matrix.
struct Slot {
    float sigma;       // UNIT / (stored |X0| + stored eps): how much larger the normalised matrix is than the stored one
    int32_t status;
    int32_t pad[2];
};

// ---- the buffer B, its norm, its image ---------------------------------------------------------
struct PrepArgs {
    int64_t rows, cols, ld_g, ld_m;
    int32_t g_bf16, nesterov;
    float mu, rest;              // momentum, 1 - momentum
    double eps;
    int32_t parts, terms;
    int32_t vec;                 // rows start on 16-byte boundaries
    double* part;                // [matrix][MAX_PARTS]
    Slot* slot;
    __half* img;
    int64_t pitch, term_stride, mat_stride;      // of the image, in elements
};

// 8 entries of B at (row, col) and of the updated momentum; entries beyond the last column are zeros.
__device__ __forceinline__ void load_buffer(const Mat& w, const PrepArgs& a, int64_t row, int64_t col, float (&b)[8], float (&m)[8]) {
    const int64_t gi = row * a.ld_g + col, mi = row * a.ld_m + col;
    float g[8];
    if (a.vec) {
        if (a.g_bf16) {
            const uint4 u = *reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(w.G) + gi);
            g[0] = bf16lo_to_f32(u.x); g[1] = bf16hi_to_f32(u.x); g[2] = bf16lo_to_f32(u.y); g[3] = bf16hi_to_f32(u.y);
            g[4] = bf16lo_to_f32(u.z); g[5] = bf16hi_to_f32(u.z); g[6] = bf16lo_to_f32(u.w); g[7] = bf16hi_to_f32(u.w);
        } else {
            const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(w.G) + gi);
            const float4 x = p[0], y = p[1];
            g[0] = x.x; g[1] = x.y; g[2] = x.z; g[3] = x.w; g[4] = y.x; g[5] = y.y; g[6] = y.z; g[7] = y.w;
        }
        if (w.M) {
            const float4* p = reinterpret_cast<const float4*>(w.M + mi);
            const float4 x = p[0], y = p[1];
            m[0] = x.x; m[1] = x.y; m[2] = x.z; m[3] = x.w; m[4] = y.x; m[5] = y.y; m[6] = y.z; m[7] = y.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool in = col + e < a.cols;
            g[e] = !in ? 0.f : a.g_bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(w.G)[gi + e])
                                        : reinterpret_cast<const float*>(w.G)[gi + e];
            m[e] = in && w.M ? w.M[mi + e] : 0.f;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (!w.M) { b[e] = g[e]; continue; }
        // (the same instructions wherever B is formed: the same bits)
        m[e] = __fmaf_rn(a.mu, m[e], __fmul_rn(a.rest, g[e]));
        b[e] = a.nesterov ? __fmaf_rn(a.mu, m[e], __fmul_rn(a.rest, g[e])) : m[e];
    }
}

// Walks the 8-column chunks of the matrix that this block takes of `blocks`.
template <class F>
__device__ __forceinline__ void for_chunks(const PrepArgs& a, int block, int blocks, F f) {
    const int64_t cpr = (a.cols + 7) / 8, total = cpr * a.rows, step = (int64_t)blocks * blockDim.x;
    int64_t i = (int64_t)block * blockDim.x + threadIdx.x;
    int64_t row = i / cpr, c = i - row * cpr;
    const int64_t drow = step / cpr, dc = step - drow * cpr;
    for (; i < total; i += step) {
        f(row, c * 8);
        row += drow; c += dc;
        if (c >= cpr) { c -= cpr; ++row; }
    }
}

__device__ __forceinline__ double block_sum(double v, double* red) {
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0.0;
    for (int i = 0; i < (int)blockDim.x / 32; ++i) v += red[i];
    return v;
}

// Sums of squares of B, one per block, in 64 bits (a sum over up to 10^8 entries, and squares of any finite entry).
__global__ void __launch_bounds__(256) norm_kernel(const __grid_constant__ Table t, const __grid_constant__ PrepArgs a) {
    __shared__ double red[8];
    grid_dependency();
    const Mat& w = t.w[blockIdx.y];
    double sum = 0.0;
    for_chunks(a, blockIdx.x, a.parts, [&](int64_t row, int64_t col) {
        float b[8], m[8];
        load_buffer(w, a, row, col, b, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fma((double)b[e], (double)b[e], sum);
    });
    sum = block_sum(sum, red);
    if (threadIdx.x == 0) a.part[(int64_t)blockIdx.y * MAX_PARTS + blockIdx.x] = sum;
}

// The image of B, scaled by the power of two that brings its norm to [128, 256) (a gradient in bf16 is then held exactly; what is left
// of the normalisation, sigma, goes into the factors of the first products), and the updated momentum.  A matrix whose norm is
// not finite keeps its momentum.
__global__ void __launch_bounds__(256) prep_kernel(const __grid_constant__ Table t, const __grid_constant__ PrepArgs a) {
    __shared__ double red[8];
    grid_dependency();
    const Mat& w = t.w[blockIdx.y];
    double sum = 0.0;
    for (int i = threadIdx.x; i < a.parts; i += blockDim.x) sum += a.part[(int64_t)blockIdx.y * MAX_PARTS + i];
    sum = block_sum(sum, red);
    const double norm = sqrt(sum);
    const bool finite = norm <= 1.7e308;
    int e = 0;
    if (finite && norm > 0.0) frexp(norm, &e);
    const int k = finite && norm > 0.0 ? 8 - e : 0;
    // (the power itself may be beyond fp32, so two factors)
    const float f1 = ldexpf(1.f, k / 2), f2 = ldexpf(1.f, k - k / 2);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        Slot s{};
        s.sigma = finite && norm > 0.0 ? (float)((double)UNIT / ldexp(norm + a.eps, k)) : 0.f;
        s.status = finite ? 0 : ST_NONFINITE;
        a.slot[blockIdx.y] = s;
        *w.status = s.status;
    }
    if (!finite) return;
    __half* img = a.img + (int64_t)blockIdx.y * a.mat_stride;
    for_chunks(a, blockIdx.x, gridDim.x, [&](int64_t row, int64_t col) {
        float b[8], m[8];
        load_buffer(w, a, row, col, b, m);
        if (w.M) {
            float* dst = w.M + row * a.ld_m + col;
            if (a.vec) {
                reinterpret_cast<float4*>(dst)[0] = make_float4(m[0], m[1], m[2], m[3]);
                reinterpret_cast<float4*>(dst)[1] = make_float4(m[4], m[5], m[6], m[7]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (col + i < a.cols) dst[i] = m[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = b[i] * f1 * f2;
        __half* dst = img + row * a.pitch + col;
        const uint4 hi = half8(b, 1.f);
        *reinterpret_cast<uint4*>(dst) = hi;
        if (a.terms == 2) {
            const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
                b[2 * i] -= v.x; b[2 * i + 1] -= v.y;
            }
            *reinterpret_cast<uint4*>(dst + a.term_stride) = half8(b, 1.f);
        }
    });
}

// ---- products between images ---------------------------------------------------------------------
// D = alpha sigma^p (A B^T) + beta C + diag I, with A rows x depth, B cols x depth.
enum Epi : int { EPI_IMAGE = 0, EPI_FINAL = 1 };

constexpr int STAGE_BYTES = 196608;           // operand ring
constexpr int THREADS = 32 * 10;              // producer, issuer, eight epilogue warps
constexpr int MAX_STAGES = 8;
constexpr int GROUP_ROWS = 8;                 // tile rows that are walked together, column by column

struct GemmArgs {
    int32_t rows, cols, kblocks, chunk;       // chunk: depth blocks that are summed in tensor memory
    int32_t m_tiles, n_tiles, tiles, total;   // tiles: of one matrix
    int32_t sym;                              // symmetric result: tiles on and below the diagonal, mirrored
    int32_t a_mn, b_mn;                       // 1: depth runs along the rows of the image
    int32_t sigma_pow;
    float alpha, beta, diag;
    __half* out;                              // image of the result ...
    const __half* add;                        // ... and of C, laid out alike; null: D = alpha sigma^p (A B^T)
    int64_t pitch, term_stride, mat_stride;
    Slot* slot;
    int32_t count;
    int32_t update, x_bf16;                   // EPI_FINAL: X <- wc X - wd D, or X <- D
    float wc, wd;
    int64_t ld_x;
    alignas(64) CUtensorMap map_a;
    alignas(64) CUtensorMap map_b;
    alignas(64) CUtensorMap map_out;
};
struct NoTable { int32_t unused; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_float(float v) {
    if constexpr (sizeof(T) == 2) return __float2bfloat16_rn(v);
    else return v;
}

__device__ __forceinline__ void tma_load4(uint32_t dst, const CUtensorMap* map, int x, int row, int term, int mat, uint32_t bar, bool pair) {
    if (pair)
        asm volatile(
            "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
            ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(row), "r"(term), "r"(mat), "r"(bar) : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
            ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(row), "r"(term), "r"(mat), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_store4(const CUtensorMap* map, uint32_t src, int x, int row, int term, int mat) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(src), "r"(x), "r"(row), "r"(term), "r"(mat) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr) : "memory");
}

// Rows of a result tile, and rows of B that one CTA holds of it.
template <bool PAIR> __host__ __device__ constexpr int tile_rows() { return PAIR ? 256 : 128; }
template <bool PAIR, int BN> __host__ __device__ constexpr int side_rows() { return PAIR ? BN / 2 : BN; }
template <bool PAIR, int BN, int TERMS> __host__ __device__ constexpr int stage_bytes() { return (128 + side_rows<PAIR, BN>()) * 128 * TERMS; }
template <bool PAIR, int BN, int TERMS> __host__ __device__ constexpr int stages() {
    constexpr int n = STAGE_BYTES / stage_bytes<PAIR, BN, TERMS>();
    return n < MAX_STAGES ? n : MAX_STAGES;
}
constexpr int SMEM_BYTES = 1024 + STAGE_BYTES + 8 * 4096 + 256;

struct Tile { int mat, row0, col0; bool active, mirror; };

template <bool PAIR, int BN>
__device__ __forceinline__ Tile decode(const GemmArgs& g, int t) {
    constexpr int TM = tile_rows<PAIR>();
    Tile r;
    r.mat = t / g.tiles;
    t -= r.mat * g.tiles;
    int i, j;
    if (g.sym) {
        // tiles before tile row i: i (i + 1) / 2 of square tiles, i (i + 1) of tiles half as wide as high
        constexpr int Q = TM / BN;
        i = Q == 1 ? (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f) : (int)((sqrtf(4.f * t + 1.f) - 1.f) * 0.5f);
        auto before = [](int k) { return Q == 1 ? k * (k + 1) / 2 : k * (k + 1); };
        while (before(i) > t) --i;
        while (before(i + 1) <= t) ++i;
        j = t - before(i);
    } else {
        const int per = GROUP_ROWS * g.n_tiles, grp = t / per;
        const int first = grp * GROUP_ROWS, high = min(GROUP_ROWS, g.m_tiles - first);
        const int in = t - grp * per;
        j = in / high;
        i = first + in - j * high;
    }
    r.row0 = i * TM; r.col0 = j * BN;
    r.active = r.col0 < g.cols;
    r.mirror = g.sym && r.col0 + BN <= r.row0;
    return r;
}

template <bool PAIR, int BN, int TERMS, int EPI, class TABLE>
__global__ void __launch_bounds__(THREADS, 1) gemm_kernel(const __grid_constant__ TABLE table, const __grid_constant__ GemmArgs g) {
    constexpr int NB = side_rows<PAIR, BN>(), STAGE = stage_bytes<PAIR, BN, TERMS>(), NS = stages<PAIR, BN, TERMS>();
    constexpr int A_BYTES = 128 * 128 * TERMS;
    constexpr int NC = BN / 2;                       // columns of one epilogue warp
    constexpr uint32_t NCTA = PAIR ? 2 : 1;
    const int crank = PAIR ? (int)cluster_ctarank() : 0;
    const int tile0 = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x, tstep = PAIR ? (int)(gridDim.x >> 1) : (int)gridDim.x;

    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    unsigned char* smem = smem_raw + (base - raw);
    const uint32_t staging0 = base + STAGE_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + STAGE_BYTES + 8 * 4096);
    const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * MAX_STAGES, tfull0 = empty0 + 8 * MAX_STAGES, tempty0 = tfull0 + 16;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * MAX_STAGES + 4);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    if (threadIdx.x == 0) {
        for (int s = 0; s < NS; ++s) { mbar_init(full0 + 8 * s, NCTA); mbar_init(empty0 + 8 * s, 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(tfull0 + 8 * a, 1); mbar_init(tempty0 + 8 * a, NCTA * 8); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
        prefetch_tensor_map(&g.map_a);
        prefetch_tensor_map(&g.map_b);
        if (EPI == EPI_IMAGE) prefetch_tensor_map(&g.map_out);
    }
    if (warp == 1) {
        if (PAIR) tmem_alloc_pair(smem_u32(tmem_slot), 2 * BN);
        else tmem_alloc(smem_u32(tmem_slot), 2 * BN);
    }
    grid_dependency_launch();
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();       // the peer's barriers are initialised before anything reaches them
    tc_fence_after();
    grid_dependency_wait();
    const uint32_t tmem_base = *tmem_slot;
    const uint32_t full_ld = PAIR ? map_to_rank(full0, 0) : full0, tempty_ld = PAIR ? map_to_rank(tempty0, 0) : tempty0;

    if (warp == 0) {
        // ---------------- producer: this CTA's rows of A and of B, both planes of a 64-deep block per stage ----------------
        if (lane == 0) {
            int s = 0; uint32_t ph = 0;
            bool ok = true;
            for (int t = tile0; t < g.total && ok; t += tstep) {
                const Tile c = decode<PAIR, BN>(g, t);
                if (!c.active) continue;
                const int ar = c.row0 + crank * 128, br = c.col0 + crank * NB;
                for (int kb = 0; kb < g.kblocks; ++kb) {
                    if (!mbar_wait(empty0 + 8 * s, ph ^ 1, abort_flag)) { ok = false; break; }
                    const uint32_t fb = full_ld + 8 * s, dst = base + s * STAGE;
                    if (PAIR) mbar_arrive_expect_tx_remote(fb, STAGE);
                    else mbar_arrive_expect_tx(fb, STAGE);
                    if (g.a_mn) {
                        tma_load4(dst, &g.map_a, ar, kb * 64, 0, c.mat, fb, PAIR);
                        tma_load4(dst + 8192 * TERMS, &g.map_a, ar + 64, kb * 64, 0, c.mat, fb, PAIR);
                    } else {
                        tma_load4(dst, &g.map_a, kb * 64, ar, 0, c.mat, fb, PAIR);
                    }
                    if (g.b_mn) {
#pragma unroll
                        for (int q = 0; q < NB / 64; ++q)
                            tma_load4(dst + A_BYTES + q * 8192 * TERMS, &g.map_b, br + q * 64, kb * 64, 0, c.mat, fb, PAIR);
                    } else {
                        tma_load4(dst + A_BYTES, &g.map_b, kb * 64, br, 0, c.mat, fb, PAIR);
                    }
                    if (++s == NS) { s = 0; ph ^= 1; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (lane == 0 && crank == 0) {
            const uint32_t a_step = g.a_mn ? (2048u >> 4) : (32u >> 4), b_step = g.b_mn ? (2048u >> 4) : (32u >> 4);     // one 16-deep slice
            const uint32_t a_term = g.a_mn ? (8192u >> 4) : (16384u >> 4), b_term = g.b_mn ? (8192u >> 4) : (uint32_t)(NB * 128) >> 4;
            const uint64_t a_desc = g.a_mn ? smem_desc(0, 8192 * TERMS, 1024) : smem_desc(0, 16, 1024);
            const uint64_t b_desc = g.b_mn ? smem_desc(0, 8192 * TERMS, 1024) : smem_desc(0, 16, 1024);
            const uint32_t a_hi = (uint32_t)(a_desc >> 32), b_hi = (uint32_t)(b_desc >> 32);
            const uint32_t a0 = (uint32_t)a_desc + (base >> 4), b0 = (uint32_t)b_desc + ((base + A_BYTES) >> 4);
            const uint32_t idesc = instr_desc(BN, g.a_mn, g.b_mn, 0u, PAIR ? 256u : 128u);
            int s = 0, acc = 0; uint32_t ph = 0, aph = 0;
            bool ok = true;
            for (int t = tile0; t < g.total && ok; t += tstep) {
                if (!decode<PAIR, BN>(g, t).active) continue;
                for (int k0 = 0; k0 < g.kblocks && ok; k0 += g.chunk) {
                    if (!mbar_wait(tempty0 + 8 * acc, aph ^ 1, abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d = tmem_base + acc * BN;
                    const int k1 = min(g.kblocks, k0 + g.chunk);
                    for (int kb = k0; kb < k1; ++kb) {
                        if (!mbar_wait(full0 + 8 * s, ph, abort_flag)) { ok = false; break; }
                        const uint32_t off = (uint32_t)(s * STAGE) >> 4;
                        if (TERMS == 2) {
                            // the small products first: an addition truncates at the accumulator's size of the moment
                            umma_slices<PAIR, 4, false>(d, a0 + off, a_hi, b0 + off + b_term, b_hi, a_step, b_step, 0, 0, idesc, kb > k0 ? 1u : 0u);
                            umma_slices<PAIR, 4, false>(d, a0 + off + a_term, a_hi, b0 + off, b_hi, a_step, b_step, 0, 0, idesc, 1u);
                            umma_slices<PAIR, 4, false>(d, a0 + off, a_hi, b0 + off, b_hi, a_step, b_step, 0, 0, idesc, 1u);
                        } else {
                            umma_slices<PAIR, 4, false>(d, a0 + off, a_hi, b0 + off, b_hi, a_step, b_step, 0, 0, idesc, kb > k0 ? 1u : 0u);
                        }
                        commit_any<PAIR>(empty0 + 8 * s);
                        if (++s == NS) { s = 0; ph ^= 1; }
                    }
                    if (!ok) break;
                    commit_any<PAIR>(tfull0 + 8 * acc);
                    if (++acc == 2) { acc = 0; aph ^= 1; }
                }
            }
        }
        __syncwarp();
    } else {
        // ---------------- epilogue: warp w has the 32 rows that its tensor-memory quarter holds, and half the columns ----------------
        const int quarter = warp % 4, half = (warp - 2) / 4;
        const uint32_t staging = staging0 + (uint32_t)(warp - 2) * 4096u;
        unsigned char* stage_ptr = smem + STAGE_BYTES + (warp - 2) * 4096;
        int acc = 0; uint32_t aph = 0;
        bool ok = true;
        for (int t = tile0; t < g.total && ok; t += tstep) {
            const Tile c = decode<PAIR, BN>(g, t);
            if (!c.active) continue;
            float v[NC];
            for (int k0 = 0; k0 < g.kblocks; k0 += g.chunk) {
                // (all lanes alike: a wait that ran out for one ends the warp's work)
                ok = __all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * acc, aph, abort_flag));
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem_base + acc * BN + half * NC + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
                for (int q = 0; q < NC / 16; ++q) {
                    uint32_t u[16];
                    tmem_ld16(d + q * 16, u);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[q * 16 + e] = (TERMS == 2 && k0 > 0) ? v[q * 16 + e] + __uint_as_float(u[e]) : __uint_as_float(u[e]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) { if (PAIR) mbar_arrive_remote(tempty_ld + 8 * acc); else mbar_arrive(tempty0 + 8 * acc); }
                if (++acc == 2) { acc = 0; aph ^= 1; }
            }
            if (!ok) break;
            const int row_w = c.row0 + crank * 128 + quarter * 32, row = row_w + lane;
            const int col_w = c.col0 + half * NC;
            float alpha = g.alpha;
            if (g.sigma_pow) {
                const float sg = g.slot[c.mat].sigma;
                alpha *= g.sigma_pow == 2 ? sg * sg : sg;
            }
            if (row_w >= g.rows) continue;
            if constexpr (EPI == EPI_IMAGE) {
#pragma unroll
                for (int q = 0; q < NC / 64; ++q) {
                    const int col = col_w + q * 64;
                    if (col < g.cols) {
#pragma unroll
                        for (int e = 0; e < 64; ++e) v[q * 64 + e] *= alpha;
                        if (g.add) {
                            if (row < g.rows) {
                                const __half* src = g.add + c.mat * g.mat_stride + (int64_t)row * g.pitch + col;
#pragma unroll
                                for (int term = 0; term < TERMS; ++term)
#pragma unroll
                                    for (int e = 0; e < 64; e += 8) {
                                        const uint4 u = *reinterpret_cast<const uint4*>(src + term * g.term_stride + e);
                                        const uint32_t h[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                                        for (int i = 0; i < 4; ++i) {
                                            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
                                            v[q * 64 + e + 2 * i] += g.beta * f.x;
                                            v[q * 64 + e + 2 * i + 1] += g.beta * f.y;
                                        }
                                    }
                            }
                            if (col + 64 > row_w && col < row_w + 32) {
#pragma unroll
                                for (int e = 0; e < 64; ++e) v[q * 64 + e] += col + e == row ? g.diag : 0.f;
                            }
                        }
#pragma unroll
                        for (int term = 0; term < TERMS; ++term) {
                            bulk_wait_read();
                            __syncwarp();
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                uint32_t h[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    float &x = v[q * 64 + i * 8 + 2 * k], &y = v[q * 64 + i * 8 + 2 * k + 1];
                                    h[k] = pack_f16x2(x, y);
                                    if (c.mirror) {
                                        __half* m = g.out + c.mat * g.mat_stride + term * g.term_stride + (int64_t)(col + i * 8 + 2 * k) * g.pitch + row;
                                        const __half2 hh = *reinterpret_cast<const __half2*>(&h[k]);
                                        if (row < g.rows) {
                                            if (col + i * 8 + 2 * k < g.cols) m[0] = __low2half(hh);
                                            if (col + i * 8 + 2 * k + 1 < g.cols) m[g.pitch] = __high2half(hh);
                                        }
                                    }
                                    if (TERMS == 2 && term == 0) {
                                        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[k]));
                                        x -= f.x; y -= f.y;
                                    }
                                }
                                *reinterpret_cast<uint4*>(stage_ptr + lane * 128 + ((i ^ (lane & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
                            }
                            fence_async_smem();
                            __syncwarp();
                            if (lane == 0) tma_store4(&g.map_out, staging, col, row_w, term, c.mat);
                        }
                    }
                }
            } else {
                const Mat& w = table.w[c.mat];
                if (g.slot[c.mat].status) continue;
                float* blk = reinterpret_cast<float*>(stage_ptr);
#pragma unroll
                for (int q = 0; q < NC / 32; ++q) {
                    const int col = col_w + q * 32;
                    if (col < g.cols) {
                        // through shared memory, so that the lanes run along a row
#pragma unroll
                        for (int e = 0; e < 32; ++e) blk[lane * 32 + (e ^ lane)] = v[q * 32 + e] * alpha;
                        __syncwarp();
                        const int cl = col + lane, high = min(32, g.rows - row_w);
                        if (cl < g.cols) {
                            const int64_t at = (int64_t)row_w * g.ld_x + cl;
                            auto rows16 = [&](auto* x) {
                                using T = std::remove_pointer_t<decltype(x)>;
                                // (sixteen loads under way: stores to X in between would hold each of them back)
#pragma unroll 1
                                for (int r0 = 0; r0 < high; r0 += 16) {
                                    float old[16];
                                    if (g.update) {
#pragma unroll
                                        for (int r = 0; r < 16; ++r) old[r] = r0 + r < high ? to_float(x[(r0 + r) * g.ld_x]) : 0.f;
                                    }
#pragma unroll
                                    for (int r = 0; r < 16; ++r) {
                                        const float d = blk[(r0 + r) * 32 + (lane ^ (r0 + r))];
                                        if (r0 + r < high) x[(r0 + r) * g.ld_x] = from_float<T>(g.update ? g.wc * old[r] - g.wd * d : d);
                                    }
                                }
                            };
                            if (g.x_bf16) rows16(reinterpret_cast<__nv_bfloat16*>(w.X) + at);
                            else rows16(reinterpret_cast<float*>(w.X) + at);
                        }
                        __syncwarp();
                    }
                }
            }
        }
        if (EPI == EPI_IMAGE) bulk_wait();
    }

    // ---------------- teardown ----------------
    // A role that gave up on a bounded wait leaves copies and MMAs possibly still in flight: a pause far longer than any of them
    // takes lets them land before shared and tensor memory are given back.
    if (*abort_flag) {
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000LL) {}
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();
    tc_fence_after();
    if (threadIdx.x == 0) {
        if (*abort_flag)
            for (int i = 0; i < g.count; ++i) atomicOr(&g.slot[i].status, ST_WAIT);
        if constexpr (EPI == EPI_FINAL) {
            if (*abort_flag || blockIdx.x == 0)
                for (int i = 0; i < g.count; ++i) {
                    const int st = *abort_flag ? ST_WAIT : g.slot[i].status;
                    if (st) atomicOr(table.w[i].status, st);
                }
        }
    }
    if (warp == 1) {
        if (PAIR) tmem_dealloc_pair(tmem_base, 2 * BN);
        else tmem_dealloc(tmem_base, 2 * BN);
    }
}

}  // namespace ns
}  // namespace od
