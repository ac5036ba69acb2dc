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

// 8 entries of G and M at (row, col) as they lie in memory; zeros beyond the last column.
struct Raw { uint4 g[2], m[2]; };
template <bool VEC>
__device__ __forceinline__ void load_raw(const Mat& w, const PrepArgs& a, int64_t row, int64_t col, Raw& r) {
    const int64_t gi = row * a.ld_g + col, mi = row * a.ld_m + col;
    if (VEC) {
        if (a.g_bf16) {
            r.g[0] = *reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(w.G) + gi);
        } else {
            const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(w.G) + gi);
            r.g[0] = p[0]; r.g[1] = p[1];
        }
        if (w.M) {
            const uint4* p = reinterpret_cast<const uint4*>(w.M + mi);
            r.m[0] = p[0]; r.m[1] = p[1];
        }
    } else {
        uint32_t* gw = reinterpret_cast<uint32_t*>(r.g);
        uint32_t* mw = reinterpret_cast<uint32_t*>(r.m);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool in = col + e < a.cols;
            if (a.g_bf16) {
                const uint32_t v = in ? reinterpret_cast<const uint16_t*>(w.G)[gi + e] : 0u;
                if (e % 2) gw[e / 2] |= v << 16;
                else gw[e / 2] = v;
            } else {
                gw[e] = in ? reinterpret_cast<const uint32_t*>(w.G)[gi + e] : 0u;
            }
            if (w.M) mw[e] = in ? reinterpret_cast<const uint32_t*>(w.M)[mi + e] : 0u;
        }
    }
}
// Those 8 entries of B, and of the updated momentum.
__device__ __forceinline__ void buffer_of(const Raw& r, const PrepArgs& a, bool momentum, float (&b)[8], float (&m)[8]) {
    const uint32_t gw[8] = {r.g[0].x, r.g[0].y, r.g[0].z, r.g[0].w, r.g[1].x, r.g[1].y, r.g[1].z, r.g[1].w};
    const uint32_t mw[8] = {r.m[0].x, r.m[0].y, r.m[0].z, r.m[0].w, r.m[1].x, r.m[1].y, r.m[1].z, r.m[1].w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float g = a.g_bf16 ? (e % 2 ? bf16hi_to_f32(gw[e / 2]) : bf16lo_to_f32(gw[e / 2])) : __uint_as_float(gw[e]);
        if (!momentum) { b[e] = g; continue; }
        // (the same instructions wherever B is formed: the same bits)
        m[e] = __fmaf_rn(a.mu, __uint_as_float(mw[e]), __fmul_rn(a.rest, g));
        b[e] = a.nesterov ? __fmaf_rn(a.mu, m[e], __fmul_rn(a.rest, g)) : m[e];
    }
}

// Walks the 8-column chunks of the matrix that this block takes of `blocks`, U of them loaded before the first is used (one at a time:
// 16 us for a sweep over a 4096 x 4096 bf16 matrix).
template <int U, bool VEC, class F>
__device__ __forceinline__ void for_chunks(const Mat& w, const PrepArgs& a, int block, int blocks, F f) {
    const int64_t cpr = (a.cols + 7) / 8, total = cpr * a.rows, step = (int64_t)blocks * blockDim.x;
    int64_t i = (int64_t)block * blockDim.x + threadIdx.x;
    int64_t row = i / cpr, c = i - row * cpr;
    const int64_t drow = step / cpr, dc = step - drow * cpr;
    while (i < total) {
        Raw r[U];
        int64_t rows[U], cols[U];
        int n = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i < total) {
                rows[u] = row; cols[u] = c * 8;
                load_raw<VEC>(w, a, row, c * 8, r[u]);
                n = u + 1;
            }
            i += step; row += drow; c += dc;
            if (c >= cpr) { c -= cpr; ++row; }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < n) f(r[u], rows[u], cols[u]);
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
    auto add = [&](const Raw& r, int64_t, int64_t) {
        float b[8], m[8];
        buffer_of(r, a, w.M != nullptr, b, m);
        // eight squares in 32 bits (2^-22 of them at most), unless they overflow or come near what vanishes
        float q = b[0] * b[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) q = fmaf(b[e], b[e], q);
        if (q >= 1e-28f && q <= 1e38f) {
            sum += (double)q;
        } else {
#pragma unroll 1
            for (int e = 0; e < 8; ++e) sum = fma((double)b[e], (double)b[e], sum);
        }
    };
    if (a.vec) for_chunks<4, true>(w, a, blockIdx.x, a.parts, add);
    else for_chunks<2, false>(w, a, blockIdx.x, a.parts, add);
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
    auto write = [&](const Raw& r, int64_t row, int64_t col) {
        float b[8], m[8];
        buffer_of(r, a, w.M != nullptr, b, m);
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
    };
    if (a.vec) for_chunks<4, true>(w, a, blockIdx.x, gridDim.x, write);
    else for_chunks<2, false>(w, a, blockIdx.x, gridDim.x, write);
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
    int32_t update, x_bf16, x_vec;            // EPI_FINAL: X <- wc X - wd D, or X <- D; x_vec: rows of X on 16-byte boundaries, and whole vectors
    float wc, wd;
    int64_t ld_x;
    alignas(64) CUtensorMap map_a;
    alignas(64) CUtensorMap map_b;
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
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]),
          "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

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

// The rows of one warp (row_w + lane) and NC columns from col_w of a result in tensor memory at d -> image, 32 columns at a time,
// through shared memory so that four lanes write 64 bytes of a row; with `mirror` also to the mirrored place, where pairs of rows and
// columns are exchanged between neighbouring lanes first.  (With TMA stores out of two such blocks in turn a block took 1200 cycles,
// most of them the wait until the one before was read, and its mirror image in 4-byte stores as long again.)
template <int TERMS, int NC>
__device__ __forceinline__ void image_epilogue(const GemmArgs& g, uint32_t d, float alpha, int mat, int row_w, int lane, int col_w, bool mirror,
                                               unsigned char* stage_ptr) {
    const int row = row_w + lane;
    const int64_t base = mat * g.mat_stride;
    const __half* add = g.add ? g.add + base + (int64_t)min(row, g.rows - 1) * g.pitch : nullptr;
    const int sr = lane / 4, sc = lane % 4;              // row and 16-byte chunk that this lane moves out
    const bool odd = lane & 1;
    unsigned char* mir_ptr = stage_ptr + 2048;
    uint4 cq[TERMS][4];
    auto fetch = [&](int col) {
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) cq[t][i] = *reinterpret_cast<const uint4*>(add + t * g.term_stride + col + i * 8);
    };
    if (add) fetch(col_w);
#pragma unroll 1
    for (int q = 0; q < NC / 32; ++q) {
        const int col = col_w + q * 32;
        if (col >= g.cols) break;
        float v[32];
        {
            uint32_t u[32];
            tmem_ld32(d + q * 32, u);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = alpha * __uint_as_float(u[e]);
        }
        if (add) {
#pragma unroll
            for (int t = 0; t < TERMS; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t h[4] = {cq[t][i].x, cq[t][i].y, cq[t][i].z, cq[t][i].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[k]));
                        v[i * 8 + 2 * k] = fmaf(g.beta, f.x, v[i * 8 + 2 * k]);
                        v[i * 8 + 2 * k + 1] = fmaf(g.beta, f.y, v[i * 8 + 2 * k + 1]);
                    }
                }
            if (col == row_w) {          // the block on the diagonal
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] += e == lane ? g.diag : 0.f;
            }
            if (q + 1 < NC / 32 && col + 32 < g.cols) fetch(col + 32);
        }
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t h[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float &x = v[i * 8 + 2 * k], &y = v[i * 8 + 2 * k + 1];
                    h[k] = pack_f16x2(x, y);
                    if (TERMS == 2 && t == 0) {
                        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[k]));
                        x -= f.x; y -= f.y;
                    }
                    if (mirror) {
                        // an even lane gets its neighbour's entry of the first column, an odd one that of the second
                        const uint32_t o = __shfl_xor_sync(0xffffffffu, h[k], 1);
                        *reinterpret_cast<uint32_t*>(mir_ptr + (i * 8 + 2 * k + odd) * 64 + (lane - odd) * 2) =
                            odd ? __byte_perm(o, h[k], 0x7632) : __byte_perm(h[k], o, 0x5410);
                    }
                }
                *reinterpret_cast<uint4*>(stage_ptr + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
            }
            __syncwarp();
            __half* out = g.out + base + t * g.term_stride;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = sr + 8 * i;
                if (row_w + r < g.rows && col + sc * 8 < g.cols)
                    *reinterpret_cast<uint4*>(out + (int64_t)(row_w + r) * g.pitch + col + sc * 8) =
                        *reinterpret_cast<const uint4*>(stage_ptr + r * 64 + ((sc ^ ((r >> 1) & 3)) << 4));
                if (mirror && col + r < g.cols && row_w + sc * 8 < g.rows)
                    *reinterpret_cast<uint4*>(out + (int64_t)(col + r) * g.pitch + row_w + sc * 8) = *reinterpret_cast<const uint4*>(mir_ptr + r * 64 + sc * 16);
            }
        }
    }
}

// The same rows and columns -> the caller's matrix, along rows: 8 entries a lane where rows start on 16-byte boundaries.
template <class T, int NC>
__device__ __forceinline__ void final_epilogue(const GemmArgs& g, uint32_t d, float alpha, void* X, int row_w, int lane, int col_w, unsigned char* stage_ptr) {
    float* blk = reinterpret_cast<float*>(stage_ptr);
    const int high = min(32, g.rows - row_w);
    constexpr int V = 16 / sizeof(T), PER = 32 / V, STEP = 32 / PER;      // entries a lane takes, lanes a row, rows a turn
    const int vr = lane / PER, vc = (lane % PER) * V;
    uint4 old[32 / STEP];
    auto fetch = [&](int col) {
#pragma unroll
        for (int i = 0; i < 32 / STEP; ++i) {
            const int r = vr + i * STEP;
            if (r < high && col + vc < g.cols) old[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(X) + (int64_t)(row_w + r) * g.ld_x + col + vc);
        }
    };
    if (g.x_vec && g.update) fetch(col_w);
#pragma unroll 1
    for (int q = 0; q < NC / 32; ++q) {
        const int col = col_w + q * 32;
        if (col >= g.cols) break;
        {
            uint32_t u[32];
            tmem_ld32(d + q * 32, u);
            tmem_ld_wait();
            __syncwarp();
            // rows of 32, four-entry groups exchanged within a row so that neither side meets a bank twice
#pragma unroll
            for (int e = 0; e < 32; e += 4)
                *reinterpret_cast<float4*>(blk + lane * 32 + (e ^ ((lane & 7) * 4))) =
                    make_float4(alpha * __uint_as_float(u[e]), alpha * __uint_as_float(u[e + 1]), alpha * __uint_as_float(u[e + 2]), alpha * __uint_as_float(u[e + 3]));
            __syncwarp();
        }
        if (g.x_vec) {
#pragma unroll
            for (int i = 0; i < 32 / STEP; ++i) {
                const int r = vr + i * STEP;
                if (r >= high || col + vc >= g.cols) continue;
                float v[V];
#pragma unroll
                for (int e = 0; e < V; e += 4) {
                    const float4 f = *reinterpret_cast<const float4*>(blk + r * 32 + ((vc + e) ^ ((r & 7) * 4)));
                    v[e] = f.x; v[e + 1] = f.y; v[e + 2] = f.z; v[e + 3] = f.w;
                }
                if (g.update) {
                    const uint32_t w[4] = {old[i].x, old[i].y, old[i].z, old[i].w};
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float x = sizeof(T) == 4 ? __uint_as_float(w[e * 4 / V]) : e % 2 ? bf16hi_to_f32(w[e / 2]) : bf16lo_to_f32(w[e / 2]);
                        v[e] = g.wc * x - g.wd * v[e];
                    }
                }
                T* x = reinterpret_cast<T*>(X) + (int64_t)(row_w + r) * g.ld_x + col + vc;
                if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(x) = make_float4(v[0], v[1], v[2], v[3]);
                else *reinterpret_cast<uint4*>(x) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
            }
            if (g.update && q + 1 < NC / 32) fetch(col + 32);
        } else if (col + lane < g.cols) {
            T* x = reinterpret_cast<T*>(X) + (int64_t)row_w * g.ld_x + col + lane;
            // (sixteen loads under way: stores to X in between would hold each of them back)
#pragma unroll 1
            for (int r0 = 0; r0 < high; r0 += 16) {
                float x0[16];
                if (g.update) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) x0[r] = r0 + r < high ? to_float(x[(r0 + r) * g.ld_x]) : 0.f;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float f = blk[(r0 + r) * 32 + (lane ^ ((r & 7) * 4))];
                    if (r0 + r < high) x[(r0 + r) * g.ld_x] = from_float<T>(g.update ? g.wc * x0[r] - g.wd * f : f);
                }
            }
        }
        __syncwarp();
    }
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
        unsigned char* stage_ptr = smem + STAGE_BYTES + (warp - 2) * 4096;
        int acc = 0; uint32_t aph = 0;
        bool ok = true;
        for (int t = tile0; t < g.total && ok; t += tstep) {
            const Tile c = decode<PAIR, BN>(g, t);
            if (!c.active) continue;
            const int row_w = c.row0 + crank * 128 + quarter * 32, col_w = c.col0 + half * NC;
            const bool mine = row_w < g.rows && col_w < g.cols;
            const uint32_t mine_tmem = tmem_base + half * NC + ((uint32_t)(quarter * 32) << 16);
            if (TERMS == 1) {
                // (all lanes alike: a wait that ran out for one ends the warp's work)
                ok = __all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * acc, aph, abort_flag));
                if (!ok) break;
                tc_fence_after();
            } else {
                // Sums of the chunks, in registers; the total goes back to where the last chunk was, so that what follows is one
                // rolled loop for either form (unrolled, its code is fetched more slowly than it runs).
                float v[NC];
#pragma unroll
                for (int e = 0; e < NC; ++e) v[e] = 0.f;
                int left = (g.kblocks + g.chunk - 1) / g.chunk;
                while (true) {
                    ok = __all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * acc, aph, abort_flag));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t d = mine_tmem + acc * BN;
#pragma unroll
                    for (int q = 0; q < NC / 16; ++q) {
                        uint32_t u[16];
                        tmem_ld16(d + q * 16, u);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[q * 16 + e] += __uint_as_float(u[e]);
                    }
                    if (--left == 0) break;
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) { if (PAIR) mbar_arrive_remote(tempty_ld + 8 * acc); else mbar_arrive(tempty0 + 8 * acc); }
                    if (++acc == 2) { acc = 0; aph ^= 1; }
                }
                if (!ok) break;
                const uint32_t d = mine_tmem + acc * BN;
#pragma unroll
                for (int q = 0; q < NC / 16; ++q) tmem_st16(d + q * 16, &v[q * 16]);
                tmem_st_wait();
            }
            const uint32_t d = mine_tmem + acc * BN;
            float alpha = g.alpha;
            if (g.sigma_pow) {
                const float sg = g.slot[c.mat].sigma;
                alpha *= g.sigma_pow == 2 ? sg * sg : sg;
            }
            if constexpr (EPI == EPI_IMAGE) {
                if (mine) image_epilogue<TERMS, NC>(g, d, alpha, c.mat, row_w, lane, col_w, c.mirror, stage_ptr);
            } else {
                if (mine && !g.slot[c.mat].status) {
                    if (g.x_bf16) final_epilogue<__nv_bfloat16, NC>(g, d, alpha, table.w[c.mat].X, row_w, lane, col_w, stage_ptr);
                    else final_epilogue<float, NC>(g, d, alpha, table.w[c.mat].X, row_w, lane, col_w, stage_ptr);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) { if (PAIR) mbar_arrive_remote(tempty_ld + 8 * acc); else mbar_arrive(tempty0 + 8 * acc); }
            if (++acc == 2) { acc = 0; aph ^= 1; }
        }
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
