// The AdamW step of tensors of any length: one pass over X, G and both moments, bound by HBM.  A block takes one piece of one tensor, two groups of
// eight entries a thread: 65.5 M bf16 entries (1.44 GB) in 216 us, 6.65 TB/s; with 1184 blocks that walk over the pieces 255 us (they all
// wait for their loads at once), with one group a thread 237, with streaming hints on loads and stores 242 to 265.
#pragma once
#include "common.cuh"
#include "launch.cuh"

namespace od {
namespace adamw {

constexpr int MAX_TENSORS = 96;          // of one launch (its table: 5.5 KB of kernel parameters)
constexpr int MAX_KINDS = 8;             // different constants among them
constexpr int THREADS = 256, GROUPS = 2;
constexpr int CHUNK = 8 * THREADS * GROUPS;   // entries of one block

struct Tensor {
    void* X;
    float *M, *V;
    const void* G;
    int64_t numel;
    int32_t first_chunk;                 // chunks of the tensors before it
    int32_t kind;
};
struct Kind {
    double log_beta1, log_beta2;
    float beta1, rest1, beta2, rest2, eps, eta, wd, pad;
};
struct Table {
    int32_t count, chunks;
    int64_t* step;                       // [0]: steps taken, [1]: blocks of this step that are done
    int32_t last, pad;                   // last: this launch ends the step
    Kind kind[MAX_KINDS];
    Tensor t[MAX_TENSORS];
};

template <bool BF16>
__device__ __forceinline__ void load8(const void* p, int64_t i, float (&v)[8]) {
    if (BF16) {
        const uint4 u = *reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(p) + i);
        v[0] = bf16lo_to_f32(u.x); v[1] = bf16hi_to_f32(u.x); v[2] = bf16lo_to_f32(u.y); v[3] = bf16hi_to_f32(u.y);
        v[4] = bf16lo_to_f32(u.z); v[5] = bf16hi_to_f32(u.z); v[6] = bf16lo_to_f32(u.w); v[7] = bf16hi_to_f32(u.w);
    } else {
        const float4* q = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + i);
        const float4 x = q[0], y = q[1];
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

struct Consts { float beta1, rest1, beta2, rest2, eps, eta, wd, c1, c2; };   // c1, c2: 1 / (1 - beta^t)

__device__ __forceinline__ void update(const Consts& k, float& x, float& m, float& v, float g) {
    m = fmaf(k.beta1, m, k.rest1 * g);
    v = fmaf(k.beta2, v, k.rest2 * g * g);
    x -= k.eta * fmaf(k.wd, x, m * k.c1 / (sqrtf(v * k.c2) + k.eps));
}

template <bool X_BF16, bool G_BF16>
__global__ void __launch_bounds__(THREADS) adamw_kernel(const __grid_constant__ Table a) {
    __shared__ float correction[2];
    grid_dependency();
    const int chunk = (int)blockIdx.x;
    int at = 0;                              // the last tensor that begins at this piece or before
    for (int end = a.count; end - at > 1;) {
        const int middle = (at + end) / 2;
        if (a.t[middle].first_chunk <= chunk) at = middle;
        else end = middle;
    }
    const Tensor& t = a.t[at];
    const Kind& kind = a.kind[t.kind];
    const int64_t begin = (int64_t)(chunk - t.first_chunk) * CHUNK + threadIdx.x * 8;
    float x[8], m[8], v[8], g[8];
    auto load = [&](int64_t i) {
        load8<X_BF16>(t.X, i, x);
        load8<G_BF16>(t.G, i, g);
        load8<false>(t.M, i, m);
        load8<false>(t.V, i, v);
    };
    if (begin + 8 <= t.numel) load(begin);
    // the bias corrections in 64 bits: 1 - beta^t of a beta near 1 loses most of 24
    if (threadIdx.x < 2) correction[threadIdx.x] = (float)(-1.0 / expm1((double)(a.step[0] + 1) * (threadIdx.x ? kind.log_beta2 : kind.log_beta1)));
    __syncthreads();
    const Consts k{kind.beta1, kind.rest1, kind.beta2, kind.rest2, kind.eps, kind.eta, kind.wd, correction[0], correction[1]};
#pragma unroll
    for (int u = 0; u < GROUPS; ++u) {
        const int64_t i = begin + u * 8 * THREADS;
        if (i + 8 <= t.numel) {
            if (u) load(i);
#pragma unroll
            for (int e = 0; e < 8; ++e) update(k, x[e], m[e], v[e], g[e]);
            if (X_BF16)
                *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(t.X) + i) =
                    make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
            else
                store8(reinterpret_cast<float*>(t.X) + i, x);
            store8(t.M + i, m);
            store8(t.V + i, v);
        } else {
            for (int64_t j = i; j < t.numel && j < i + 8; ++j) {
                float w = X_BF16 ? __bfloat162float(reinterpret_cast<__nv_bfloat16*>(t.X)[j]) : reinterpret_cast<float*>(t.X)[j];
                const float d = G_BF16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(t.G)[j]) : reinterpret_cast<const float*>(t.G)[j];
                float mj = t.M[j], vj = t.V[j];
                update(k, w, mj, vj, d);
                if (X_BF16) reinterpret_cast<__nv_bfloat16*>(t.X)[j] = __float2bfloat16_rn(w);
                else reinterpret_cast<float*>(t.X)[j] = w;
                t.M[j] = mj; t.V[j] = vj;
            }
        }
    }
    // The block that is done last counts the step: every block has read the count by then, and a replayed graph finds it raised.
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned long long* s = reinterpret_cast<unsigned long long*>(a.step);
        if (atomicAdd(&s[1], 1ULL) + 1 == (unsigned long long)gridDim.x) {
            s[1] = 0;
            if (a.last) s[0] += 1;
        }
    }
}

}  // namespace adamw
}  // namespace od
