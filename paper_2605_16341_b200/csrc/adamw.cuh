// The AdamW step of tensors of any length: one pass over X, G and both moments.
#pragma once
#include "common.cuh"
#include "launch.cuh"

namespace od {
namespace adamw {

constexpr int MAX_TENSORS = 64;          // of one launch (its table: 3.5 KB of kernel parameters)
constexpr int MAX_KINDS = 8;             // different constants among them
constexpr int THREADS = 256;
constexpr int CHUNK = 8 * THREADS * 2;   // entries that one block takes at a time

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
    int32_t last, blocks;                // last: this launch ends the step
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
    __shared__ Consts consts[MAX_KINDS];
    grid_dependency();
    // the bias corrections in 64 bits: 1 - beta^t of a beta near 1 loses most of 24
    if (threadIdx.x < MAX_KINDS) {
        const Kind& k = a.kind[threadIdx.x];
        const double t = (double)(a.step[0] + 1);
        consts[threadIdx.x] = Consts{k.beta1, k.rest1, k.beta2, k.rest2, k.eps, k.eta, k.wd, (float)(-1.0 / expm1(t * k.log_beta1)),
                                     (float)(-1.0 / expm1(t * k.log_beta2))};
    }
    __syncthreads();
    int at = 0;
    for (int chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        while (at + 1 < a.count && a.t[at + 1].first_chunk <= chunk) ++at;
        const Tensor& t = a.t[at];
        const Consts k = consts[t.kind];
        const int64_t begin = (int64_t)(chunk - t.first_chunk) * CHUNK;
#pragma unroll
        for (int u = 0; u < CHUNK; u += 8 * THREADS) {
            const int64_t i = begin + u + threadIdx.x * 8;
            if (i + 8 <= t.numel) {
                float x[8], m[8], v[8], g[8];
                load8<X_BF16>(t.X, i, x);
                load8<G_BF16>(t.G, i, g);
                load8<false>(t.M, i, m);
                load8<false>(t.V, i, v);
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
                    float x = X_BF16 ? __bfloat162float(reinterpret_cast<__nv_bfloat16*>(t.X)[j]) : reinterpret_cast<float*>(t.X)[j];
                    const float g = G_BF16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(t.G)[j]) : reinterpret_cast<const float*>(t.G)[j];
                    float m = t.M[j], v = t.V[j];
                    update(k, x, m, v, g);
                    if (X_BF16) reinterpret_cast<__nv_bfloat16*>(t.X)[j] = __float2bfloat16_rn(x);
                    else reinterpret_cast<float*>(t.X)[j] = x;
                    t.M[j] = m; t.V[j] = v;
                }
            }
        }
    }
    // The block that is done last counts the step: every block has read the count by then, and a replayed graph finds it raised.
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned long long* s = reinterpret_cast<unsigned long long*>(a.step);
        if (atomicAdd(&s[1], 1ULL) + 1 == (unsigned long long)a.blocks) {
            s[1] = 0;
            if (a.last) s[0] += 1;
        }
    }
}

}  // namespace adamw
}  // namespace od
