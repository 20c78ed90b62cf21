// The KNN-LM mixture: one row of target probabilities from a row of logits and the neighbours that
// the search returned for it,
//     p[v] = (1 - lambda) softmax(logits / T)[v] + lambda * sum over {i: values[id_i] = v} of w_i,
// with w the softmax of the neighbours' scores over their own temperature.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "common.cuh"

namespace ralm {
namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(float x) { return x; }

constexpr int kMixThreads = 512;
constexpr int kMixSlots = 2048;     // hash slots for the neighbours' tokens, twice RALM_MAX_K
constexpr int kMixMaxCluster = 8;

struct MixParams {
    const void *logits;
    int64_t ld_logits;
    int V;
    const int64_t *ids;
    const float *scores;
    int k;
    const int32_t *values;
    int64_t N;
    float score_scale;   // log2(e) / knn temperature, negative for distances
    float logit_scale;   // log2(e) / temperature
    float lambda;
    float *probs;
    int64_t ld_probs;
    int slice;           // elements of a row that one CTA of the cluster handles, a multiple of 16
};

template <typename T> struct MixVec {
    static constexpr int n = 16 / sizeof(T);
    union { uint4 raw; T x[n]; };
};

// The sum of a value over the CTA; every thread gets it. `buf`: 32 floats.
template <typename Op>
__device__ __forceinline__ float block_reduce(float v, float *buf, Op op) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    float r = buf[0];
    for (int i = 1; i < (int)(blockDim.x >> 5); ++i) r = op(r, buf[i]);
    return r;
}

// One cluster per row; CTA c of it handles elements [c * slice, (c + 1) * slice) of the row, counted
// from the 16-byte boundary at or below the row's start, so that 16-byte loads stay aligned for any
// row pitch. STAGED keeps the slice in shared memory between the two passes.
//
// Shared neighbours' weights are summed per token in a hash table whose sums are integers (54-bit
// fixed point in three 18-bit limbs), so the result does not depend on the order of the atomics.
template <typename T, bool STAGED>
__global__ void __launch_bounds__(kMixThreads)
mix_kernel(const MixParams p) {
    constexpr int VEC = MixVec<T>::n;
    extern __shared__ __align__(16) unsigned char mix_smem[];
    __shared__ int slot_token[kMixSlots];
    __shared__ uint32_t slot_sum[3][kMixSlots];
    __shared__ float buf[32];
    __shared__ float2 peers[kMixMaxCluster];
    cg::cluster_group cluster = cg::this_cluster();
    const int C = cluster.num_blocks(), c = cluster.block_rank();
    const int row = blockIdx.x / C, tid = threadIdx.x;
    const T *x = static_cast<const T *>(p.logits) + static_cast<int64_t>(row) * p.ld_logits;
    float *out = p.probs + static_cast<int64_t>(row) * p.ld_probs;
    const int mis = static_cast<int>(reinterpret_cast<uintptr_t>(x) / sizeof(T) % VEC);
    const int base = c * p.slice - mis;              // row element that slice position 0 holds
    const int count = min(p.slice, p.V - base);      // positions of the slice inside the row (<= 0: none)
    T *stage = reinterpret_cast<T *>(mix_smem);

    // the neighbours: weights relative to the best one, their sum, and the sum per token
    float mass = 0.f;
    if (p.k > 0) {
        for (int i = tid; i < kMixSlots; i += kMixThreads) {
            slot_token[i] = -1;
            slot_sum[0][i] = slot_sum[1][i] = slot_sum[2][i] = 0;
        }
        float s[2];
        int token[2];
        float best = -INFINITY;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = tid + j * kMixThreads;
            token[j] = -1;
            if (i < p.k) {
                const int64_t id = p.ids[static_cast<int64_t>(row) * p.k + i];
                const float sc = p.scores[static_cast<int64_t>(row) * p.k + i] * p.score_scale;
                if (id >= 0 && id < p.N && fabsf(sc) < INFINITY) {
                    const int t = p.values[id];
                    if (t >= 0 && t < p.V) {
                        token[j] = t;
                        s[j] = sc;
                        best = fmaxf(best, sc);
                    }
                }
            }
        }
        best = block_reduce(best, buf, [](float a, float b) { return fmaxf(a, b); });
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (token[j] < 0) continue;
            const float w = exp2_approx(s[j] - best);
            sum += w;
            const int pos = token[j] - base;
            if (pos < 0 || pos >= p.slice) continue;
            int h = (token[j] * 0x9E3779B1u) >> 21;
            for (;;) {
                const int seen = atomicCAS(&slot_token[h], -1, token[j]);
                if (seen == -1 || seen == token[j]) break;
                h = (h + 1) & (kMixSlots - 1);
            }
            const uint64_t fixed = static_cast<uint64_t>(__float2ull_rn(w * 18014398509481984.f));  // 2^54
            atomicAdd(&slot_sum[0][h], static_cast<uint32_t>(fixed & 0x3FFFF));
            atomicAdd(&slot_sum[1][h], static_cast<uint32_t>(fixed >> 18 & 0x3FFFF));
            atomicAdd(&slot_sum[2][h], static_cast<uint32_t>(fixed >> 36));
        }
        mass = block_reduce(sum, buf, [](float a, float b) { return a + b; });
    }

    // the logits: running maximum and sum
    float m = -INFINITY, s = 0.f;
    const int vecs = count > 0 ? (count + VEC - 1) / VEC : 0;
    auto load = [&](int v, MixVec<T> &u) {
        const int e = base + v * VEC;
        if (e >= 0 && e + VEC <= p.V) {
            u.raw = *reinterpret_cast<const uint4 *>(x + e);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) u.x[j] = e + j >= 0 && e + j < p.V ? x[e + j] : T(-INFINITY);
        }
    };
#pragma unroll 4
    for (int v = tid; v < vecs; v += kMixThreads) {
        MixVec<T> u;
        load(v, u);
        if (STAGED) *reinterpret_cast<uint4 *>(stage + v * VEC) = u.raw;
        float mx = to_float(u.x[0]);
#pragma unroll
        for (int j = 1; j < VEC; ++j) mx = fmaxf(mx, to_float(u.x[j]));
        if (mx > m) {
            s *= exp2_approx((m - mx) * p.logit_scale);   // m = -inf: s is 0 (or NaN) and stays it
            m = mx;
        }
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int j = 0; j < VEC; ++j) s += exp2_approx((to_float(u.x[j]) - ref) * p.logit_scale);
    }
    const float cta_m = block_reduce(m, buf, [](float a, float b) { return fmaxf(a, b); });
    const float cta_s = block_reduce(m == -INFINITY ? s : s * exp2_approx((m - cta_m) * p.logit_scale), buf,
                                     [](float a, float b) { return a + b; });
    cluster.sync();
    if (tid < C) *cluster.map_shared_rank(&peers[c], tid) = make_float2(cta_m, cta_s);
    cluster.sync();
    float M = -INFINITY, S = 0.f;
    for (int i = 0; i < C; ++i) M = fmaxf(M, peers[i].x);
    for (int i = 0; i < C; ++i)
        S += peers[i].x == -INFINITY ? peers[i].y : peers[i].y * exp2_approx((peers[i].x - M) * p.logit_scale);
    const float ref = M == -INFINITY ? 0.f : M;
    // a row without neighbours is the model's alone; a row whose every logit is -inf the neighbours'
    const float lambda = mass > 0.f ? (S == 0.f ? 1.f : p.lambda) : 0.f;
    const float scale = S == 0.f ? 0.f : (1.f - lambda) / S;
    const float *end = out + p.V;
#pragma unroll 2
    for (int v = tid; v < vecs; v += kMixThreads) {
        MixVec<T> u;
        if (STAGED) u.raw = *reinterpret_cast<const uint4 *>(stage + v * VEC);
        else load(v, u);
        float *o = out + base + v * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (o + j >= out && o + j < end) o[j] = exp2_approx((to_float(u.x[j]) - ref) * p.logit_scale) * scale;
    }
    if (p.k > 0 && lambda > 0.f) {
        __syncthreads();
        for (int h = tid; h < kMixSlots; h += kMixThreads) {
            const int t = slot_token[h];
            if (t < 0) continue;
            const uint64_t fixed = (static_cast<uint64_t>(slot_sum[2][h]) << 36) +
                                   (static_cast<uint64_t>(slot_sum[1][h]) << 18) + slot_sum[0][h];
            const float w = __ull2float_rn(fixed) * 5.551115123125783e-17f;                          // 2^-54
            const float z = STAGED ? to_float(stage[t - base]) : to_float(x[t]);
            out[t] = exp2_approx((z - ref) * p.logit_scale) * scale + lambda * w / mass;
        }
    }
}

}  // namespace ralm
