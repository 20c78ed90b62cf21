// The KNN-LM mixture: one row of target probabilities from a row of logits and the neighbours that
// the search returned for it,
//     p[v] = (1 - lambda) softmax(logits / T)[v] + lambda * sum over {i: values[id_i] = v} of w_i,
// with w the softmax of the neighbours' scores over their own temperature.
//
// Bound by memory: a logit is read once and a probability written once (6 bytes an entry in 16 bits). One pass
// over global memory therefore, the slice of a row waiting in shared memory between maximum, sum and output,
// and a cluster per row, so that a row of 128000 entries is spread over eight SMs' shared memory. Measured (512
// rows x 128000, bf16, 64 neighbours): 72 to 76 us, 5.2 to 5.5 TB/s, 0.80 to 0.85 of the measured copy bandwidth; without
// neighbours 66 us.
// Stores had to be 16 bytes per thread and aligned whatever the input's alignment (333 -> 127 us with the slice
// staged), and the exchange between CTAs one store per warp instead of block and cluster barriers (127 -> 76 us).
// A single row of 32000 takes 3.8 us in a CUDA graph, 4.9 us with neighbours (ids, then the values they point at: two more
// round trips to memory); called one by one 6.2 us, what the host needs for a launch.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "common.cuh"

namespace ralm {
namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f;

// 2^x within 2 units of 2^-23 of it; below 2^-126 it is 0.
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(float x) { return x; }

constexpr int kMixThreads = 256;
constexpr int kMixWarps = kMixThreads / 32;
constexpr int kMixNeighbours = 4;    // per thread: RALM_MAX_K / kMixThreads
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
    float score_sign;    // -1 for distances
    float score_scale;   // log2(e) / knn temperature
    float logit_scale;   // log2(e) / temperature
    float lambda;
    float *probs;
    int64_t ld_probs;
    int slice;           // elements of a row that one CTA of the cluster handles, a multiple of a 16-byte vector's 4 or 8
    int slots;           // hash slots for the neighbours' tokens, a power of two, at least k
};

template <typename T> struct MixVec {
    static constexpr int n = 16 / sizeof(T);
    union { uint4 raw; T x[n]; };
};

// A value reduced over the CTA; every thread gets it. `buf`: 32 floats.
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
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// What the exponentials of a row are taken relative to. In powers of two the reference is a whole number r
// at or above the largest exponent m scale: x scale - r is then one fused product and sum, rounded once, and
// two references differ by an exact power of two. From 2^22 on the rounding of m scale itself would be a step of
// more than 1/4, soon of more powers of two than 32 bits have (rows masked by -1e9 or lower throughout, small
// temperatures): there the differences x - m are scaled instead.
constexpr float kMixWide = 4194304.f;
struct MixRef {
    float m, r;
    bool wide;
    __device__ __forceinline__ MixRef(float top, float scale) : m(top), r(0.f), wide(false) {
        if (top == -INFINITY) return;
        const float e = top * scale;
        wide = !(fabsf(e) < kMixWide);
        if (!wide) r = ceilf(e);
    }
    __device__ __forceinline__ float power(float x, float scale) const {   // 2^(x scale) over the reference
        return wide ? exp2_approx((x - m) * scale) : exp2_approx(fmaf(x, scale, -r));
    }
};
// A sum relative to `from`, relative to `to`; one over nothing but -inf is 0 (or NaN) and stays as it is. A reference
// is 2^(m scale) in the one form and 2^r in the other.
__device__ __forceinline__ float rescaled(const MixRef &from, float s, const MixRef &to, float scale) {
    if (from.m == -INFINITY) return s;
    float e;
    if (to.wide) e = from.wide ? (from.m - to.m) * scale : fmaf(-to.m, scale, from.r);
    else e = from.wide ? fmaf(from.m, scale, -to.r) : from.r - to.r;
    return s * exp2_approx(e);
}
__device__ __forceinline__ float vec_max(const MixVec<float> &u) { return fmaxf(fmaxf(u.x[0], u.x[1]), fmaxf(u.x[2], u.x[3])); }
__device__ __forceinline__ float vec_max(const MixVec<__half> &u) {
    const __half2 *h = reinterpret_cast<const __half2 *>(u.x);
    const __half2 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return __half2float(__hmax(__low2half(m), __high2half(m)));
}
__device__ __forceinline__ float vec_max(const MixVec<__nv_bfloat16> &u) {
    const __nv_bfloat162 *h = reinterpret_cast<const __nv_bfloat162 *>(u.x);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return __bfloat162float(__hmax(__low2bfloat16(m), __high2bfloat16(m)));
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, int rank) {   // the same variable in another CTA of the cluster
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// Stores 8 bytes into another CTA's shared memory and counts them on a barrier there.
__device__ __forceinline__ void st_async_f32x2(uint32_t addr, float a, float b, uint32_t bar) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(addr), "f"(a), "f"(b),
                 "r"(bar)
                 : "memory");
}

// 2^e or 2^-e, e the exponent of a weight in (0, 1] given by its bits (0: of the smallest normal number).
__device__ __forceinline__ float mix_unit(uint32_t bits, int sign) {
    const int e = max(static_cast<int>(bits >> 23), 1) - 127;
    return __uint_as_float(static_cast<uint32_t>(127 + sign * e) << 23);
}

// One cluster per row; CTA c of it handles elements [c * slice, (c + 1) * slice) of the row, counted
// from the 16-byte boundary at or below the row's start, so that 16-byte accesses stay aligned for any
// row pitch. STAGED: one bulk copy brings the slice into shared memory, where all passes (maximum; sum;
// probabilities) find it, and the neighbours are looked up while it is on its way; otherwise the
// slice does not fit and is read from global memory again. The CTAs exchange one (maximum, sum) per warp,
// by stores that count on the receiver's barrier.
//
// Neighbours' weights are summed per token in a hash table: first the largest weight of each token, then the
// sum in units of 2^-41 of that one's power of two, in two limbs of 21 bits. Maxima and whole numbers have no
// order, so the result does not depend on that of the atomics, and small sums keep their precision.
template <typename T, bool STAGED>
__global__ void __launch_bounds__(kMixThreads)
mix_kernel(const MixParams p) {
    constexpr int VEC = MixVec<T>::n;
    extern __shared__ __align__(16) unsigned char mix_smem[];
    __shared__ float best_of[kMixWarps], mass_of[kMixWarps];
    __shared__ __align__(8) float2 peers[kMixMaxCluster * kMixWarps];
    __shared__ __align__(8) uint64_t bars[2];
    cg::cluster_group cluster = cg::this_cluster();
    const int C = cluster.num_blocks(), c = cluster.block_rank();
    const int row = blockIdx.x / C, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const T *x = static_cast<const T *>(p.logits) + static_cast<int64_t>(row) * p.ld_logits;
    float *out = p.probs + static_cast<int64_t>(row) * p.ld_probs;
    const int mis = static_cast<int>(reinterpret_cast<uintptr_t>(x) / sizeof(T) % VEC);
    const int base = c * p.slice - mis;              // row element that slice position 0 holds
    const int count = min(p.slice, p.V - base);      // positions of the slice inside the row (<= 0: none)
    const int vecs = count > 0 ? (count + VEC - 1) / VEC : 0;
    const uint32_t arrived = smem_u32(&bars[0]), told = smem_u32(&bars[1]);
    T *stage = reinterpret_cast<T *>(mix_smem);
    uint4 *slots = reinterpret_cast<uint4 *>(mix_smem + (STAGED ? p.slice * sizeof(T) : 0));   // two limbs, largest weight, token
    auto load = [&](int v, MixVec<T> &u) {
        const int e = base + v * VEC;
        if (e >= 0 && e + VEC <= p.V) {
            u.raw = *reinterpret_cast<const uint4 *>(x + e);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) u.x[j] = e + j >= 0 && e + j < p.V ? x[e + j] : T(-INFINITY);
        }
    };
    const int v0 = base < 0 ? 1 : 0, v1 = max(vecs > 0 && base + vecs * VEC > p.V ? vecs - 1 : vecs, v0);   // whole vectors
    if (tid == 0) {
        mbar_init(arrived, 1);
        mbar_init(told, 1);
        mbar_fence_init();
        mbar_arrive_expect_tx(told, C * kMixWarps * 8);
        if (STAGED) {
            const uint32_t bytes = (v1 - v0) * 16;
            if (bytes) {
                mbar_arrive_expect_tx(arrived, bytes);
                bulk_load(smem_u32(stage + v0 * VEC), x + base + v0 * VEC, bytes, arrived);
            } else {
                mbar_arrive(arrived);
            }
        }
    }
    if (STAGED && tid < 2 && vecs > 0) {              // the row's ragged ends
        const int v = tid == 0 ? 0 : vecs - 1;
        if (v < v0 || v >= v1) {
            MixVec<T> u;
            load(v, u);
            *reinterpret_cast<uint4 *>(stage + v * VEC) = u.raw;
        }
    }
    __syncthreads();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // the barriers stand (fenced above)

    // the neighbours, by as many warps as they fill: what they are is asked for before the logits are worked on
    const int k_warps = min((p.k + 31) / 32, kMixWarps);
    float score[kMixNeighbours];
    int token[kMixNeighbours];
    if (warp < k_warps) {
        int64_t id[kMixNeighbours];
#pragma unroll
        for (int j = 0; j < kMixNeighbours; ++j) {
            const int i = tid + j * k_warps * 32;
            id[j] = i < p.k ? p.ids[static_cast<int64_t>(row) * p.k + i] : -1;
            score[j] = i < p.k ? p.scores[static_cast<int64_t>(row) * p.k + i] * p.score_sign : 0.f;
        }
        for (int i = tid; i < p.slots; i += k_warps * 32) slots[i] = make_uint4(0, 0, 0, 0xFFFFFFFFu);
#pragma unroll
        for (int j = 0; j < kMixNeighbours; ++j) {
            token[j] = -1;
            if (id[j] >= 0 && id[j] < p.N && fabsf(score[j]) < INFINITY) token[j] = p.values[id[j]];
        }
    }

    // the logits: the warp's maximum, then its sum
    bool lost = STAGED && !mbar_wait_bounded(arrived, 0);
    float m = -INFINITY;
#pragma unroll 4
    for (int v = tid; v < vecs; v += kMixThreads) {
        MixVec<T> u;
        if (STAGED) u.raw = *reinterpret_cast<const uint4 *>(stage + v * VEC);
        else load(v, u);
        m = fmaxf(m, vec_max(u));
    }
    const MixRef mine(warp_max(m), p.logit_scale);
    float s = lost ? NAN : 0.f;                       // never seen: the row says so
#pragma unroll 4
    for (int v = tid; v < vecs; v += kMixThreads) {
        MixVec<T> u;
        if (STAGED) u.raw = *reinterpret_cast<const uint4 *>(stage + v * VEC);
        else load(v, u);
        float part[2] = {0.f, 0.f};
        if (mine.wide) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) part[j & 1] += exp2_approx((to_float(u.x[j]) - mine.m) * p.logit_scale);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) part[j & 1] += exp2_approx(fmaf(to_float(u.x[j]), p.logit_scale, -mine.r));
        }
        s += part[0] + part[1];
    }
    s = warp_sum(s);
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (lane < C) st_async_f32x2(map_to_rank(smem_u32(&peers[c * kMixWarps + warp]), lane), mine.m, s, map_to_rank(told, lane));
    // weights relative to the best neighbour, their sum, and their sums per token of the slice
    int own[kMixNeighbours];                          // slots that this thread was the first to take
    if (warp < k_warps) {
        float best = -INFINITY;
#pragma unroll
        for (int j = 0; j < kMixNeighbours; ++j) {
            if (token[j] >= p.V) token[j] = -1;
            if (token[j] >= 0) best = fmaxf(best, score[j]);
        }
        best = warp_max(best);
        if (lane == 0) best_of[warp] = best;
        named_barrier(1, k_warps * 32);
        for (int i = 0; i < k_warps; ++i) best = fmaxf(best, best_of[i]);
        float sum = 0.f;
        int in_slot[kMixNeighbours];
#pragma unroll
        for (int j = 0; j < kMixNeighbours; ++j) {
            own[j] = in_slot[j] = -1;
            if (token[j] < 0) continue;
            // the weight from here on: differences are scaled, and halves subtracted, so that no finite score is too large
            score[j] = exp2_approx(2.f * (fmaf(score[j], 0.5f, -0.5f * best) * p.score_scale));
            sum += score[j];
            const int pos = token[j] - base;
            if (pos < 0 || pos >= p.slice) continue;
            int h = (token[j] * 0x9E3779B1u) >> 20 & (p.slots - 1);
            for (;;) {                                // at most k tokens in k slots or more: there is always a place
                const uint32_t seen = atomicCAS(&slots[h].w, 0xFFFFFFFFu, static_cast<uint32_t>(token[j]));
                if (seen == 0xFFFFFFFFu) own[j] = h;
                if (seen == 0xFFFFFFFFu || seen == static_cast<uint32_t>(token[j])) break;
                h = (h + 1) & (p.slots - 1);
            }
            in_slot[j] = h;
            atomicMax(&slots[h].z, __float_as_uint(score[j]));
        }
        named_barrier(1, k_warps * 32);
#pragma unroll
        for (int j = 0; j < kMixNeighbours; ++j) {
            if (in_slot[j] < 0) continue;
            uint4 &slot = slots[in_slot[j]];
            const uint64_t fixed = __float2ull_rn(score[j] * mix_unit(slot.z, -1) * 2199023255552.f);     // 2^41
            atomicAdd(&slot.x, static_cast<uint32_t>(fixed & 0x1FFFFF));
            atomicAdd(&slot.y, static_cast<uint32_t>(fixed >> 21));
        }
        sum = warp_sum(sum);
        if (lane == 0) mass_of[warp] = sum;
    }
    __syncthreads();                                  // the neighbours' sums
    lost = !mbar_wait_bounded(told, 0);
    float M = -INFINITY, S = lost ? NAN : 0.f;
    for (int i = lane; i < C * kMixWarps; i += 32) M = fmaxf(M, peers[i].x);
    const MixRef ref(warp_max(M), p.logit_scale);
    for (int i = lane; i < C * kMixWarps; i += 32) S += rescaled(MixRef(peers[i].x, p.logit_scale), peers[i].y, ref, p.logit_scale);
    S = warp_sum(S);
    float mass = 0.f;
    for (int i = 0; i < k_warps; ++i) mass += mass_of[i];
    // a row without neighbours is the model's alone; a row whose every logit is -inf the neighbours'
    const float lambda = mass > 0.f ? (S == 0.f ? 1.f : p.lambda) : 0.f;
    const float scale = S == 0.f ? 0.f : (1.f - lambda) / S;
    // 16-byte stores from the first aligned element of the slice's output on, whatever that is in the input
    const int e0 = max(base, 0), e1 = min(base + p.slice, p.V);
    if (e0 < e1) {
        const int head = min(static_cast<int>((4 - reinterpret_cast<uintptr_t>(out + e0) / 4 % 4) % 4), e1 - e0);
        const int quads = (e1 - e0 - head) / 4;
        const int first = e0 + head;
        auto write = [&](auto wide_type) {
            constexpr bool wide = decltype(wide_type)::value;
            auto prob = [&](T z) {
                return exp2_approx(wide ? (to_float(z) - ref.m) * p.logit_scale : fmaf(to_float(z), p.logit_scale, -ref.r)) * scale;
            };
            auto value = [&](int e) { return prob(STAGED ? stage[e - base] : x[e]); };
            float4 *o = reinterpret_cast<float4 *>(out + first);
            if (STAGED && (first - base) % 4 == 0) {
#pragma unroll 4
                for (int i = tid; i < quads; i += kMixThreads) {
                    union { uint2 half; uint4 full; T x[4]; } u;
                    if (sizeof(T) == 2) u.half = *reinterpret_cast<const uint2 *>(stage + (first - base) + 4 * i);
                    else u.full = *reinterpret_cast<const uint4 *>(stage + (first - base) + 4 * i);
                    __stcs(o + i, make_float4(prob(u.x[0]), prob(u.x[1]), prob(u.x[2]), prob(u.x[3])));
                }
            } else {
#pragma unroll 4
                for (int i = tid; i < quads; i += kMixThreads) {
                    const int e = first + 4 * i;
                    __stcs(o + i, make_float4(value(e), value(e + 1), value(e + 2), value(e + 3)));
                }
            }
            const int tail = first + 4 * quads;
            if (tid < head) out[e0 + tid] = value(e0 + tid);
            if (tid < e1 - tail) out[tail + tid] = value(tail + tid);
        };
        if (ref.wide) write(std::true_type{});
        else write(std::false_type{});
    }
    if (lambda > 0.f) {
        __syncthreads();
        if (warp < k_warps) {
#pragma unroll
            for (int j = 0; j < kMixNeighbours; ++j) {
                if (own[j] < 0) continue;
                const uint4 limbs = slots[own[j]];
                const uint64_t fixed = (static_cast<uint64_t>(limbs.y) << 21) + limbs.x;
                const float w = __ull2float_rn(fixed) * 4.547473508864641e-13f * mix_unit(limbs.z, 1);   // 2^-41
                const int t = token[j];
                out[t] = ref.power(to_float(STAGED ? stage[t - base] : x[t]), p.logit_scale) * scale + lambda * w / mass;
            }
        }
    }
}

}  // namespace ralm
