// Verification of drafted tokens against the target's probabilities from given random numbers
// (speculative sampling): position i is accepted while u_i q_i[t_i] < p_i[t_i]; at the first
// rejection the token is drawn from max(p - q, 0), after a full acceptance from the next row of p.
//
// The draw inverts a cumulative sum whose terms are whole numbers, w = floor(2^40 x): integer sums
// have no order, so any split over lanes, warps and CTAs gives the same token.
//
// Bound by memory: only the row of the first rejection is read (p and q, 8 bytes an entry), once, plus the run of
// it that holds the drawn token. Measured (256 requests, 8 drafts, 128000 entries): 52 us, 5.1 TB/s, 0.79 of the
// measured copy bandwidth; 64 requests of 50257 entries with certain drafts 10.3 us (7.8 us in a CUDA graph); one request
// 6.2 us (5.3), three dependent round trips to memory. Rows are read 4 bytes per lane, coalesced, eight loads in flight, because p's and q's rows
// of an odd vocabulary never share an alignment; the sums in two 32-bit words (nine plain instructions a term)
// instead of 64-bit shifts took 256 requests from 164 to 49 us.
#pragma once

#include <cooperative_groups.h>
#include <stdint.h>

#include <type_traits>

#include "common.cuh"

namespace ralm {

constexpr int kVtThreads = 512;
constexpr int kVtWarps = kVtThreads / 32;
constexpr int kVtMaxCluster = 8;

struct VerifyTokensParams {
    const int64_t *draft;        // [R][S]
    const float *draft_probs;    // or null: the draft was certain of its tokens
    int64_t draft_ld_r, draft_ld_s;
    const float *target_probs;
    int64_t target_ld_r, target_ld_s;
    const float *uniforms;       // [R][S + 1]
    const int32_t *draft_len;    // or null
    int S, V, slice;             // slice: elements of a row that one CTA handles
    int64_t *tokens;             // [R][S + 1]
    int32_t *accepted;           // [R]
};

// floor(2^40 min(max(x, 0), 1)), NaN counts as 0, as the sum of 2^20 hi and lo. Adding 8 and rounding
// towards zero leaves floor(2^20 x) in the last bits of the word; what that cut off is treated the same way
// at 2^-20 of the size. The constants (the words of 8 and 2^-17) stay in the sums until the end.
struct FixedSum { uint32_t hi, lo; };
constexpr uint32_t kFixedHi = 0x41000000u, kFixedLo = 0x37000000u;
__device__ __forceinline__ void fixed_add(FixedSum &s, float x) {
    x = fminf(fmaxf(x, 0.f), 1.f);
    const float y = __fadd_rz(x, 8.f);
    const float rest = __fsub_rn(x, __fsub_rn(y, 8.f));      // both exact
    s.hi += __float_as_uint(y) - kFixedHi;
    s.lo += __float_as_uint(__fadd_rz(rest, 7.62939453125e-6f)) - kFixedLo;
}
__device__ __forceinline__ uint64_t fixed_total(const FixedSum &s) { return (static_cast<uint64_t>(s.hi) << 20) + s.lo; }
constexpr int kFixedMost = 4095;                             // terms that the 32-bit sums hold
__device__ __forceinline__ uint64_t warp_sum_u64(uint64_t v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// One cluster per request. CTA c sums the weights of elements [c * slice, (c + 1) * slice), each warp
// a run of its own; the sums say which run holds the drawn token, and that CTA looks for it there.
__global__ void __launch_bounds__(kVtThreads, 2)
verify_tokens_kernel(const VerifyTokensParams p) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = cluster.num_blocks(), c = cluster.block_rank();
    const int r = blockIdx.x / C, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ uint64_t peers[2][kVtMaxCluster];
    __shared__ uint64_t warp_total[kVtWarps];
    __shared__ int first;
    const int64_t *draft = p.draft + static_cast<int64_t>(r) * p.S;
    const float *u = p.uniforms + static_cast<int64_t>(r) * (p.S + 1);
    const float *target = p.target_probs + r * p.target_ld_r;
    const float *dprobs = p.draft_probs ? p.draft_probs + r * p.draft_ld_r : nullptr;
    const int n = p.draft_len ? min(max(p.draft_len[r], 0), p.S) : p.S;

    if (warp == 0) {
        int a = n;
        for (int i0 = 0; i0 < n; i0 += 32) {
            const int i = i0 + lane;
            bool ok = true;
            if (i < n) {
                const int64_t t = draft[i];
                ok = false;
                if (t >= 0 && t < p.V) {
                    const float q = dprobs ? dprobs[i * p.draft_ld_s + t] : 1.f;
                    ok = __fmul_rn(u[i], q) < target[i * p.target_ld_s + t];
                }
            }
            const uint32_t bad = __ballot_sync(0xffffffffu, !ok);
            if (bad) {
                a = i0 + __ffs(bad) - 1;
                break;
            }
        }
        if (lane == 0) first = a;
    }
    __syncthreads();
    const int a = first;
    const float *prow = target + a * p.target_ld_s;
    const float *qrow = a < n && dprobs ? dprobs + a * p.draft_ld_s : nullptr;
    const int64_t gone = a < n && !dprobs ? draft[a] : -1;   // a certain draft: its token leaves the row

    const int lo = min(c * p.slice, p.V), hi = min(lo + p.slice, p.V);
    const int run = ((hi - lo + kVtWarps - 1) / kVtWarps + 31) & ~31;
    auto weight = [&](int v, bool whole) -> uint64_t {
        float x = prow[v];
        if (!whole) {
            if (qrow) x = __fsub_rn(x, qrow[v]);
            if (v == gone) x = 0.f;
        }
        FixedSum s = {0, 0};
        fixed_add(s, x);
        return fixed_total(s);
    };
    // the sum over a warp's run, each lane's part; the loads of a batch are all in flight together
    auto run_sum = [&](int w0, int w1, auto with_q) -> uint64_t {
        constexpr bool minus_q = decltype(with_q)::value;
        constexpr int kBatch = 8;
        uint64_t total = 0;
        FixedSum s = {0, 0};
        int terms = 0, v = w0 + lane;
        for (; v + 32 * (kBatch - 1) < w1; v += 32 * kBatch) {
            float x[kBatch], y[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) x[j] = __ldcs(prow + v + 32 * j);
            if (minus_q) {
#pragma unroll
                for (int j = 0; j < kBatch; ++j) y[j] = __ldcs(qrow + v + 32 * j);
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) fixed_add(s, minus_q ? __fsub_rn(x[j], y[j]) : x[j]);
            terms += kBatch;
            if (terms > kFixedMost - kBatch) {
                total += fixed_total(s);
                s = {0, 0};
                terms = 0;
            }
        }
        for (; v < w1; v += 32) fixed_add(s, minus_q ? __fsub_rn(prow[v], qrow[v]) : prow[v]);   // fewer than kBatch
        total += fixed_total(s);
        return total;
    };
    int64_t *out = p.tokens + static_cast<int64_t>(r) * (p.S + 1);
    if (c == 0) {
        for (int i = tid; i <= p.S; i += kVtThreads)
            if (i != a) out[i] = i < a ? draft[i] : -1;
        if (tid == 0) p.accepted[r] = a;
    }
    // the residual; should nothing be left of it, the target's row itself
    for (int round = 0; round < 2; ++round) {
        const bool whole = round == 1 || a >= n;
        const int w0 = min(lo + warp * run, hi), w1 = min(w0 + run, hi);
        uint64_t sum;
        if (qrow && !whole) sum = run_sum(w0, w1, std::true_type{});
        else sum = run_sum(w0, w1, std::false_type{});
        if (!whole && gone >= w0 && gone < w1 && lane == 0) sum -= weight(static_cast<int>(gone), true);
        sum = warp_sum_u64(sum);
        if (lane == 0) warp_total[warp] = sum;
        if (round == 0) cluster.sync(); else __syncthreads();   // warp totals; every CTA of the cluster runs
        uint64_t total = 0;
        for (int i = 0; i < kVtWarps; ++i) total += warp_total[i];
        if (tid < C) *cluster.map_shared_rank(&peers[round][c], tid) = total;
        cluster.sync();
        uint64_t T = 0, before = 0;
        for (int i = 0; i < C; ++i) {
            if (i < c) before += peers[round][i];
            T += peers[round][i];
        }
        if (T == 0) {                                           // the same for the whole cluster
            if (!whole) continue;
            if (c == 0 && tid == 0) out[a] = -1;                // no token has any probability
            break;
        }
        const float us = u[p.S];
        const uint64_t U = min(static_cast<uint32_t>(fminf(fmaxf(us, 0.f), 1.f) * 16777216.f), 16777215u);
        const uint64_t t = U * (T >> 32) * 256 + (U * (T & 0xFFFFFFFFull) >> 24);
        if (t < before || t >= before + total) break;      // another CTA of the cluster has it
        // the run that holds it, then the element: each thread a few consecutive ones
        uint64_t at = before;
        int w = 0;
        while (w < kVtWarps - 1 && t >= at + warp_total[w]) at += warp_total[w++];
        const int r0 = min(lo + w * run, hi), r1 = min(r0 + run, hi);
        const int each = (r1 - r0 + kVtThreads - 1) / kVtThreads;
        const int e0 = min(r0 + tid * each, r1), e1 = min(e0 + each, r1);
        uint64_t mine = 0;
        for (int v = e0; v < e1; ++v) mine += weight(v, whole);
        uint64_t scan = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t y = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += y;
        }
        __syncthreads();
        if (lane == 31) warp_total[warp] = scan;
        __syncthreads();
        for (int i = 0; i < warp; ++i) at += warp_total[i];
        at += scan - mine;
        if (t >= at && t < at + mine) {
            int v = e0;
            for (;; ++v) {
                const uint64_t x = weight(v, whole);
                if (t < at + x || v == e1 - 1) break;
                at += x;
            }
            out[a] = v;
        }
        break;
    }
}

}  // namespace ralm
