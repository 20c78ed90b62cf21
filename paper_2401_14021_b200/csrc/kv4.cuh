// A key-value cache held in 4 bits: layout, append and read.
//
// A page holds `ps` tokens of every key-value head; per head
//     [K codes: ps * D / 2][V codes: ps * D / 2][K (scale, offset): ps * 4][V (scale, offset): ps * 4]
// bytes. A vector x of a token and head is held as
//     s = fp16((max x - min x) / 15),  b = fp16(min x + 8 s),  c = clamp(rint((x - b) / s) + 8, 0, 15)
// and stands for s (c - 8) + b. K codes lie token by token, dimension 2i in the low half of byte i.
// V codes lie in blocks of 16 tokens in the order in which a warp's matrix instruction wants them:
// token 8c + 2t + e of the block has dimension g + 8j as nibble j of the D / 16 bytes at [c][g][t][e],
// so that lane 4g + t finds its operands in consecutive bytes and each token owns whole bytes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "common.cuh"
#include "mix.cuh"
#include "pages.cuh"

namespace ralm {

constexpr float kKvLimit = 57344.f;     // values saturate here, so that s (c - 8) + b stays finite in fp16
constexpr int kKvThreads = 256;

struct KvParams {
    unsigned char *layer;     // pool + layer * layer_stride
    int64_t page_bytes;
    const int32_t *table, *lengths, *refs;
    int32_t *status;
    int table_rows, max_pages, pages, page_size, heads;
    const int32_t *rows;      // table row of each batch entry, or null: the entry's own number
    int batch;
};

// The table row of batch entry b, or -1 (and the status word) if there is none.
__device__ __forceinline__ int kv_row(const KvParams &p, int b) {
    const int row = p.rows ? p.rows[b] : b;
    if (row >= 0 && row < p.table_rows) return row;
    atomicMax(p.status, kStatusInvalid);
    return -1;
}
__device__ __forceinline__ int kv_length(const KvParams &p, int row) {
    const long long cap = static_cast<long long>(p.max_pages) * p.page_size;
    return static_cast<int>(min(static_cast<long long>(max(p.lengths[row], 0)), cap));
}

struct KvTokens {
    const void *k, *v;                       // append: source; read: destination
    int64_t k_b, k_n, k_h, v_b, v_n, v_h;    // strides in elements; the last dimension is contiguous
    int n;
    const int32_t *starts, *count;           // count may be null: n tokens for every entry
};

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }

__device__ __forceinline__ float kv_clean(float x) {   // NaN counts as zero
    return x != x ? 0.f : fminf(fmaxf(x, -kKvLimit), kKvLimit);
}
__device__ __forceinline__ uint32_t kv_code(float x, float b, float inv) {
    return static_cast<uint32_t>(fminf(fmaxf(rintf(__fmul_rn(__fsub_rn(x, b), inv)) + 8.f, 0.f), 15.f));
}
// offset of a token's D / 16 bytes of V codes for g, in a head's V codes
template <int D> __device__ __forceinline__ int kv_v_offset(int slot, int g) {
    const int s = slot & 15;
    return (slot >> 4) * (8 * D) + (s >> 3) * (4 * D) + g * (D / 2) + ((s & 7) >> 1) * (D / 8) + (s & 1) * (D / 16);
}

// Where token `i` of batch entry `b` lives, or null if it is not to be touched.
template <int D>
__device__ __forceinline__ unsigned char *kv_token(const KvParams &p, const KvTokens &t, int b, int i, int h, bool write, int *slot) {
    const int row = kv_row(p, b);
    if (row < 0) return nullptr;
    const int64_t pos = static_cast<int64_t>(t.starts[b]) + i;
    if (pos < 0 || pos >= kv_length(p, row)) {
        if (write) atomicMax(p.status, kStatusInvalid);
        return nullptr;
    }
    const int page = p.table[static_cast<int64_t>(row) * p.max_pages + pos / p.page_size];
    if (page < 0 || page >= p.pages || (write && p.refs[page] != 1)) {   // a shared page is never written
        atomicMax(p.status, kStatusInvalid);
        return nullptr;
    }
    *slot = static_cast<int>(pos % p.page_size);
    return p.layer + page * p.page_bytes + static_cast<int64_t>(h) * p.page_size * (D + 8);
}

// One warp per token and head.
template <typename T, int D>
__global__ void __launch_bounds__(kKvThreads)
kv_append_kernel(const KvParams p, const KvTokens t) {
    constexpr int E = D / 32;                // elements per lane
    const int lane = threadIdx.x & 31;
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kKvThreads / 32);
    const int64_t jobs = static_cast<int64_t>(p.batch) * t.n * p.heads;
    for (int64_t job = static_cast<int64_t>(blockIdx.x) * (kKvThreads / 32) + (threadIdx.x >> 5); job < jobs; job += warps) {
        const int h = static_cast<int>(job % p.heads);
        const int i = static_cast<int>(job / p.heads % t.n);
        const int b = static_cast<int>(job / p.heads / t.n);
        if (t.count && i >= t.count[b]) continue;
        int slot;
        unsigned char *base = kv_token<D>(p, t, b, i, h, true, &slot);
        if (!base) continue;
        const int ps = p.page_size;
        const T *src[2] = {static_cast<const T *>(t.k) + b * t.k_b + i * t.k_n + h * t.k_h,
                           static_cast<const T *>(t.v) + b * t.v_b + i * t.v_n + h * t.v_h};
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            // K: dimensions E * lane ..; V: g + 8 j with g = lane / 4, j = E * (lane % 4) ..
            float x[E], lo = INFINITY, hi = -INFINITY;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int d = which == 0 ? E * lane + j : (lane >> 2) + 8 * (E * (lane & 3) + j);
                x[j] = kv_clean(to_float(src[which][d]));
                lo = fminf(lo, x[j]);
                hi = fmaxf(hi, x[j]);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
                hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
            }
            const __half s = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f));
            const float sf = __half2float(s);
            const __half off = __float2half_rn(__fadd_rn(lo, 8.f * sf));
            const float inv = sf > 0.f ? __frcp_rn(sf) : 0.f, bf = __half2float(off);
            uint32_t codes = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) codes |= kv_code(x[j], bf, inv) << (4 * j);
            unsigned char *at = which == 0 ? base + slot * (D / 2) + lane * (E / 2)
                                           : base + ps * (D / 2) + kv_v_offset<D>(slot, lane >> 2) + (lane & 3) * (E / 2);
            if (E == 4) *reinterpret_cast<uint16_t *>(at) = static_cast<uint16_t>(codes);
            else *at = static_cast<unsigned char>(codes);
            if (lane == 0)
                *reinterpret_cast<__half2 *>(base + ps * (which == 0 ? D : D + 4) + slot * 4) = __halves2half2(s, off);
        }
    }
}

// The values that tokens starts[b] .. starts[b] + n - 1 stand for; zeros beyond a row's length.
template <typename T, int D>
__global__ void __launch_bounds__(kKvThreads)
kv_read_kernel(const KvParams p, const KvTokens t) {
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31;
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kKvThreads / 32);
    const int64_t jobs = static_cast<int64_t>(p.batch) * t.n * p.heads;
    for (int64_t job = static_cast<int64_t>(blockIdx.x) * (kKvThreads / 32) + (threadIdx.x >> 5); job < jobs; job += warps) {
        const int h = static_cast<int>(job % p.heads);
        const int i = static_cast<int>(job / p.heads % t.n);
        const int b = static_cast<int>(job / p.heads / t.n);
        int slot = 0;
        const unsigned char *base = kv_token<D>(p, t, b, i, h, false, &slot);
        const int ps = p.page_size;
        T *dst[2] = {static_cast<T *>(const_cast<void *>(t.k)) + b * t.k_b + i * t.k_n + h * t.k_h,
                     static_cast<T *>(const_cast<void *>(t.v)) + b * t.v_b + i * t.v_n + h * t.v_h};
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            uint32_t codes = 0;
            float2 pair = make_float2(0.f, 0.f);
            if (base) {
                const unsigned char *at = which == 0 ? base + slot * (D / 2) + lane * (E / 2)
                                                     : base + ps * (D / 2) + kv_v_offset<D>(slot, lane >> 2) + (lane & 3) * (E / 2);
                codes = E == 4 ? *reinterpret_cast<const uint16_t *>(at) : *at;
                pair = __half22float2(*reinterpret_cast<const __half2 *>(base + ps * (which == 0 ? D : D + 4) + slot * 4));
            }
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int d = which == 0 ? E * lane + j : (lane >> 2) + 8 * (E * (lane & 3) + j);
                dst[which][d] = from_float<T>((static_cast<float>(codes >> (4 * j) & 15) - 8.f) * pair.x + pair.y);
            }
        }
    }
}

}  // namespace ralm
