// A key-value cache held in 4 bits: layout, append and read.
//
// A page holds `ps` tokens of every key-value head; per head
//     [K codes: ps * D / 2][V codes: ps * D / 2][K (scale, offset): ps * 4][V (scale, offset): ps * 4]
// bytes. A vector x of a token and head is held as
//     s = fp16((max x - min x) / 15),  b = fp16(min x + 8 s),  c = clamp(rint((x - b) / s) + 8, 0, 15)
// (in 32 bits; the divisions are products with 1 / 15 and 1 / s as rounded to 32 bits) and stands for s (c - 8) + b. K codes lie token by token, dimension 2i in the low half of byte i.
// V codes lie in blocks of 16 tokens in the order in which a warp's matrix instruction wants them:
// token 8c + 2t + e of the block has dimension g + 8j as nibble j of the D / 16 bytes at [c][g][t][e],
// so that lane 4g + t finds its operands in consecutive bytes and each token owns whole bytes.
//
// Append and read are bound by memory, 2.3 times the cache's bytes for 16-bit tensors, and close behind by
// instructions (about five per value to quantise). Measured (16 x 509 tokens, 32 heads of 128, bf16): append 43 us
// (issue slots 73 % used) and read 29 us, 72 to 74 us together, 4.6 TB/s, 0.71 of the measured copy bandwidth; 210 us with
// a warp per token, whose V codes left in pieces of two bytes. One token for each of 8 requests and back: 6.3 us for both
// launches.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

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
    int table_rows, max_pages, pages, page_size, page_shift, heads;
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
    int vec;                                 // every vector is 16-byte aligned
};

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }

__device__ __forceinline__ float kv_clean(float x) {   // NaN counts as zero
    return x != x ? 0.f : fminf(fmaxf(x, -kKvLimit), kKvLimit);
}
// offset of a token's D / 16 bytes of V codes for g, in a head's V codes
template <int D> __device__ __forceinline__ int kv_v_offset(int slot, int g) {
    const int s = slot & 15;
    return (slot >> 4) * (8 * D) + (s >> 3) * (4 * D) + g * (D / 2) + ((s & 7) >> 1) * (D / 8) + (s & 1) * (D / 16);
}

// D / 16 lanes share a token's vector, 16 consecutive dimensions each. For K their codes are 8 consecutive
// bytes. For V a lane's codes are one byte, its own, of each of the 8 groups g: the lanes of a token turn
// rows into columns among themselves, so that each then holds whole groups.
// D = 128: 8 lanes with 8 bytes each, a square; the same steps lead back.
__device__ __forceinline__ uint2 kv_transpose8(uint2 x, int lane) {
    const bool b2 = lane & 4, b1 = lane & 2, b0 = lane & 1;
    const uint32_t got2 = __shfl_xor_sync(0xffffffffu, b2 ? x.x : x.y, 4), kept2 = b2 ? x.y : x.x;
    const uint32_t r0 = b2 ? got2 : kept2, r1 = b2 ? kept2 : got2;
    const uint32_t lo = __byte_perm(r0, r1, 0x5410), hi = __byte_perm(r0, r1, 0x7632);
    const uint32_t got1 = __shfl_xor_sync(0xffffffffu, b1 ? lo : hi, 2), kept1 = b1 ? hi : lo;
    const uint32_t u0 = b1 ? got1 : kept1, u1 = b1 ? kept1 : got1;
    const uint32_t even = __byte_perm(u0, u1, 0x6420), odd = __byte_perm(u0, u1, 0x7531);
    const uint32_t got0 = __shfl_xor_sync(0xffffffffu, b0 ? even : odd, 1), kept0 = b0 ? odd : even;
    const uint32_t w0 = b0 ? got0 : kept0, w1 = b0 ? kept0 : got0;
    return make_uint2(__byte_perm(w0, w1, 0x6240), __byte_perm(w0, w1, 0x7351));
}
// D = 64: 4 lanes with 8 bytes each; lane q then holds the 4 bytes of groups 2 q (x) and 2 q + 1 (y).
__device__ __forceinline__ uint2 kv_transpose4(uint2 x, int lane) {
    const bool b1 = lane & 2, b0 = lane & 1;
    const uint32_t got1 = __shfl_xor_sync(0xffffffffu, b1 ? x.x : x.y, 2), kept1 = b1 ? x.y : x.x;
    const uint32_t r0 = b1 ? got1 : kept1, r1 = b1 ? kept1 : got1;
    const uint32_t lo = __byte_perm(r0, r1, 0x5410), hi = __byte_perm(r0, r1, 0x7632);
    const uint32_t got0 = __shfl_xor_sync(0xffffffffu, b0 ? lo : hi, 1), kept0 = b0 ? hi : lo;
    const uint32_t w0 = b0 ? got0 : kept0, w1 = b0 ? kept0 : got0;
    return make_uint2(__byte_perm(w0, w1, 0x6240), __byte_perm(w0, w1, 0x7351));
}
__device__ __forceinline__ uint2 kv_transpose4_back(uint2 x, int lane) {
    const bool b1 = lane & 2, b0 = lane & 1;
    const uint32_t lo = __byte_perm(x.x, x.y, 0x5410), hi = __byte_perm(x.x, x.y, 0x7632);
    const uint32_t got1 = __shfl_xor_sync(0xffffffffu, b1 ? lo : hi, 2), kept1 = b1 ? hi : lo;
    const uint32_t u0 = b1 ? got1 : kept1, u1 = b1 ? kept1 : got1;
    const uint32_t even = __byte_perm(u0, u1, 0x6420), odd = __byte_perm(u0, u1, 0x7531);
    const uint32_t got0 = __shfl_xor_sync(0xffffffffu, b0 ? even : odd, 1), kept0 = b0 ? odd : even;
    const uint32_t w0 = b0 ? got0 : kept0, w1 = b0 ? kept0 : got0;
    return make_uint2(__byte_perm(w0, w1, 0x5410), __byte_perm(w0, w1, 0x7632));
}

template <typename T> struct KvVec { union { uint4 raw[2]; T x[16]; }; };

// A warp takes one block of 16 positions (a multiple of 16 and on, so one page) of one entry and head, 512 / D
// tokens at a time; their codes fill whole sectors of the page.
template <int D> struct KvBlock {
    static constexpr int kLanes = D / 16, kTokens = 32 / kLanes, kSteps = 16 / kTokens;
    int b, h, first, count;    // first: number in the entry's list of the block's first position; it takes those in 0 .. count - 1
    int inside;                // of them, the numbers below this lie in the row
    int slot;
    unsigned char *base;       // the head's part of the page, or null
    __device__ __forceinline__ KvBlock(const KvParams &p, const KvTokens &t, uint32_t job, uint32_t blocks, bool write) {
        const uint32_t rest = job / static_cast<uint32_t>(p.heads);
        h = static_cast<int>(job - rest * p.heads);
        b = static_cast<int>(rest / blocks);
        const int start = t.starts[b];
        const int64_t pos = (static_cast<int64_t>(start) & ~int64_t{15}) + static_cast<int>(rest - b * blocks) * 16;
        first = static_cast<int>(pos - start);
        count = t.count ? min(t.count[b], t.n) : t.n;
        base = nullptr;
        inside = 0;
        slot = 0;
        const int lo = max(first, 0), hi = min(first + 16, count);  // the entry's tokens that the block takes
        if (lo >= hi) return;                                       // none: nothing to refuse either
        const int row = kv_row(p, b);
        if (row < 0) return;
        inside = static_cast<int>(min(max(static_cast<int64_t>(kv_length(p, row)) - start, int64_t{0}), static_cast<int64_t>(count)));
        if (write && (hi > inside || pos < 0)) atomicMax(p.status, kStatusInvalid);   // 0 is a block's first position
        if (lo >= inside || pos < 0) return;
        const int page = p.table[static_cast<int64_t>(row) * p.max_pages + (pos >> p.page_shift)];
        if (page < 0 || page >= p.pages || (write && p.refs[page] != 1)) {   // a shared page is never written
            atomicMax(p.status, kStatusInvalid);
            return;
        }
        slot = static_cast<int>(pos) & (p.page_size - 1);
        base = p.layer + page * p.page_bytes + static_cast<int64_t>(h) * p.page_size * (D + 8);
    }
};
__host__ __device__ __forceinline__ int kv_blocks(int n) { return (n + 14) / 16 + 1; }   // blocks that n positions can touch

// Smallest and largest of 16 values, two at a time in their own type; NaN if one is NaN.
__device__ __forceinline__ void kv_range(const KvVec<__half> &v, float &lo, float &hi) {
    const __half2 *h = reinterpret_cast<const __half2 *>(v.x);
    __half2 a = h[0], b = h[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) a = __hmin2_nan(a, h[j]), b = __hmax2_nan(b, h[j]);
    const float2 x = __half22float2(a), y = __half22float2(b);
    lo = x.x != x.x || x.y != x.y ? NAN : fminf(x.x, x.y);
    hi = fmaxf(y.x, y.y);
}
__device__ __forceinline__ void kv_range(const KvVec<__nv_bfloat16> &v, float &lo, float &hi) {
    const __nv_bfloat162 *h = reinterpret_cast<const __nv_bfloat162 *>(v.x);
    __nv_bfloat162 a = h[0], b = h[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) a = __hmin2_nan(a, h[j]), b = __hmax2_nan(b, h[j]);
    const float2 x = __bfloat1622float2(a), y = __bfloat1622float2(b);
    lo = x.x != x.x || x.y != x.y ? NAN : fminf(x.x, x.y);
    hi = fmaxf(y.x, y.y);
}

// Quantises 16 values of a vector that D / 16 lanes share: codes in nibbles, low first, and (s, b).
template <typename T, int D> __device__ __forceinline__ uint2 kv_quantise(const KvVec<T> &v, __half2 *pair) {
    float x[16], lo, hi;
    kv_range(v, lo, hi);
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = to_float(v.x[j]);
    if (!(lo >= -kKvLimit && hi <= kKvLimit)) {            // also where lo is NaN
        lo = INFINITY, hi = -INFINITY;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            x[j] = kv_clean(x[j]);
            lo = fminf(lo, x[j]);
            hi = fmaxf(hi, x[j]);
        }
    }
#pragma unroll
    for (int o = 1; o < D / 16; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const __half s = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f));
    const float sf = __half2float(s);
    const __half off = __float2half_rn(__fadd_rn(lo, 8.f * sf));
    const float inv = sf > 0.f ? __frcp_rn(sf) : 0.f, bf = __half2float(off);
    *pair = __halves2half2(s, off);
    // rint by adding 1.5 2^23, which leaves the code (+ 8) in the last bits; the constant's bits are taken off
    // the packed word as a whole. The codes need clamping only where the rounding of b moved the range.
    constexpr float kMagic = 12582912.f + 8.f;
    constexpr uint32_t kBits = 0x4B400000u;
    const bool clamp = !(__fmul_rn(__fsub_rn(hi, bf), inv) < 7.5f && __fmul_rn(__fsub_rn(lo, bf), inv) > -8.5f);
    uint32_t word[2];
    auto encode = [&](auto clamp_type) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            uint32_t packed = 0, extra = 0;
#pragma unroll
            for (int j = 7; j >= 0; --j) {
                float c = __fmul_rn(__fsub_rn(x[8 * w + j], bf), inv);
                if (decltype(clamp_type)::value) c = fminf(fmaxf(c, -8.f), 7.f);
                packed = packed * 16u + __float_as_uint(__fadd_rn(c, kMagic));
                extra = extra * 16u + kBits;
            }
            word[w] = packed - extra;
        }
    };
    if (__any_sync(0xffffffffu, clamp)) encode(std::true_type{});
    else encode(std::false_type{});
    return make_uint2(word[0], word[1]);
}
// Nibbles of one lane's 16 dimensions -> its byte of each group g: dimension 16 p + i is nibble i / 8 of the byte of g = i % 8.
__device__ __forceinline__ uint2 kv_bytes_by_group(uint2 codes) {
    // word x holds i = 0 .. 7, word y i = 8 .. 15: byte g = x's nibble g | y's nibble g << 4
    const uint32_t lo = codes.x, hi = codes.y;
    const uint32_t even = (lo & 0x0F0F0F0Fu) | ((hi & 0x0F0F0F0Fu) << 4);          // g = 0, 2, 4, 6
    const uint32_t odd = ((lo >> 4) & 0x0F0F0F0Fu) | (hi & 0xF0F0F0F0u);            // g = 1, 3, 5, 7
    return make_uint2(__byte_perm(even, odd, 0x5140), __byte_perm(even, odd, 0x7362));
}
__device__ __forceinline__ uint2 kv_codes_by_dim(uint2 bytes) {                     // the way back
    const uint32_t even = __byte_perm(bytes.x, bytes.y, 0x6420), odd = __byte_perm(bytes.x, bytes.y, 0x7531);
    return make_uint2((even & 0x0F0F0F0Fu) | ((odd & 0x0F0F0F0Fu) << 4), ((even >> 4) & 0x0F0F0F0Fu) | (odd & 0xF0F0F0F0u));
}

__device__ __forceinline__ void kv_codes(uint32_t word, __half2 (&y)[4]) {             // c - 8 of nibbles (i, i + 4)
    uint32_t e1024, e64;
    asm volatile("mov.b32 %0, 0x64006400;" : "=r"(e1024));                              // kept in registers: mask and insert in one
    asm volatile("mov.b32 %0, 0x54005400;" : "=r"(e64));
    const uint32_t high = word >> 8;
    const uint32_t r[4] = {(word & 0x000F000Fu) | e1024, (word & 0x00F000F0u) | e64, (high & 0x000F000Fu) | e1024, (high & 0x00F000F0u) | e64};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        y[j] = __hsub2(*reinterpret_cast<const __half2 *>(&r[j]), __float2half2_rn(j % 2 == 0 ? 1032.f : 72.f));
}
// Values of the 8 codes of a word: nibbles i and i + 4 come out of one masking instruction as fp16 1024 + c or
// 64 + c; c - 8 is exact, and s (c - 8) + b is rounded once (fp16) or in 32 bits first (bf16).
__device__ __forceinline__ void kv_values(uint32_t word, __half2 pair, __half (&out)[8]) {
    const __half2 s = __half2half2(__low2half(pair)), b = __half2half2(__high2half(pair));
    __half2 y[4];
    kv_codes(word, y);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __half2 v = __hfma2(y[j], s, b);
        out[j] = __low2half(v);
        out[j + 4] = __high2half(v);
    }
}
__device__ __forceinline__ void kv_values(uint32_t word, __half2 pair, __nv_bfloat16 (&out)[8]) {
    const float2 f = __half22float2(pair);
    __half2 y[4];
    kv_codes(word, y);
    float x[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 c = __half22float2(y[j]);
        x[j] = fmaf(c.x, f.x, f.y);
        x[j + 4] = fmaf(c.y, f.x, f.y);
    }
#pragma unroll
    for (int j = 0; j < 8; j += 2) *reinterpret_cast<__nv_bfloat162 *>(&out[j]) = __floats2bfloat162_rn(x[j], x[j + 1]);
}

template <typename T, int D>
__global__ void __launch_bounds__(kKvThreads, 4)
kv_append_kernel(const KvParams p, const KvTokens t) {
    cudaGridDependencySynchronize();                     // what ran before in the stream has ended
    using Block = KvBlock<D>;
    const int lane = threadIdx.x & 31, part = lane % Block::kLanes;
    const int ps = p.page_size;
    const uint32_t blocks = kv_blocks(t.n), warps = gridDim.x * (kKvThreads / 32);
    const uint32_t jobs = static_cast<uint32_t>(p.batch) * blocks * p.heads;             // below 2^31
    for (uint32_t job = blockIdx.x * (kKvThreads / 32) + (threadIdx.x >> 5); job < jobs; job += warps) {
        const Block at(p, t, job, blocks, true);
        if (!at.base) continue;
        const T *src_k = static_cast<const T *>(t.k) + at.b * t.k_b + at.h * t.k_h + 16 * part;
        const T *src_v = static_cast<const T *>(t.v) + at.b * t.v_b + at.h * t.v_h + 16 * part;
        KvVec<T> in[2][2];                                     // K and V of this step and the next
        auto fetch = [&](int step) {
            const int i = at.first + step * Block::kTokens + lane / Block::kLanes;
            const bool mine = i >= 0 && i < at.inside;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                KvVec<T> &u = in[step & 1][which];
                const T *src = which == 0 ? src_k + i * t.k_n : src_v + i * t.v_n;
                u.raw[0] = u.raw[1] = make_uint4(0, 0, 0, 0);
                if (mine && t.vec) {
                    u.raw[0] = __ldcs(reinterpret_cast<const uint4 *>(src));
                    u.raw[1] = __ldcs(reinterpret_cast<const uint4 *>(src) + 1);
                } else if (mine) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) u.x[j] = src[j];
                }
            }
        };
        fetch(0);
#pragma unroll
        for (int step = 0; step < Block::kSteps; ++step) {
            if (step + 1 < Block::kSteps) fetch(step + 1);
            const int i0 = at.first + step * Block::kTokens;
            if (i0 + Block::kTokens <= 0 || i0 >= at.inside) continue;   // the same for the whole warp
            const int i = i0 + lane / Block::kLanes;
            const bool mine = i >= 0 && i < at.inside;
            const int slot = at.slot + step * Block::kTokens + lane / Block::kLanes;
            __half2 pair;
            const uint2 k = kv_quantise<T, D>(in[step & 1][0], &pair);
            if (mine) {
                *reinterpret_cast<uint2 *>(at.base + slot * (D / 2) + 8 * part) = k;
                if (part == 0) *reinterpret_cast<__half2 *>(at.base + ps * D + slot * 4) = pair;
            }
            const uint2 bytes = kv_bytes_by_group(kv_quantise<T, D>(in[step & 1][1], &pair));
            const uint2 v = D == 128 ? kv_transpose8(bytes, lane) : kv_transpose4(bytes, lane);
            if (mine) {
                unsigned char *codes = at.base + ps * (D / 2);
                if (D == 128) {
                    *reinterpret_cast<uint2 *>(codes + kv_v_offset<D>(slot, part)) = v;
                } else {
                    *reinterpret_cast<uint32_t *>(codes + kv_v_offset<D>(slot, 2 * part)) = v.x;
                    *reinterpret_cast<uint32_t *>(codes + kv_v_offset<D>(slot, 2 * part + 1)) = v.y;
                }
                if (part == 0) *reinterpret_cast<__half2 *>(at.base + ps * (D + 4) + slot * 4) = pair;
            }
        }
    }
}

// The values that tokens starts[b] .. starts[b] + n - 1 stand for; zeros beyond a row's length.
template <typename T, int D>
__global__ void __launch_bounds__(kKvThreads, 6)
kv_read_kernel(const KvParams p, const KvTokens t) {
    cudaGridDependencySynchronize();                     // what ran before in the stream has ended
    using Block = KvBlock<D>;
    const int lane = threadIdx.x & 31, part = lane % Block::kLanes;
    const int ps = p.page_size;
    const uint32_t blocks = kv_blocks(t.n), warps = gridDim.x * (kKvThreads / 32);
    const uint32_t jobs = static_cast<uint32_t>(p.batch) * blocks * p.heads;
    for (uint32_t job = blockIdx.x * (kKvThreads / 32) + (threadIdx.x >> 5); job < jobs; job += warps) {
        const Block at(p, t, job, blocks, false);
        T *dst_k = static_cast<T *>(const_cast<void *>(t.k)) + at.b * t.k_b + at.h * t.k_h + 16 * part;
        T *dst_v = static_cast<T *>(const_cast<void *>(t.v)) + at.b * t.v_b + at.h * t.v_h + 16 * part;
#pragma unroll
        for (int step = 0; step < Block::kSteps; ++step) {
            const int i0 = at.first + step * Block::kTokens;
            if (i0 + Block::kTokens <= 0 || i0 >= t.n) continue;
            const int i = i0 + lane / Block::kLanes;
            const int slot = at.slot + step * Block::kTokens + lane / Block::kLanes;
            uint2 code[2] = {make_uint2(0, 0), make_uint2(0, 0)};
            __half2 pair[2] = {__float2half2_rn(0.f), __float2half2_rn(0.f)};
            if (at.base && i >= 0 && i < at.inside) {
                const unsigned char *codes = at.base + ps * (D / 2);
                code[0] = *reinterpret_cast<const uint2 *>(at.base + slot * (D / 2) + 8 * part);
                if (D == 128) {
                    code[1] = *reinterpret_cast<const uint2 *>(codes + kv_v_offset<D>(slot, part));
                } else {
                    code[1].x = *reinterpret_cast<const uint32_t *>(codes + kv_v_offset<D>(slot, 2 * part));
                    code[1].y = *reinterpret_cast<const uint32_t *>(codes + kv_v_offset<D>(slot, 2 * part + 1));
                }
                pair[0] = *reinterpret_cast<const __half2 *>(at.base + ps * D + slot * 4);
                pair[1] = *reinterpret_cast<const __half2 *>(at.base + ps * (D + 4) + slot * 4);
            }
            code[1] = kv_codes_by_dim(D == 128 ? kv_transpose8(code[1], lane) : kv_transpose4_back(code[1], lane));
            if (i < 0 || i >= t.n) continue;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                T *dst = which == 0 ? dst_k + i * t.k_n : dst_v + i * t.v_n;
                union { KvVec<T> u; T eight[2][8]; } out;
                kv_values(code[which].x, pair[which], out.eight[0]);
                kv_values(code[which].y, pair[which], out.eight[1]);
                if (t.vec) {
                    __stcs(reinterpret_cast<uint4 *>(dst), out.u.raw[0]);
                    __stcs(reinterpret_cast<uint4 *>(dst) + 1, out.u.raw[1]);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) dst[j] = out.u.x[j];
                }
            }
        }
    }
}

}  // namespace ralm
