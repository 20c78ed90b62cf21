// Attention of a request's newest tokens over its 4-bit cache:
//     out = softmax(scale q.k) v over the keys that the query may see.
//
// With k = s_k (c - 8) + b_k the score is s_k q.c + (b_k - 8 s_k) sum(q), and the output is
// sum (p s_v)(c - 8) + sum p b_v: the matrix instructions see whole numbers, and the scales enter in 32 bits.
// For the first product a code needs no conversion: four bits in the lowest places of an fp16 word ARE the number
// c 2^-24, and in the next four c 2^-20, subnormals that the instructions take exactly. One masking instruction makes an
// operand of two codes; the powers of two go into q and the results. The instructions line addends up by their exponents,
// and a subnormal's counts as 2^-14: sums keep 2^-14 of a step of the code times the largest |q|, measured 2^-23.1 of
// sum |q c| at worst over 128 dimensions (2^-24.2 with normal numbers, one more instruction an operand).
// In the second product the addends differ by far more, by the weights of a softmax: there the operand is c - 8 as a normal
// number, two instructions shared by all query rows, and what is small beside the largest weight of a tile is not cut off.
// The weights p s_v are rounded to fp16 (11 bits) before the second product; maxima, sums and outputs stay in
// 32 bits. The error against 64 bits of an fp16 output is 2.7e-4 of its size with that and 2.1e-4 without (the output's
// own rounding, which in bf16 hides the weights' altogether); the cut-off bits as a second fp16 operand would cost 12 %
// of a decode step and 20 % of a verification. What p is relative to is, for each query row, the largest p s_v, not the
// largest p: the weights that count lie high in fp16's range whatever the sizes of the values, and one large value that
// does not count for a row costs it nothing (2^22 lie between the largest weight and the first that loses bits).
//
// A warp is a worker with its own stages in shared memory (bulk copies of 32 tokens, completion on a
// barrier of its own): no warp waits for another, and any mix of lengths keeps all of them busy.
//
// Orientation: keys are the rows of the instructions (m16n8k16) and query rows the columns, so that a
// decode step with up to 8 query rows per key-value head fills one column block, and the codes go from
// 16-byte loads to operand registers without passing through shared memory.
//
// Bound, with up to 8 query rows per key-value head, by the cache's bytes (136 a token and head of 128) and by
// issue slots at almost the same rate: a tile of 16 tokens is 2176 bytes, 90 cycles of an SM's share of the memory
// bandwidth, and about 265 instructions, 66 cycles of its four schedulers at best. Measured (32 requests of 2000 to
// 32000 tokens, 8 heads of 128): 1 row 127 us, 8 rows 133 us (4.6 and 4.5 TB/s, 0.72 and 0.69 of the measured copy
// bandwidth); 16 rows 206 us, 24 rows 260 us, 32 rows 364 us, 36 rows (two passes) 461 us, bound by the 16 matrix
// instructions and 50 others that 8 more rows cost a tile, at the rate that two to three warps a scheduler reach (issue
// slots 39 % used, matrix pipe 33 %). With 64 dimensions (64 requests of 500 to 8000 tokens, 32 heads) 162 us, 0.60 of
// the copy bandwidth: half the bytes for more than half the instructions. Steps: codes loaded into registers from
// global memory 215 us; bulk copies of whole pages, one per 64 tokens 154 us; two tiles side by side 145 us; K's codes as
// subnormals instead of converting them 125 us. Small calls are latency: 7.1 us for four requests of 64 tokens, of
// which 1 is the launch, 1.4 the cut of the work, 1 the first pages, 1.7 the queries. In between the join counts: of
// 24.8 us for 16 requests of up to 4600 tokens (8 heads, 4 rows) 3 are spent in the CTA and 5 between CTAs.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "common.cuh"
#include "kv4.cuh"
#include "mix.cuh"

namespace ralm {

constexpr int kAttendMaxBatch = 4096;
constexpr int kAttendStage = 64;         // tokens of a stage in shared memory, the largest unit of work
constexpr float kAttendLazy = 6.f;       // a maximum may be this far (powers of two) behind before sums are rescaled
constexpr float kAttendBias = 8.f;       // exponent added to the weights: 2^(6 + 8 + 1) is below fp16's largest

// Warps per CTA (one CTA per SM) and whether the query operands stay in registers, by column blocks.
__host__ __device__ constexpr int attend_warps(int nt, int d) { return nt >= 3 ? 8 : nt == 1 && d == 64 ? 16 : 12; }
__host__ __device__ constexpr bool attend_q_in_regs(int nt) { return nt == 1; }
// Shared memory of a warp: stages of kAttendStage tokens and, where they are not in registers, the queries. With two
// column blocks of 128 dimensions there is room for one stage only (the other warps work while it is filled):
// 208 us on 32 x 8 heads of 2000 to 32000 tokens with 16 rows, against 203 to 213 with 8 warps and two stages, but
// 77 us against 80 to 90 on 64 x 32 heads of 700 with 9.
__host__ __device__ constexpr int attend_stage_bytes(int d) { return kAttendStage * (d + 8); }
__host__ __device__ constexpr int attend_q_bytes(int nt, int d) { return attend_q_in_regs(nt) ? 0 : 16 * nt * d; }
constexpr int kAttendSmem = 210 * 1024;  // for the warps; the prefix sums and static variables take the rest
__host__ __device__ constexpr int attend_stages(int nt, int d) {
    const int fit = (kAttendSmem / attend_warps(nt, d) - attend_q_bytes(nt, d)) / attend_stage_bytes(d);
    return fit > 4 ? 4 : fit;
}
__host__ __device__ constexpr int attend_warp_bytes(int nt, int d) {
    return attend_stages(nt, d) * attend_stage_bytes(d) + attend_q_bytes(nt, d);
}
static_assert(attend_stages(1, 128) >= 2 && attend_stages(3, 128) >= 2 && attend_stages(4, 128) >= 2 && attend_stages(1, 64) >= 2 &&
                  attend_stages(4, 64) >= 2,
              "one stage is read while another is on its way");
// A warp's partial result (rows of D + 4 floats: values, maximum, sum) fits where its stages were.
__host__ __device__ constexpr int attend_row_floats(int d) { return d + 4; }
static_assert(attend_stages(2, 128) * attend_stage_bytes(128) >= 16 * attend_row_floats(128) * 4 &&
                  attend_stages(4, 128) * attend_stage_bytes(128) >= 32 * attend_row_floats(128) * 4 &&
                  attend_stages(4, 64) * attend_stage_bytes(64) >= 32 * attend_row_floats(64) * 4,
              "partial results");

struct AttendParams {
    KvParams kv;
    const void *q;
    void *out;
    int64_t q_b, q_n, q_h, o_b, o_n, o_h;
    const int32_t *q_len;     // or null: n queries for every entry
    int n, group;             // queries per entry; query heads per key-value head
    int row_blocks;           // blocks of 8 * NT query rows
    float scale;              // softmax scale * log2(e)
    float *part, *part_ml;    // per warp [2 * workers][8 * NT][D] partial outputs and [..][2] their maxima and sums
    float *cta_part, *cta_ml; // the same per CTA
    int *counters;            // [CTAs], zero between calls
    int workers;
    int vec;                  // q is 16-byte aligned in every row
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t hsub2(uint32_t a, uint32_t b) {
    const __half2 r = __hsub2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
// The four pairs (nibble i of the low half, nibble i of the high half) of a word as fp16 numbers: c 2^-24
// for i = 0 and 2, c 2^-20 for i = 1 and 3.
__device__ __forceinline__ void unpack4(uint32_t x, uint32_t (&y)[4]) {
    const uint32_t z = x >> 8;
    y[0] = x & 0x000F000Fu;
    y[1] = x & 0x00F000F0u;
    y[2] = z & 0x000F000Fu;
    y[3] = z & 0x00F000F0u;
}

// c - 8 of the same pairs, as normal numbers: 1024 + c and 64 + c are a mask and an exponent away, the difference is exact.
// The exponents come out of a shuffle so that the compiler holds them in ordinary registers, where mask and exponent are
// one instruction (32 x 8 heads of 2000 to 32000 tokens: 129 us, 138 with two).
struct Exponents {
    uint32_t e1024, e64, e23;
    __device__ __forceinline__ Exponents() {
        e1024 = __shfl_sync(0xffffffffu, 0x64006400u, threadIdx.x & 31);
        e64 = __shfl_sync(0xffffffffu, 0x54005400u, threadIdx.x & 31);
        e23 = __shfl_sync(0xffffffffu, 0x4B000000u, threadIdx.x & 31);
    }
    __device__ __forceinline__ void unpack4(uint32_t x, uint32_t (&y)[4]) const {
        const uint32_t z = x >> 8;
        y[0] = hsub2((x & 0x000F000Fu) | e1024, 0x64086408u);
        y[1] = hsub2((x & 0x00F000F0u) | e64, 0x54805480u);
        y[2] = hsub2((z & 0x000F000Fu) | e1024, 0x64086408u);
        y[3] = hsub2((z & 0x00F000F0u) | e64, 0x54805480u);
    }
    // floor(log2 x), x the fp16 number in the low half of a word; -15 for zero and subnormals. The exponent's bits, put
    // behind those of 2^23.
    __device__ __forceinline__ float log2_floor(uint32_t pair) const {
        return fmaf(__uint_as_float((pair & 0x7C00u) | e23), 1.f / 1024.f, -8207.f);   // 2^23 / 1024 + 15
    }
};

// The largest finite absolute value of eight; infinities and NaN do not set a row's scale.
__device__ __forceinline__ float q_top(const __half *x) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        const float2 a = __half22float2(__habs2(*reinterpret_cast<const __half2 *>(x + j)));
        top = fmaxf(top, fmaxf(a.x < INFINITY ? a.x : 0.f, a.y < INFINITY ? a.y : 0.f));
    }
    return top;
}
__device__ __forceinline__ float q_top(const __nv_bfloat16 *x) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        const float2 a = __bfloat1622float2(__habs2(*reinterpret_cast<const __nv_bfloat162 *>(x + j)));
        top = fmaxf(top, fmaxf(a.x < INFINITY ? a.x : 0.f, a.y < INFINITY ? a.y : 0.f));
    }
    return top;
}

template <int D> struct LaneCodes;                                    // a lane's D / 8 bytes of a tile
template <> struct LaneCodes<128> { union { uint4 raw; uint32_t w[4]; }; };
template <> struct LaneCodes<64> { union { uint2 raw; uint32_t w[2]; }; };
template <int D> __device__ __forceinline__ void load_codes(LaneCodes<D> &c, const unsigned char *at) {
    c.raw = *reinterpret_cast<const decltype(c.raw) *>(at);
}

// How the work is cut: segments (entry, head, row block) follow one another, each `units` long (at least
// one, so that an entry without keys is written too), and worker w, a warp, takes units
// [total w / W, total (w + 1) / W): any mix of lengths is balanced to one unit. A unit is 64 tokens, or
// 32 where there are so few that the warps would get less than two of them each.
//
// Where every segment is short and there are CTAs enough, a segment is given a CTA of its own instead (its
// units cut over the CTA's warps): nothing is left to merge between CTAs, which costs more than the shares save.
struct Share {
    long long total;
    int workers, shift;                  // log2 of a unit's tokens
    bool own_cta;                        // one CTA per segment
    long long each, more;                // the first `more` workers take each + 1 units, the others `each`
    __device__ __forceinline__ void cut() {
        if (total < (1LL << 31)) {
            const uint32_t q = static_cast<uint32_t>(total) / static_cast<uint32_t>(workers);
            each = q;
            more = total - static_cast<long long>(q) * workers;
        } else {
            each = total / workers;
            more = total - each * workers;
        }
    }
    __device__ __forceinline__ long long begin(int w) const { return each * w + min(static_cast<long long>(w), more); }
    __device__ __forceinline__ int owner(long long u) const {
        const long long wide = more * (each + 1);
        if (total < (1LL << 31))
            return u < wide ? static_cast<int>(static_cast<uint32_t>(u) / static_cast<uint32_t>(each + 1))
                            : static_cast<int>(more) + static_cast<int>(static_cast<uint32_t>(u - wide) / static_cast<uint32_t>(each));
        return static_cast<int>(u < wide ? u / (each + 1) : more + (u - wide) / each);
    }
};
// own_cta: at most this many units of 32 tokens per warp. Measured on 8 requests x 8 heads, 8 query rows, up to 2000
// tokens (5 units a warp): 20.2 us against 23.1 cut over all CTAs; on 16 x 8 heads, up to 6000 tokens (16 units):
// 37.1 us against 29.6.
constexpr int kAttendOwnUnits = 8;
// Inclusive prefix sums of the entries' units (without heads and row blocks) in shared memory: cum[b + 1]
// for b < batch. Returns the whole.
__device__ inline int attend_prefix(const AttendParams &p, int shift, int *cum, int *scratch) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int carry = 0;
    for (int b0 = 0; b0 < p.kv.batch; b0 += blockDim.x) {
        const int b = b0 + tid;
        int units = 0;
        if (b < p.kv.batch) {
            const int row = kv_row(p.kv, b);
            units = row < 0 ? 1 : max((kv_length(p.kv, row) + (1 << shift) - 1) >> shift, 1);
        }
        int scan = units;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += y;
        }
        __syncthreads();
        if (lane == 31) scratch[warp] = scan;
        __syncthreads();
        int before = carry, all = 0;
        for (int i = 0; i < (int)(blockDim.x >> 5); ++i) {
            if (i < warp) before += scratch[i];
            all += scratch[i];
        }
        if (b < p.kv.batch) cum[b + 1] = before + scan;
        carry += all;
    }
    if (tid == 0) cum[0] = 0;
    __syncthreads();
    return carry;
}
__device__ inline Share attend_share(const AttendParams &p, int *cum, int *scratch) {
    const long long per = static_cast<long long>(p.kv.heads) * p.row_blocks;
    Share s;
    if (p.kv.batch <= (int)blockDim.x) {   // both cuts from one look at the lengths, packed in 64 bits
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        unsigned long long units = 0;
        bool brief = true;
        if (tid < p.kv.batch) {
            const int row = kv_row(p.kv, tid);
            const int len = row < 0 ? 0 : kv_length(p.kv, row);
            units = static_cast<unsigned long long>(max((len + 63) >> 6, 1)) << 32 | max((len + 31) >> 5, 1);
            brief = len <= 32 * kAttendOwnUnits * static_cast<int>(blockDim.x >> 5);
        }
        unsigned long long scan = units;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long y = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += y;
        }
        unsigned long long *sums = reinterpret_cast<unsigned long long *>(scratch);
        if (lane == 31) sums[warp] = scan;
        brief = __syncthreads_and(brief);
        unsigned long long before = 0, all = 0;
        const int warps = (p.kv.batch + 31) >> 5;
        for (int i = 0; i < warps; ++i) {
            if (i < warp) before += sums[i];
            all += sums[i];
        }
        s.shift = 6;
        s.total = static_cast<long long>(all >> 32) * per;
        s.own_cta = brief && p.kv.batch * per <= gridDim.x;
        if (s.own_cta || s.total < 2LL * p.workers) {
            s.shift = 5;
            s.total = static_cast<long long>(all & 0xFFFFFFFFull) * per;
        }
        const unsigned long long to = before + scan;
        if (tid < p.kv.batch) cum[tid + 1] = static_cast<int>(s.shift == 6 ? to >> 32 : to);
        if (tid == 0) cum[0] = 0;
        __syncthreads();
        s.workers = static_cast<int>(min(static_cast<long long>(p.workers), s.total));
        s.cut();
        return s;
    }
    s.own_cta = false;
    s.shift = 6;
    s.total = attend_prefix(p, 6, cum, scratch) * per;
    if (s.total < 2LL * p.workers) {
        s.shift = 5;
        s.total = attend_prefix(p, 5, cum, scratch) * per;
    }
    s.workers = static_cast<int>(min(static_cast<long long>(p.workers), s.total));
    s.cut();
    return s;
}
struct Segment { int b, h, rb, unit, units; };                     // unit: place inside the segment
__device__ __forceinline__ Segment attend_segment(const AttendParams &p, const int *cum, long long unit) {
    const int per = p.kv.heads * p.row_blocks;
    int lo = 0, hi = p.kv.batch - 1;
    while (lo < hi) {                                               // the last entry that begins at or before the unit
        const int mid = (lo + hi + 1) >> 1;
        if (static_cast<long long>(cum[mid]) * per <= unit) lo = mid; else hi = mid - 1;
    }
    Segment s;
    s.b = lo;
    s.units = cum[lo + 1] - cum[lo];
    const long long in = unit - static_cast<long long>(cum[lo]) * per;
    const int which = in < (1LL << 31) ? static_cast<int>(static_cast<uint32_t>(in) / static_cast<uint32_t>(s.units)) : static_cast<int>(in / s.units);
    s.unit = static_cast<int>(in - static_cast<long long>(which) * s.units);
    s.h = which / p.row_blocks;
    s.rb = which - s.h * p.row_blocks;
    return s;
}
__device__ __forceinline__ void attend_next(const AttendParams &p, const int *cum, Segment &s) {   // the segment after s
    s.unit = 0;
    if (++s.rb < p.row_blocks) return;
    s.rb = 0;
    if (++s.h < p.kv.heads) return;
    s.h = 0;
    if (++s.b < p.kv.batch) s.units = cum[s.b + 1] - cum[s.b];
}

// One query row's place in the output: query i and head of the group, from its number in the segment's entry.
template <typename T>
__device__ __forceinline__ T *attend_row(const AttendParams &p, const Segment &s, int row) {
    const int i = row / p.group, gq = row - i * p.group;
    return static_cast<T *>(p.out) + s.b * p.o_b + i * p.o_n + (static_cast<int64_t>(s.h) * p.group + gq) * p.o_h;
}

// A row's merged result: its values d of a lane's D / 32 dimensions, in units of 2^M, and the sum of weights.
template <int D> struct RowSum {
    float x[D / 32], M, L;
};
// Merges `count` pieces of one query row; a warp. A piece is a row of D values and a (maximum, sum), which the lanes
// keep for the first 32 pieces. This warp takes every `parts`-th piece, from `part` on; M is of all of them.
template <int D, typename Piece>
__device__ __forceinline__ RowSum<D> attend_merge(int count, int part, int parts, Piece piece_of, const float *values, const float *ml) {
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31;
    auto pair = [&](int j) { return j < count ? __ldcg(reinterpret_cast<const float2 *>(ml + 2 * piece_of(j))) : make_float2(-1e30f, 0.f); };
    RowSum<D> r;
    const float2 mine = pair(part + lane * parts);
    r.M = mine.x;
    if (parts > 1 || count > 32)
        for (int j = lane; j < count; j += 32) r.M = fmaxf(r.M, pair(j).x);
    r.M = warp_max(r.M);
    r.L = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) r.x[e] = 0.f;
    for (int j0 = part; j0 < count; j0 += 32 * parts) {
        const float2 p = j0 == part ? mine : pair(j0 + lane * parts);
        const float w = exp2_approx(p.x - r.M);                     // 0 where there is no piece
        r.L = fmaf(p.y, w, r.L);
        const int some = min(32, (count - j0 + parts - 1) / parts);
#pragma unroll 4
        for (int i = 0; i < some; ++i) {
            const float wi = __shfl_sync(0xffffffffu, w, i);
            const float *v = values + piece_of(j0 + i * parts) * D + E * lane;
            if (E == 4) {
                const float4 y = __ldcg(reinterpret_cast<const float4 *>(v));
                r.x[0] = fmaf(y.x, wi, r.x[0]), r.x[1] = fmaf(y.y, wi, r.x[1]);
                r.x[E - 2] = fmaf(y.z, wi, r.x[E - 2]), r.x[E - 1] = fmaf(y.w, wi, r.x[E - 1]);
            } else {
                const float2 y = __ldcg(reinterpret_cast<const float2 *>(v));
                r.x[0] = fmaf(y.x, wi, r.x[0]), r.x[1] = fmaf(y.y, wi, r.x[1]);
            }
        }
    }
    r.L = warp_sum(r.L);
    return r;
}
template <typename T, int D>
__device__ __forceinline__ void attend_write_row(const AttendParams &p, int segment, int rows_per_block, int lr, const RowSum<D> &r) {
    constexpr int E = D / 32;
    const int per = p.kv.heads * p.row_blocks;
    Segment s;
    s.b = segment / per;
    const int which = segment - s.b * per;
    s.h = which / p.row_blocks;
    s.rb = which - s.h * p.row_blocks;
    const int row = s.rb * rows_per_block + lr;
    if (row >= p.n * p.group) return;
    const float inv = r.L > 0.f ? 1.f / r.L : r.L == 0.f ? 0.f : NAN;
#pragma unroll
    for (int e = 0; e < E; ++e) attend_row<T>(p, s, row)[E * (threadIdx.x & 31) + e] = from_float<T>(r.x[e] * inv);
}

// One CTA per segment: the pieces of its `working` warps are in shared memory, where their stages were.
template <typename T, int D, int NT>
__device__ __forceinline__ void attend_join_near(const AttendParams &p, int working, const unsigned char *smem) {
    constexpr int WARPS = attend_warps(NT, D), ROWS = 8 * NT, E = D / 32, STRIDE = attend_warp_bytes(NT, D) / 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rows = min(p.n * p.group, ROWS);
    const float *base = reinterpret_cast<const float *>(smem);
    __syncthreads();
    for (int lr = warp; lr < rows; lr += WARPS) {
        const float *row = base + lr * attend_row_floats(D);
        const float2 ml = lane < working ? *reinterpret_cast<const float2 *>(row + lane * STRIDE + D) : make_float2(-1e30f, 0.f);
        RowSum<D> r;
        r.M = warp_max(ml.x);
        const float w = exp2_approx(ml.x - r.M);
        r.L = warp_sum(ml.y * w);
#pragma unroll
        for (int e = 0; e < E; ++e) r.x[e] = 0.f;
        for (int k = 0; k < working; ++k) {
            const float wk = __shfl_sync(0xffffffffu, w, k);
#pragma unroll
            for (int e = 0; e < E; ++e) r.x[e] = fmaf(row[k * STRIDE + 32 * e + lane], wk, r.x[e]);
        }
        // the lane's dimensions here are 32 e + lane
        const int per = p.kv.heads * p.row_blocks, segment = blockIdx.x;
        Segment s;
        s.b = segment / per;
        const int which = segment - s.b * per;
        s.h = which / p.row_blocks;
        s.rb = which - s.h * p.row_blocks;
        const int qr = s.rb * ROWS + lr;
        if (qr >= p.n * p.group) continue;
        const float inv = r.L > 0.f ? 1.f / r.L : r.L == 0.f ? 0.f : NAN;
        T *o = attend_row<T>(p, s, qr);
#pragma unroll
        for (int e = 0; e < E; ++e) o[32 * e + lane] = from_float<T>(r.x[e] * inv);
    }
}

// Brings the pieces of split segments together, in two steps. Inside a CTA: the warps' shares follow one
// another, so a segment's pieces belong to neighbouring warps; a segment that begins and ends in the CTA is
// written, of any other one piece per CTA is left. Across CTAs: each CTA that holds a piece of a segment
// counts itself at the segment's first CTA, and the one that finds the count complete merges (in the order of
// the CTAs, whoever it is) and puts the count back to zero.
//   open_piece[w]: warp w's last segment begins there and does not end: (1, segment), in piece 2 * worker + 1.
//   left_piece[w]: warp w's first segment began before it: (1, or 2 if it ends there, segment), piece 2 * worker.
template <typename T, int D, int NT>
__device__ __forceinline__ void attend_join(const AttendParams &p, const Share &share, const int *cum, int working, const int2 *open_piece,
                                            const int2 *left_piece, float *smem) {
    constexpr int WARPS = attend_warps(NT, D), ROWS = 8 * NT, E = D / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, cta = blockIdx.x;
    const int rows = min(p.n * p.group, ROWS);
    __syncthreads();
    const bool valid = lane < working;
    const uint32_t opens = __ballot_sync(0xffffffffu, valid && open_piece[lane < WARPS ? lane : 0].x != 0);
    const uint32_t ends = __ballot_sync(0xffffffffu, valid && left_piece[lane < WARPS ? lane : 0].x == 2);
    const bool carried = left_piece[0].x != 0;                         // the CTA's first segment began before it
    const int groups = __popc(opens) + (carried ? 1 : 0);
    bool last_open = false;                                            // a segment goes on in the next CTA
    for (int i = warp; i < groups * rows; i += WARPS) {
        int q = i / rows;
        const int lr = i - q * rows;
        const bool from_before = carried && q == 0;
        int leader = 0;
        if (!from_before) {
            q -= carried ? 1 : 0;
            uint32_t m = opens;
            for (; q > 0; --q) m &= m - 1;
            leader = __ffs(m) - 1;
        }
        const int begin = from_before ? 0 : leader + 1;                // first warp with a piece that it was left
        const uint32_t ending = begin < 32 ? ends >> begin : 0;
        const bool ended = ending != 0;
        const int until = ended ? begin + __ffs(ending) : working;      // one past the last warp of the segment
        const int count = until - begin + (from_before ? 0 : 1);
        const int64_t worker0 = static_cast<int64_t>(cta) * WARPS;
        auto piece_of = [&](int j) -> int64_t {
            if (from_before) return (2 * (worker0 + j)) * ROWS + lr;
            return (2 * (worker0 + leader + j) + (j == 0 ? 1 : 0)) * ROWS + lr;
        };
        const RowSum<D> r = attend_merge<D>(count, 0, 1, piece_of, p.part, p.part_ml);
        if (!from_before && ended) {
            attend_write_row<T, D>(p, open_piece[leader].y, ROWS, lr, r);
        } else {
            const int64_t at = (2LL * cta + (from_before ? 0 : 1)) * ROWS + lr;
            float *o = p.cta_part + at * D + E * lane;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = r.x[e];
            if (lane == 0) *reinterpret_cast<float2 *>(p.cta_ml + 2 * at) = make_float2(r.M, r.L);
        }
    }
    // the CTA's own pieces: of the segment that came in, and of the one that goes out (which may be the same)
    const int last_leader = 31 - __clz(opens);
    last_open = opens != 0 && (last_leader + 1 >= 32 || (ends >> (last_leader + 1)) == 0);
    __shared__ int merge[2], merge_from[2], merge_to[2];
    if (threadIdx.x < 2) merge[threadIdx.x] = 0;
    __syncthreads();
    // one thread each counts this CTA in at the first CTA of the segment that came in, and of the one that goes out
    if (threadIdx.x % 32 == 0 && threadIdx.x < 64) {
        const int turn = threadIdx.x / 32;
        if (turn == 0 ? carried : last_open) {
            const int segment = turn == 0 ? left_piece[0].y : open_piece[last_leader].y;
            const int per = p.kv.heads * p.row_blocks;
            const int b = segment / per, units = cum[b + 1] - cum[b];
            const long long first = static_cast<long long>(cum[b]) * per + static_cast<long long>(segment - b * per) * units;
            const int c0 = share.owner(first) / WARPS, c1 = share.owner(first + units - 1) / WARPS;
            // releases this CTA's pieces (the barrier above is before it) and acquires the others'
            int before;
            asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(before) : "l"(p.counters + c0) : "memory");
            if (before == c1 - c0) {
                p.counters[c0] = 0;
                merge[turn] = 1;
                merge_from[turn] = c0;
                merge_to[turn] = c1;
            }
        }
    }
    __syncthreads();
    for (int turn = 0; turn < 2; ++turn) {
        if (!merge[turn]) continue;                                     // the same for the whole CTA
        const int segment = turn == 0 ? left_piece[0].y : open_piece[last_leader].y;
        const int c0 = merge_from[turn], c1 = merge_to[turn];
        // few rows: several warps share a row, every parts-th piece each
        const int count = c1 - c0 + 1, parts = max(WARPS / rows, 1);
        for (int i0 = 0; i0 < rows * parts; i0 += WARPS) {
            const int i = i0 + warp, lr = i / parts, part = i - lr * parts;
            const bool busy = i < rows * parts;
            auto piece_of = [&](int j) -> int64_t { return (2LL * (c0 + j) + (j == 0 ? 1 : 0)) * ROWS + lr; };
            RowSum<D> r;
            if (busy) r = attend_merge<D>(count, part, parts, piece_of, p.cta_part, p.cta_ml);
            if (parts > 1) {
                if (busy) {
#pragma unroll
                    for (int e = 0; e < E; ++e) smem[warp * (D + 1) + E * lane + e] = r.x[e];
                    if (lane == 0) smem[warp * (D + 1) + D] = r.L;
                }
                __syncthreads();
                if (busy && part == 0)
                    for (int k = 1; k < parts; ++k) {
#pragma unroll
                        for (int e = 0; e < E; ++e) r.x[e] += smem[(warp + k) * (D + 1) + E * lane + e];
                        r.L += smem[(warp + k) * (D + 1) + D];
                    }
                __syncthreads();
            }
            if (busy && part == 0) attend_write_row<T, D>(p, segment, ROWS, lr, r);
        }
    }
}

// The stream of a worker's stages: which unit is asked for next. All lanes keep the same state except
// `held`, where lane i holds table entry base + i of the row that is being read.
struct AttendFeed {
    Segment seg;
    int units_left;            // of the worker
    int len, row, slot;        // slot: the stage that is filled next
    int held, base;
    __device__ __forceinline__ void enter(const AttendParams &p) {
        row = kv_row(p.kv, seg.b);
        len = row < 0 ? 0 : kv_length(p.kv, row);
        base = -64;
    }
    // Makes sure that entries index .. index + 3 are held.
    __device__ __forceinline__ void hold(const AttendParams &p, int index, int lane) {
        if (index >= base && index + 3 < base + 32) return;
        base = index;
        held = index + lane < p.kv.max_pages ? p.kv.table[static_cast<int64_t>(row) * p.kv.max_pages + index + lane] : 0;
        if (index + lane < ((len - 1) >> p.kv.page_shift) + 1 && (held < 0 || held >= p.kv.pages)) {
            atomicMax(p.kv.status, kStatusInvalid);
            held = 0;
        }
    }
};

template <typename T, int D, int NT>
__global__ void __launch_bounds__(attend_warps(NT, D) * 32, 1)
attend_kernel(const AttendParams p) {
    constexpr int WARPS = attend_warps(NT, D);
    constexpr int W = D / 32;            // words of K codes per lane and key; also dimensions / 32
    constexpr int MT = D / 16;           // row blocks of the output
    constexpr int ROWS = 8 * NT;
    constexpr int STAGES = attend_stages(NT, D);
    constexpr int STAGE = attend_stage_bytes(D);
    constexpr bool QREG = attend_q_in_regs(NT);
    constexpr int TILES = NT == 1 || NT == 3 ? 2 : 1;   // tiles that are worked on side by side, where registers allow it
    extern __shared__ __align__(128) unsigned char attend_smem[];
    __shared__ __align__(8) int scratch[64];
    __shared__ __align__(8) uint64_t bars[WARPS * STAGES];
    __shared__ int2 open_piece[WARPS], left_piece[WARPS];
    __shared__ __align__(8) float row_factor[WARPS][ROWS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    unsigned char *ring = attend_smem + warp * attend_warp_bytes(NT, D);
    uint4 *q_smem = reinterpret_cast<uint4 *>(ring + STAGES * STAGE);
    int *cum = reinterpret_cast<int *>(attend_smem + WARPS * attend_warp_bytes(NT, D));
    const uint32_t bar0 = smem_u32(&bars[warp * STAGES]), ring0 = smem_u32(ring);
    if (lane == 0) {
        for (int i = 0; i < STAGES; ++i) mbar_init(bar0 + 8 * i, 1);
        mbar_fence_init();
    }
    cudaGridDependencySynchronize();                     // what ran before in the stream has ended
    const Share share = attend_share(p, cum, scratch);
    const int worker = blockIdx.x * WARPS + warp;
    Segment mine_first;                  // where the warp begins, and how many units it takes
    int working, units;
    if (share.own_cta) {
        const int per = p.kv.heads * p.row_blocks, segment = blockIdx.x;
        if (segment >= p.kv.batch * per) return;                        // the whole CTA
        const int b = segment / per, which = segment - b * per, all = cum[b + 1] - cum[b];
        working = min(WARPS, all);
        mine_first.b = b;
        mine_first.h = which / p.row_blocks;
        mine_first.rb = which - mine_first.h * p.row_blocks;
        mine_first.units = all;
        mine_first.unit = all * min(warp, working) / working;
        units = all * min(warp + 1, working) / working - mine_first.unit;
    } else {
        working = min(share.workers - static_cast<int>(blockIdx.x) * WARPS, WARPS);
        if (working <= 0) return;        // the whole CTA
        mine_first = attend_segment(p, cum, share.begin(warp < working ? worker : worker - warp));
        units = warp < working ? static_cast<int>(share.begin(worker + 1) - share.begin(worker)) : 0;
    }
    if (lane == 0) open_piece[warp] = left_piece[warp] = make_int2(0, 0);
    const int psh = p.kv.page_shift, ps = 1 << psh;
    const int head_bytes = ps * (D + 8);
    const int unit_tokens = 1 << share.shift;

    // A stage mirrors the layout of the pages that its unit lies in: page j of the unit at j * head_bytes,
    // the parts of a page at their own offsets. Half a page is four copies, a whole one is one.
    AttendFeed feed;
    feed.seg = mine_first;
    feed.units_left = units;
    feed.slot = 0;
    feed.enter(p);
    auto issue = [&]() {                 // one unit into the next stage; its barrier completes when it has arrived
        if (feed.units_left == 0) return;
        const uint32_t bar = bar0 + 8 * feed.slot, dst = ring0 + feed.slot * STAGE;
        const int tok = feed.seg.unit << share.shift;
        if (tok < feed.len) {
            const int index = tok >> psh;
            feed.hold(p, index, lane);
            const unsigned char *src = p.kv.layer + feed.seg.h * head_bytes;
            if (unit_tokens < ps) {
                const int page = __shfl_sync(0xffffffffu, feed.held, index - feed.base);
                if (lane == 0) {
                    src += page * p.kv.page_bytes;
                    const int o = tok & (ps - 1), codes = unit_tokens * (D / 2), pairs = unit_tokens * 4;
                    mbar_arrive_expect_tx(bar, 2 * codes + 2 * pairs);
                    const int at[4] = {o * (D / 2), (ps + o) * (D / 2), ps * D + o * 4, ps * (D + 4) + o * 4};
#pragma unroll
                    for (int i = 0; i < 4; ++i) bulk_load(dst + at[i], src + at[i], i < 2 ? codes : pairs, bar);
                }
            } else {
                const int count = min((unit_tokens - 1) >> psh, (feed.len - 1 - tok) >> psh) + 1;   // pages with tokens of the unit
                if (lane == 0) mbar_arrive_expect_tx(bar, count * head_bytes);
                for (int i = 0; i < count; ++i) {
                    const int page = __shfl_sync(0xffffffffu, feed.held, index + i - feed.base);
                    if (lane == 0) bulk_load(dst + i * head_bytes, src + page * p.kv.page_bytes, head_bytes, bar);
                }
            }
        } else if (lane == 0) {
            mbar_arrive(bar);            // an entry without keys
        }
        feed.slot = feed.slot + 1 == STAGES ? 0 : feed.slot + 1;
        --feed.units_left;
        if (++feed.seg.unit == feed.seg.units && feed.units_left > 0) {
            const int b = feed.seg.b;
            attend_next(p, cum, feed.seg);
            if (feed.seg.b != b) feed.enter(p);
        }
    };
    const Exponents exponents;
    Segment seg = mine_first;
#pragma unroll 1
    for (int i = 0; i < STAGES; ++i) issue();

    int done = 0, slot = 0;
    uint32_t parity = 0;
    while (done < units) {
        const int mine = min(units - done, seg.units - seg.unit);
        const int row = kv_row(p.kv, seg.b);
        const int len = row < 0 ? 0 : kv_length(p.kv, row);
        const int n = p.q_len ? min(max(p.q_len[seg.b], 0), p.n) : p.n;
        const int rows = p.n * p.group;

        // ---- the query rows: column `g` of block nt is row rb * ROWS + 8 nt + g; a lane holds dimensions
        // (D / 4) t + 8 w + q and + 4 of it for w < W, q < 4
        uint32_t qf[QREG ? NT : 1][W][4];
        float qsum[NT][2];
        int last[NT][2];                 // the newest key that columns 2 t and 2 t + 1 see
        float f = 1.f;
        int all_see;                     // the newest key that all columns see alike; -1: some column is no query, or has a factor
        {
            // bring the rows to [2^10, 2^11) by a power of two: bf16 fits fp16, and 16 q does too. One power for the rows of
            // a pass, which then share the keys' scales, unless a row lies more than 2^10 below the largest or that one above
            // 2^51 (where the common factor would leave fp32's range): such a row gets its own, and its scores a factor.
            // Within the 2^10 a row is rounded at 2^-25 of its own largest value at worst.
            union Eight { uint4 raw; T x[8]; } u[NT][W];
            float row_top[NT], top = 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int qr = seg.rb * ROWS + nt * 8 + g;
                const bool real = qr < rows;
                const int i = real ? qr / p.group : 0, gq = real ? qr - i * p.group : 0;
                const T *src = static_cast<const T *>(p.q) + seg.b * p.q_b + i * p.q_n +
                               (static_cast<int64_t>(seg.h) * p.group + gq) * p.q_h + t * (D / 4);
                row_top[nt] = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    u[nt][w].raw = make_uint4(0, 0, 0, 0);
                    if (real) {
                        if (p.vec) u[nt][w].raw = *reinterpret_cast<const uint4 *>(src + 8 * w);
                        else
#pragma unroll
                            for (int j = 0; j < 8; ++j) u[nt][w].x[j] = src[8 * w + j];
                    }
                    row_top[nt] = fmaxf(row_top[nt], q_top(u[nt][w].x));
                }
                row_top[nt] = fmaxf(row_top[nt], __shfl_xor_sync(0xffffffffu, row_top[nt], 1));
                row_top[nt] = fmaxf(row_top[nt], __shfl_xor_sync(0xffffffffu, row_top[nt], 2));
                top = fmaxf(top, row_top[nt]);
            }
            top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));     // not negative: bits have its order
            auto power = [](float x) { return min(max(static_cast<int>(__float_as_uint(x) >> 23) - 127 - 10, -126), 117); };
            const int e = top > 0.f ? min(power(top), 40) : 0;
            auto row_power = [&](float x) {
                const int r = x > 0.f ? max(power(x), e - 120) : e;
                return r <= e && r >= e - 10 ? e : r;
            };
            f = __uint_as_float((127 + e) << 23);
            bool own = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) own |= row_power(row_top[nt]) != e;
            const bool spread = __any_sync(0xffffffffu, own);
            all_see = n < p.n || spread ? -1 : len - n;
            __syncwarp();                // the last segment's factors have been read
            float inv = __uint_as_float((127 - e) << 23);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float by = 1.f;
                if (spread) {
                    const int r = row_power(row_top[nt]);
                    inv = __uint_as_float((127 - r) << 23);
                    by = __uint_as_float((127 + r - e) << 23);
                }
                if (t == 0) row_factor[warp][nt * 8 + g] = by;
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    uint32_t packed[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const __half2 h = __floats2half2_rn(to_float(u[nt][w].x[j]) * inv, to_float(u[nt][w].x[j + 4]) * inv);
                        const float2 back = __half22float2(h);
                        sum += back.x + back.y;
                        const __half2 up = j % 2 == 0 ? __hmul2(h, __float2half2_rn(16.f)) : h;   // c 2^-24 against c 2^-20
                        packed[j] = *reinterpret_cast<const uint32_t *>(&up);
                    }
                    if (QREG)
#pragma unroll
                        for (int j = 0; j < 4; ++j) qf[QREG ? nt : 0][w][j] = packed[j];
                    else
                        q_smem[(nt * W + w) * 32 + lane] = make_uint4(packed[0], packed[1], packed[2], packed[3]);
                }
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                sum *= by;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    qsum[nt][c] = __shfl_sync(0xffffffffu, sum, (2 * t + c) * 4);
                    const int qi = (seg.rb * ROWS + nt * 8 + 2 * t + c) / p.group;
                    last[nt][c] = qi < n ? len - n + qi : -1;
                }
            }
        }
        __syncwarp();                    // the factors are in place
        f *= p.scale * 1048576.f;        // the codes' 2^-20

        // the weights are 2^(score - mb), mb a maximum of score + floor(log2 s_v) less kAttendBias: that maximum's p is a power of
        // two, and its p s_v exact in fp16
        float acc[NT][MT][4], mb[NT][2], l[NT][2], ob[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) mb[nt][e] = -1e30f, l[nt][e] = ob[nt][e] = 0.f;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[nt][i][j] = 0.f;
        }

        for (int u = 0; u < mine; ++u) {
            bool here = mbar_try_wait(bar0 + 8 * slot, parity);
            if (!here) here = mbar_wait_bounded(bar0 + 8 * slot, parity);
            if (!__all_sync(0xffffffffu, here)) {
                // a copy did not arrive: say so, give the others a chance to land, and leave
                if (lane == 0) atomicMax(p.kv.status, kStatusTimeout);
                for (int i = 1; i < STAGES && i < units - done; ++i) {
                    slot = slot + 1 == STAGES ? 0 : slot + 1;
                    parity ^= slot == 0;
                    mbar_wait_bounded(bar0 + 8 * slot, parity);
                }
                done = units;
                break;
            }
            ++done;
            const int tok0 = (seg.unit + u) << share.shift;
            const unsigned char *st = ring + slot * STAGE;
            // tiles of 16 tokens, side by side where all queries see all of them and share a power of two; MASKED: one
            // where that does not hold
            auto tile = [&](auto masked_type, int h) {
                constexpr bool masked = decltype(masked_type)::value;
                constexpr int KT = masked ? 1 : TILES;
                const int tok = tok0 + 16 * h;
                LaneCodes<D> xk[KT][2], xv[KT][2];
                float ks[KT][2], kb[KT][2], vs[KT][2], vb[KT][2], vl[KT][2];
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    const int at = tok + 16 * kt;
                    const unsigned char *page = st + ((at >> psh) - (tok0 >> psh)) * head_bytes;
                    const unsigned char *codes = page + (at & (ps - 1)) * (D / 2) + lane * (D / 8);
                    const unsigned char *pairs = page + ps * D + ((at & (ps - 1)) + g) * 4;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        load_codes<D>(xk[kt][j], codes + j * (4 * D));
                        load_codes<D>(xv[kt][j], codes + ps * (D / 2) + j * (4 * D));
                        const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(pairs + j * 32));
                        const uint32_t v_pair = *reinterpret_cast<const uint32_t *>(pairs + ps * 4 + j * 32);
                        const float2 b = __half22float2(*reinterpret_cast<const __half2 *>(&v_pair));
                        ks[kt][j] = a.x * f;
                        kb[kt][j] = (a.y - 8.f * a.x) * (f * 9.5367431640625e-7f);        // sum(q) carries no 2^-20
                        vs[kt][j] = b.x;
                        vb[kt][j] = b.y;
                        vl[kt][j] = exponents.log2_floor(v_pair);
                        if (masked && at + g + 8 * j >= len) vs[kt][j] = vb[kt][j] = 0.f;   // the rest of a page holds anything
                    }
                }
                // ---- scores of keys g, g + 8 against columns 2 t, 2 t + 1
                float sc[KT][NT][4];
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) sc[kt][nt][j] = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) {
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) {
                        uint32_t a[4], b[4];
                        unpack4(xk[kt][0].w[w], a);
                        unpack4(xk[kt][1].w[w], b);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            uint4 q4;
                            if (QREG) q4 = make_uint4(qf[QREG ? nt : 0][w][0], qf[QREG ? nt : 0][w][1], qf[QREG ? nt : 0][w][2], qf[QREG ? nt : 0][w][3]);
                            else q4 = q_smem[(nt * W + w) * 32 + lane];
                            mma_f16(sc[kt][nt], a[0], b[0], a[1], b[1], q4.x, q4.y);
                            mma_f16(sc[kt][nt], a[2], b[2], a[3], b[3], q4.z, q4.w);
                        }
                    }
                }
                if (masked) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const float2 by = *reinterpret_cast<const float2 *>(&row_factor[warp][nt * 8 + 2 * t]);
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt) {
                            sc[kt][nt][0] *= by.x, sc[kt][nt][2] *= by.x;
                            sc[kt][nt][1] *= by.y, sc[kt][nt][3] *= by.y;
                        }
                    }
                }
                float pr[KT][NT][4];
                float ahead = -INFINITY;
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float key = -INFINITY;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float v = fmaf(ks[kt][j], sc[kt][nt][2 * j + e], fmaf(kb[kt][j], qsum[nt][e], -mb[nt][e]));
                                if (masked && tok + 16 * kt + g + 8 * j > last[nt][e]) v = -INFINITY;
                                pr[kt][nt][2 * j + e] = v;
                                key = fmaxf(key, v);
                            }
                        ahead = fmaxf(ahead, key + vl[kt][j]);
                    }
                if (__any_sync(0xffffffffu, ahead > kAttendLazy + kAttendBias)) {
                    // a new maximum: bring the sums to the new reference
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float top = -INFINITY;
#pragma unroll
                            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    float v = fmaf(ks[kt][j], sc[kt][nt][2 * j + e], kb[kt][j] * qsum[nt][e]);
                                    if (masked && tok + 16 * kt + g + 8 * j > last[nt][e]) v = -INFINITY;
                                    pr[kt][nt][2 * j + e] = v;
                                    top = fmaxf(top, v + vl[kt][j]);
                                }
                            top -= kAttendBias;
#pragma unroll
                            for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                            const float now = fmaxf(mb[nt][e], top);
                            const float by = exp2_approx(mb[nt][e] - now);
                            mb[nt][e] = now;
                            l[nt][e] *= by;
                            ob[nt][e] *= by;
#pragma unroll
                            for (int i = 0; i < MT; ++i) {
                                acc[nt][i][e] *= by;
                                acc[nt][i][2 + e] *= by;
                            }
#pragma unroll
                            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                                for (int j = 0; j < 2; ++j) pr[kt][nt][2 * j + e] -= now;
                        }
                }
                uint32_t pf[KT][NT][2];
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const float p0 = exp2_approx(pr[kt][nt][2 * j]), p1 = exp2_approx(pr[kt][nt][2 * j + 1]);
                            l[nt][0] += p0;
                            l[nt][1] += p1;
                            ob[nt][0] = fmaf(p0, vb[kt][j], ob[nt][0]);
                            ob[nt][1] = fmaf(p1, vb[kt][j], ob[nt][1]);
                            const __half2 hp = __floats2half2_rn(p0 * vs[kt][j], p1 * vs[kt][j]);
                            pf[kt][nt][j] = transpose8x8(*reinterpret_cast<const uint32_t *>(&hp));
                        }
                    }
                // ---- output rows (dimensions) 16 i + g, 16 i + 8 + g
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int w = 0; w < W / 2; ++w) {                    // words of a token's D / 16 bytes
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            uint32_t a[4], b[4];
                            const uint32_t pick = half ? 0x7632 : 0x5410;
                            const uint32_t xa = __byte_perm(xv[kt][0].w[w], xv[kt][0].w[W / 2 + w], pick);
                            const uint32_t xb = __byte_perm(xv[kt][1].w[w], xv[kt][1].w[W / 2 + w], pick);
                            exponents.unpack4(xa, a);
                            exponents.unpack4(xb, b);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma_f16(acc[nt][4 * w + 2 * half], a[0], a[1], b[0], b[1], pf[kt][nt][0], pf[kt][nt][1]);
                                mma_f16(acc[nt][4 * w + 2 * half + 1], a[2], a[3], b[2], b[3], pf[kt][nt][0], pf[kt][nt][1]);
                            }
                        }
                    }
            };
            const int tiles = (min(unit_tokens, len - tok0) + 15) >> 4;
#pragma unroll 1
            for (int h = 0; h < tiles;) {
                if (h + TILES > tiles || tok0 + 16 * (h + TILES) - 1 > all_see) tile(std::true_type{}, h), ++h;
                else tile(std::false_type{}, h), h += TILES;
            }
            __syncwarp();                // the stage has been read: it may be overwritten
            issue();
            slot = slot + 1 == STAGES ? 0 : slot + 1;
            parity ^= slot == 0;
        }

        // ---- the piece is done: sums over the lanes that share a column
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], o);
                    ob[nt][e] += __shfl_xor_sync(0xffffffffu, ob[nt][e], o);
                }
        const bool whole = mine == seg.units;
        const int64_t piece = 2 * worker + (seg.unit == 0 ? 1 : 0);
        const bool near = share.own_cta;         // a piece that another warp of this CTA will merge: the stages' room is free now
        if (lane == 0 && !whole && !near) {
            const int segment = seg.b * (p.kv.heads * p.row_blocks) + seg.h * p.row_blocks + seg.rb;
            if (seg.unit == 0) open_piece[warp] = make_int2(1, segment);
            else left_piece[warp] = make_int2(seg.unit + mine == seg.units ? 2 : 1, segment);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int lr = nt * 8 + 2 * t + e, qr = seg.rb * ROWS + lr;
                if (qr >= rows) continue;
                if (whole) {
                    const float inv = l[nt][e] > 0.f ? 1.f / l[nt][e] : l[nt][e] == 0.f ? 0.f : NAN;
                    T *o = attend_row<T>(p, seg, qr);
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        o[16 * i + g] = from_float<T>((acc[nt][i][e] + ob[nt][e]) * inv);
                        o[16 * i + 8 + g] = from_float<T>((acc[nt][i][2 + e] + ob[nt][e]) * inv);
                    }
                } else {
                    float *o = near ? reinterpret_cast<float *>(ring) + lr * attend_row_floats(D) : p.part + (piece * ROWS + lr) * D;
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        o[16 * i + g] = acc[nt][i][e] + ob[nt][e];
                        o[16 * i + 8 + g] = acc[nt][i][2 + e] + ob[nt][e];
                    }
                    if (g == 0) {
                        float *ml = near ? o + D : p.part_ml + (piece * ROWS + lr) * 2;
                        ml[0] = mb[nt][e];
                        ml[1] = l[nt][e];
                    }
                }
            }
        seg.unit += mine;
        if (seg.unit == seg.units) attend_next(p, cum, seg);
        if (!QREG) __syncwarp();
    }
    if (share.own_cta) {
        if (working > 1) attend_join_near<T, D, NT>(p, working, attend_smem);
        return;
    }
    attend_join<T, D, NT>(p, share, cum, working, open_piece, left_piece, reinterpret_cast<float *>(attend_smem));
}

}  // namespace ralm
