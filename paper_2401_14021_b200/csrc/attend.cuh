// Attention of a request's newest tokens over its 4-bit cache:
//     out = softmax(scale q.k) v over the keys that the query may see.
//
// With k = s_k (c - 8) + b_k the score is s_k (q.(c - 8)) + b_k sum(q), and the output is
// sum (p s_v)(c - 8) + sum p b_v: the matrix instructions see whole numbers between -8 and 7, exact in
// fp16, and the scales enter in 32 bits. The weights p s_v are rounded to fp16 (11 bits) before the
// second product; maxima, sums and outputs stay in 32 bits.
//
// Orientation: keys are the rows of the instructions (m16n8k16) and query rows the columns, so that a
// decode step with up to 8 query rows per key-value head fills one column block, and the codes go from
// 16-byte loads to operand registers without passing through shared memory.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "common.cuh"
#include "kv4.cuh"
#include "mix.cuh"

namespace ralm {

constexpr int kAttendThreads = 256;
constexpr int kAttendWarps = kAttendThreads / 32;
constexpr int kAttendMaxBatch = 4096;
constexpr int kAttendMinTiles = 4;       // a worker is given at least this many tiles of 16 tokens
constexpr float kAttendLazy = 6.f;       // a maximum may be this far (powers of two) behind before sums are rescaled
constexpr float kAttendBias = 8.f;       // exponent added to the weights: 2^(6 + 8 + 1) is below fp16's largest

struct AttendParams {
    KvParams kv;
    const void *q;
    void *out;
    int64_t q_b, q_n, q_h, o_b, o_n, o_h;
    const int32_t *q_len;     // or null: n queries for every entry
    int n, group;             // queries per entry; query heads per key-value head
    int row_blocks;           // blocks of 8 * NT query rows
    float scale;              // softmax scale * log2(e)
    float *part;              // [2 * workers][8 * NT][D] partial outputs
    float *part_ml;           // [2 * workers][8 * NT][2] their maxima and sums
    int workers;
    int vec;                  // q is 16-byte aligned in every row
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t hsub2(uint32_t a, uint32_t b) {
    const __half2 r = __hsub2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
// The four pairs (nibble i of the low half, nibble i of the high half) of a word as fp16 pairs minus 8:
// a nibble under the exponent of 1024 (in the last four mantissa bits) or of 64 (in the four above)
// reads 1024 + c or 64 + c, and the subtraction is exact.
__device__ __forceinline__ void unpack4(uint32_t x, uint32_t (&y)[4]) {
    const uint32_t z = x >> 8;
    y[0] = hsub2((x & 0x000F000Fu) | 0x64006400u, 0x64086408u);   // - 1032
    y[1] = hsub2((x & 0x00F000F0u) | 0x54005400u, 0x54805480u);   // - 72
    y[2] = hsub2((z & 0x000F000Fu) | 0x64006400u, 0x64086408u);
    y[3] = hsub2((z & 0x00F000F0u) | 0x54005400u, 0x54805480u);
}

template <int D> struct LaneCodes;                                    // a lane's D / 8 bytes of a tile
template <> struct LaneCodes<128> { union { uint4 raw; uint32_t w[4]; }; };
template <> struct LaneCodes<64> { union { uint2 raw; uint32_t w[2]; }; };
template <int D> __device__ __forceinline__ void load_codes(LaneCodes<D> &c, const unsigned char *at) {
    c.raw = *reinterpret_cast<const decltype(c.raw) *>(at);
}

// What one tile of 16 tokens brings to a lane: codes of keys g and g + 8, V codes of its two halves, and
// the (scale, offset) pairs of keys g and g + 8.
template <int D> struct Tile {
    LaneCodes<D> k[2], v[2];
    __half2 kp[2], vp[2];
};

// How the work is cut: segments (entry, head, row block) follow one another, each `tiles` long (at least
// one, so that an entry without keys is written too), and worker w takes units [total w / W, total (w + 1) / W).
struct Share {
    long long total;
    int workers;
    __device__ __forceinline__ long long begin(int w) const { return total * w / workers; }
    __device__ __forceinline__ int owner(long long u) const { return static_cast<int>(((u + 1) * workers - 1) / total); }
};
// Prefix sums of the entries' tiles (without heads and row blocks) in shared memory: cum[b] for b <= batch.
__device__ inline Share attend_share(const AttendParams &p, int *cum, int *scratch) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int carry = 0;
    for (int b0 = 0; b0 < p.kv.batch; b0 += blockDim.x) {
        const int b = b0 + tid;
        int tiles = 0;
        if (b < p.kv.batch) {
            const int row = kv_row(p.kv, b);
            tiles = row < 0 ? 1 : max((kv_length(p.kv, row) + 15) >> 4, 1);
        }
        int scan = tiles;
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
    Share s;
    s.total = static_cast<long long>(carry) * p.kv.heads * p.row_blocks;
    s.workers = static_cast<int>(min(static_cast<long long>(p.workers), max(s.total / kAttendMinTiles, 1LL)));
    return s;
}
struct Segment { int b, h, rb, tile, tiles; };                     // tile: the unit's place inside the segment
__device__ __forceinline__ Segment attend_segment(const AttendParams &p, const int *cum, long long unit) {
    const int per = p.kv.heads * p.row_blocks;
    int lo = 0, hi = p.kv.batch - 1;
    while (lo < hi) {                                               // the last entry that begins at or before the unit
        const int mid = (lo + hi + 1) >> 1;
        if (static_cast<long long>(cum[mid]) * per <= unit) lo = mid; else hi = mid - 1;
    }
    Segment s;
    s.b = lo;
    s.tiles = cum[lo + 1] - cum[lo];
    const long long in = unit - static_cast<long long>(cum[lo]) * per;
    const int which = static_cast<int>(in / s.tiles);
    s.tile = static_cast<int>(in % s.tiles);
    s.h = which / p.row_blocks;
    s.rb = which % p.row_blocks;
    return s;
}

// One query row's place: query i and head of the group, from its number in the segment's entry.
template <typename T>
__device__ __forceinline__ void attend_store(const AttendParams &p, const Segment &s, int row, int d, float x) {
    const int i = row / p.group, gq = row % p.group;
    T *o = static_cast<T *>(p.out) + s.b * p.o_b + i * p.o_n + (static_cast<int64_t>(s.h) * p.group + gq) * p.o_h;
    o[d] = from_float<T>(x);
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kAttendThreads, NT <= 2 ? 2 : 1)
attend_kernel(const AttendParams p) {
    constexpr int W = D / 32;            // words of K codes per lane and key; also E, dimensions / 32
    constexpr int MT = D / 16;           // row blocks of the output
    constexpr int ROWS = 8 * NT;
    extern __shared__ int attend_smem[];
    int *cum = attend_smem;
    __shared__ int scratch[32];
    const Share share = attend_share(p, cum, scratch);
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int worker = blockIdx.x * kAttendWarps + (threadIdx.x >> 5);
    if (worker >= share.workers) return;
    const int ps = p.kv.page_size;
    const int head_bytes = ps * (D + 8);
    long long unit = share.begin(worker);
    const long long stop = share.begin(worker + 1);

    while (unit < stop) {
        const Segment seg = attend_segment(p, cum, unit);
        const int tiles = static_cast<int>(min(stop - unit, static_cast<long long>(seg.tiles - seg.tile)));
        const int row = kv_row(p.kv, seg.b);
        const int len = row < 0 ? 0 : kv_length(p.kv, row);
        const int n = p.q_len ? min(max(p.q_len[seg.b], 0), p.n) : p.n;
        const int rows = p.n * p.group;

        // ---- the query rows: column `g` of block nt is row rb * ROWS + 8 nt + g; a lane holds dimensions
        // (D / 4) t + 8 w + q and + 4 of it for w < W, q < 4
        uint32_t qf[NT][W][4];
        float qsum[NT][2];
        int last[NT][2];                 // the newest key that columns 2 t and 2 t + 1 see
        float f = 1.f;
        {
            float top = 0.f;
#pragma unroll
            for (int pass = 0; pass < (sizeof(T) == 2 && !std::is_same<T, __half>::value ? 2 : 1); ++pass) {
                float inv = 1.f;
                if (pass == 1) {         // bf16: bring the rows into fp16's range by one power of two
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    const int e = top > 0.f ? min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127 - 8, -100), 100) : 0;
                    f = __uint_as_float((127 + e) << 23);
                    inv = __uint_as_float((127 - e) << 23);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int qr = seg.rb * ROWS + nt * 8 + g;
                    const bool real = qr < rows;
                    const int i = real ? qr / p.group : 0, gq = real ? qr % p.group : 0;
                    const T *src = static_cast<const T *>(p.q) + seg.b * p.q_b + i * p.q_n +
                                   (static_cast<int64_t>(seg.h) * p.group + gq) * p.q_h + t * (D / 4);
                    float sum = 0.f;
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        union { uint4 raw; T x[8]; } u;
                        u.raw = make_uint4(0, 0, 0, 0);
                        if (real) {
                            if (p.vec) u.raw = *reinterpret_cast<const uint4 *>(src + 8 * w);
                            else
#pragma unroll
                                for (int j = 0; j < 8; ++j) u.x[j] = src[8 * w + j];
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float x0 = to_float(u.x[j]) * inv, x1 = to_float(u.x[j + 4]) * inv;
                            if (fabsf(x0) < INFINITY) top = fmaxf(top, fabsf(x0));
                            if (fabsf(x1) < INFINITY) top = fmaxf(top, fabsf(x1));
                            const __half2 h = __floats2half2_rn(x0, x1);
                            qf[nt][w][j] = *reinterpret_cast<const uint32_t *>(&h);
                            const float2 back = __half22float2(h);
                            sum += back.x + back.y;
                        }
                    }
                    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        qsum[nt][e] = __shfl_sync(0xffffffffu, sum, (2 * t + e) * 4);
                        const int qi = (seg.rb * ROWS + nt * 8 + 2 * t + e) / p.group;
                        last[nt][e] = qi < n ? len - n + qi : -1;
                    }
                }
            }
        }
        f *= p.scale;

        float acc[NT][MT][4], m[NT][2], l[NT][2], ob[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) m[nt][e] = -1e30f, l[nt][e] = ob[nt][e] = 0.f;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[nt][i][j] = 0.f;
        }

        const int32_t *pages = p.kv.table + static_cast<int64_t>(max(row, 0)) * p.kv.max_pages;
        auto fetch = [&](Tile<D> &x, int tile) {
            const int tok = tile * 16;
            int page = pages[tok / ps];
            if (page < 0 || page >= p.kv.pages) {
                atomicMax(p.kv.status, kStatusInvalid);
                page = 0;
            }
            const int slot = tok % ps;
            const unsigned char *base = p.kv.layer + page * p.kv.page_bytes + static_cast<int64_t>(seg.h) * head_bytes;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                load_codes<D>(x.k[j], base + (slot + 8 * j) * (D / 2) + lane * (D / 8));
                load_codes<D>(x.v[j], base + ps * (D / 2) + slot * (D / 2) + j * (4 * D) + lane * (D / 8));
                x.kp[j] = *reinterpret_cast<const __half2 *>(base + ps * D + (slot + g + 8 * j) * 4);
                x.vp[j] = *reinterpret_cast<const __half2 *>(base + ps * (D + 4) + (slot + g + 8 * j) * 4);
            }
        };
        const int first_tile = seg.tile, end_tile = len > 0 ? seg.tile + tiles : seg.tile;
        Tile<D> next;
        if (first_tile < end_tile) fetch(next, first_tile);
        for (int tile = first_tile; tile < end_tile; ++tile) {
            Tile<D> x = next;
            if (tile + 1 < end_tile) fetch(next, tile + 1);
            // ---- scores of keys g, g + 8 against columns 2 t, 2 t + 1
            float sc[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) sc[nt][j] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                uint32_t a[4], b[4];
                unpack4(x.k[0].w[w], a);
                unpack4(x.k[1].w[w], b);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma_f16(sc[nt], a[0], b[0], a[1], b[1], qf[nt][w][0], qf[nt][w][1]);
                    mma_f16(sc[nt], a[2], b[2], a[3], b[3], qf[nt][w][2], qf[nt][w][3]);
                }
            }
            const int key0 = tile * 16 + g;
            float ks[2], kb[2], vs[2], vb[2], ve[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 a = __half22float2(x.kp[j]), b = __half22float2(x.vp[j]);
                ks[j] = a.x * f;
                kb[j] = a.y * f;
                const bool inside = key0 + 8 * j < len;             // the rest of a page holds anything
                vs[j] = inside ? b.x : 0.f;
                vb[j] = inside ? b.y : 0.f;
                ve[j] = static_cast<float>(static_cast<int>(__float_as_uint(fmaxf(vs[j], 5.9604645e-8f)) >> 23) - 127);
            }
            const bool masked = tile * 16 + 15 > len - n || n < p.n;
            float ahead = -INFINITY;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float v = fmaf(ks[j], sc[nt][2 * j + e], kb[j] * qsum[nt][e]);
                        if (masked && key0 + 8 * j > last[nt][e]) v = -INFINITY;
                        sc[nt][2 * j + e] = v;
                        ahead = fmaxf(ahead, v + ve[j] - m[nt][e]);
                    }
            // weights are taken relative to m >= max(score + exponent of s_v) - kAttendLazy
            if (__any_sync(0xffffffffu, ahead > kAttendLazy)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = fmaxf(sc[nt][e] + ve[0], sc[nt][2 + e] + ve[1]);
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                        const float now = fmaxf(m[nt][e], top);
                        const float by = exp2_approx(m[nt][e] - now);
                        m[nt][e] = now;
                        l[nt][e] *= by;
                        ob[nt][e] *= by;
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            acc[nt][i][e] *= by;
                            acc[nt][i][2 + e] *= by;
                        }
                    }
            }
            uint32_t pf[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float p0 = exp2_approx(sc[nt][2 * j] - (m[nt][0] - kAttendBias));
                    const float p1 = exp2_approx(sc[nt][2 * j + 1] - (m[nt][1] - kAttendBias));
                    l[nt][0] += p0;
                    l[nt][1] += p1;
                    ob[nt][0] = fmaf(p0, vb[j], ob[nt][0]);
                    ob[nt][1] = fmaf(p1, vb[j], ob[nt][1]);
                    const __half2 h = __floats2half2_rn(p0 * vs[j], p1 * vs[j]);
                    pf[nt][j] = transpose8x8(*reinterpret_cast<const uint32_t *>(&h));
                }
            // ---- output rows (dimensions) 16 i + g, 16 i + 8 + g
#pragma unroll
            for (int w = 0; w < W / 2; ++w) {                        // words of a token's D / 16 bytes
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t a[4], b[4];
                    const uint32_t pick = half ? 0x7632 : 0x5410;
                    unpack4(__byte_perm(x.v[0].w[w], x.v[0].w[W / 2 + w], pick), a);
                    unpack4(__byte_perm(x.v[1].w[w], x.v[1].w[W / 2 + w], pick), b);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma_f16(acc[nt][4 * w + 2 * half], a[0], a[1], b[0], b[1], pf[nt][0], pf[nt][1]);
                        mma_f16(acc[nt][4 * w + 2 * half + 1], a[2], a[3], b[2], b[3], pf[nt][0], pf[nt][1]);
                    }
                }
            }
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
        const bool whole = seg.tile == 0 && tiles == seg.tiles;
        const int slot = 2 * worker + (seg.tile == 0 ? 1 : 0);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int lr = nt * 8 + 2 * t + e, qr = seg.rb * ROWS + lr;
                if (qr >= rows) continue;
                if (whole) {
                    const float inv = l[nt][e] > 0.f ? 1.f / l[nt][e] : l[nt][e] == 0.f ? 0.f : NAN;
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        attend_store<T>(p, seg, qr, 16 * i + g, (acc[nt][i][e] + ob[nt][e]) * inv);
                        attend_store<T>(p, seg, qr, 16 * i + 8 + g, (acc[nt][i][2 + e] + ob[nt][e]) * inv);
                    }
                } else {
                    float *o = p.part + (static_cast<int64_t>(slot) * ROWS + lr) * D;
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        o[16 * i + g] = acc[nt][i][e] + ob[nt][e];
                        o[16 * i + 8 + g] = acc[nt][i][2 + e] + ob[nt][e];
                    }
                    if (g == 0) {
                        p.part_ml[(static_cast<int64_t>(slot) * ROWS + lr) * 2] = m[nt][e];
                        p.part_ml[(static_cast<int64_t>(slot) * ROWS + lr) * 2 + 1] = l[nt][e];
                    }
                }
            }
        unit += tiles;
    }
}

// Joins the pieces of segments that several workers shared: one CTA of D threads per segment and query row.
template <typename T, int D, int ROWS>
__global__ void __launch_bounds__(D)
attend_join_kernel(const AttendParams p) {
    extern __shared__ int attend_smem[];
    __shared__ int scratch[32];
    const Share share = attend_share(p, attend_smem, scratch);
    const int rows = p.n * p.group;
    const int lr = blockIdx.y;
    // segment number -> its first unit
    const int per = p.kv.heads * p.row_blocks;
    const int b = blockIdx.x / per, which = blockIdx.x % per;
    Segment s;
    s.b = b;
    s.h = which / p.row_blocks;
    s.rb = which % p.row_blocks;
    s.tiles = attend_smem[b + 1] - attend_smem[b];
    const long long first = static_cast<long long>(attend_smem[b]) * per + static_cast<long long>(which) * s.tiles;
    const int w0 = share.owner(first), w1 = share.owner(first + s.tiles - 1);
    const int qr = s.rb * ROWS + lr;
    if (w0 == w1 || qr >= rows) return;
    auto slot_of = [&](int w) { return static_cast<int64_t>(2 * w + (w == w0 ? 1 : 0)) * ROWS + lr; };
    float M = -1e30f;
    for (int w = w0; w <= w1; ++w) M = fmaxf(M, p.part_ml[slot_of(w) * 2]);
    float L = 0.f, o = 0.f;
    for (int w = w0; w <= w1; ++w) {
        const float by = exp2_approx(p.part_ml[slot_of(w) * 2] - M);
        L = fmaf(p.part_ml[slot_of(w) * 2 + 1], by, L);
        o = fmaf(p.part[slot_of(w) * D + threadIdx.x], by, o);
    }
    attend_store<T>(p, s, qr, threadIdx.x, L > 0.f ? o / L : L == 0.f ? 0.f : NAN);
}

}  // namespace ralm
