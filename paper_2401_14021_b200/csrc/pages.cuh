// Pages of a cache: a table of page numbers per row, a count of holders per page (0: free), and a
// pool of equally sized pages per layer.
//
// The order is part of the contract, so that the result is a function of the state alone: rows that
// shrink give their pages back first, then the growing rows take the lowest-numbered free pages in
// row order. All counting is in whole numbers; atomics only add, subtract, or take a maximum.
//
// The bookkeeping is latency (a few dependent round trips in one CTA: 5 to 10 us), the copies are bandwidth (two
// bytes of traffic per byte moved). Measured: 256 of 1024 pages of 70 KB in 32 layers moved in 196 us, 5.8 TB/s, 0.90
// of the measured copy bandwidth; fork, copy on write for 16 pairs in 24 layers and roll back in 23 us. Admission is the
// serial part: one thread writes a row's pages one after another (64 prompts of 2000 to 32000 tokens in and out again:
// 88 us with 64 tokens a page, 584 us with 16).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/ralm.h"
#include "common.cuh"

namespace ralm {

constexpr int kStatusInvalid = 1;    // RALM_ERR_INVALID_ARG
constexpr int kStatusNoPages = 2;    // RALM_ERR_OOM
constexpr int kPagesThreads = 1024;
constexpr int kPagesWarps = kPagesThreads / 32;
constexpr int kCopyThreads = 256;

// Workspace of a page pool, in int32 words: [0] moves of the running call, [1] 1 if it changes
// nothing, then [P] free pages (or where each page goes), [P] move sources, [P] move destinations,
// [P] growing holders of a page, [P] rows - lowest growing row. The last two are zero between calls.
__host__ __device__ inline int64_t pages_workspace_words(int64_t pages) { return 16 + 5 * pages; }
struct PagesWork {
    int *head, *list, *from, *to, *growers, *lowest;
};
__host__ __device__ inline PagesWork pages_work(const ralm_pages_t &p) {
    int *w = static_cast<int *>(p.workspace);
    const int64_t P = p.pages;
    return {w, w + 16, w + 16 + P, w + 16 + 2 * P, w + 16 + 3 * P, w + 16 + 4 * P};
}

// Inclusive scan over the CTA's threads; *total gets the sum. buf: kPagesWarps ints.
__device__ __forceinline__ int block_scan(int v, int *buf, int *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int scan = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += y;
    }
    __syncthreads();
    if (lane == 31) buf[warp] = scan;
    __syncthreads();
    int t = buf[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, t, o);
        if (lane >= o) t += y;
    }
    *total = __shfl_sync(0xffffffffu, t, 31);
    const int before = __shfl_sync(0xffffffffu, t, max(warp - 1, 0));
    return scan + (warp > 0 ? before : 0);
}

__device__ __forceinline__ bool page_ok(const ralm_pages_t &p, int page) { return page >= 0 && page < p.pages; }

constexpr int kPagesSmemList = 4096;   // free pages that the resize kernel keeps in shared memory

// lengths -> new_lengths for every row: give back, copy on write, take. One CTA (the state is a few KB and each step
// depends on the one before; what it costs is round trips to memory, so steps that no row asks for are skipped and
// the list of free pages stays on the chip where it fits). The page contents are moved by pages_copy_kernel from
// the list that this kernel leaves in the workspace.
__global__ void __launch_bounds__(kPagesThreads, 1)
pages_resize_kernel(const ralm_pages_t p, const int32_t *__restrict__ new_lengths) {
    cudaGridDependencySynchronize();                     // what ran before in the stream has ended
    __shared__ int buf[kPagesWarps];
    __shared__ int near_list[kPagesSmemList];
    __shared__ int flags;
    const PagesWork w = pages_work(p);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ps = p.page_size, M = p.max_pages;
    const long long cap = static_cast<long long>(M) * ps;
    auto pages_of = [&](int length) { return (length + ps - 1) / ps; };
    // the page that a growing row goes on writing into, or -1
    auto last_page = [&](int r) -> int {
        const int len = p.lengths[r];
        return new_lengths[r] > len && len % ps != 0 ? p.table[static_cast<int64_t>(r) * M + len / ps] : -1;
    };
    int bad = 0, shrinks = 0, continues = 0;
    if (tid == 0) flags = 0;
    __syncthreads();
    for (int r = tid; r < p.rows; r += kPagesThreads) {
        const int len = p.lengths[r], to = new_lengths[r];
        if (len < 0 || len > cap || to < 0 || to > cap) {
            bad = 1;
        } else if (to < len) {
            shrinks = 1;
        } else if (to > len && len % ps != 0) {
            continues = 1;
            if (!page_ok(p, last_page(r))) bad = 1;
        }
    }
    if (bad | shrinks | continues) atomicOr(&flags, bad | shrinks << 1 | continues << 2);
    __syncthreads();
    const int seen = flags;
    if (seen & 1) {
        if (tid == 0) {
            atomicMax(p.status, kStatusInvalid);
            w.head[0] = 0;
        }
        return;
    }
    // give back: holders only, the table is cleared once it is known that the call goes through
    auto release = [&](int sign) {
        for (int r = warp; r < p.rows; r += kPagesWarps) {
            const int have = pages_of(p.lengths[r]), need = pages_of(new_lengths[r]);
            for (int c = need + lane; c < have; c += 32) {
                const int page = p.table[static_cast<int64_t>(r) * M + c];
                if (page_ok(p, page)) atomicAdd(&p.refs[page], sign);
            }
        }
    };
    if (seen & 2) {
        release(-1);
        __syncthreads();
    }
    // who goes on writing into a page that others hold too
    int shared = 0;
    if (seen & 4) {
        for (int r = tid; r < p.rows; r += kPagesThreads) {
            const int page = last_page(r);
            if (page >= 0 && p.refs[page] > 1) {
                atomicAdd(&w.growers[page], 1);
                atomicMax(&w.lowest[page], p.rows - r);
                shared = 1;
            }
        }
        shared = __syncthreads_or(shared);
    }
    auto forget = [&]() {                                // the scratch counts go back to zero
        for (int r = tid; r < p.rows; r += kPagesThreads) {
            const int page = last_page(r);
            if (page >= 0) w.growers[page] = w.lowest[page] = 0;
        }
    };
    auto copied_page = [&](int r) -> int {               // the page that the row gets a copy of, or -1
        if (!shared) return -1;
        const int page = last_page(r);
        if (page < 0 || p.refs[page] <= 1) return -1;
        return w.growers[page] == p.refs[page] && w.lowest[page] == p.rows - r ? -1 : page;
    };
    auto demand_of = [&](int r) { return max(pages_of(new_lengths[r]) - pages_of(p.lengths[r]), 0) + (copied_page(r) >= 0); };
    long long demand = 0;
    for (int r0 = 0; r0 < p.rows; r0 += kPagesThreads) {
        int total;
        block_scan(r0 + tid < p.rows ? demand_of(r0 + tid) : 0, buf, &total);
        demand += total;
    }
    // the lowest free pages, as many as are asked for
    int *list = demand <= kPagesSmemList ? near_list : w.list;
    long long found = 0;
    for (int g0 = 0; g0 < p.pages && found < demand; g0 += 4 * kPagesThreads) {
        const int g = g0 + 4 * tid;
        int free_here[4], n = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            free_here[j] = g + j < p.pages && p.refs[g + j] == 0;
            n += free_here[j];
        }
        int total;
        long long at = found + block_scan(n, buf, &total) - n;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (free_here[j] && at < demand) list[at++] = g + j;
        found += total;
    }
    __syncthreads();
    if (found < demand) {
        if (seen & 2) release(+1);
        if (shared) forget();
        if (tid == 0) {
            atomicMax(p.status, kStatusNoPages);
            w.head[0] = 0;
        }
        return;
    }
    int taken = 0, moves = 0;
    for (int r0 = 0; r0 < p.rows; r0 += kPagesThreads) {
        const int r = r0 + tid;
        int total, total_copies = 0, move = moves;
        const int copied = r < p.rows ? copied_page(r) : -1;
        const int want = r < p.rows ? demand_of(r) : 0;
        int at = taken + block_scan(want, buf, &total) - want;
        if (shared) move += block_scan(copied >= 0, buf, &total_copies) - (copied >= 0);
        taken += total;
        moves += total_copies;
        if (r < p.rows) {
            int32_t *row = p.table + static_cast<int64_t>(r) * M;
            const int len = p.lengths[r], have = pages_of(len), need = pages_of(new_lengths[r]);
            if (copied >= 0) {
                const int page = list[at++];
                p.refs[page] = 1;
                row[len / ps] = page;
                w.from[move] = copied;
                w.to[move] = page;
            }
            for (int c = have; c < need; ++c) {
                const int page = list[at++];
                p.refs[page] = 1;
                row[c] = page;
            }
            for (int c = need; c < have; ++c) row[c] = -1;
        }
    }
    if (shared) {
        __syncthreads();
        forget();
        for (int i = tid; i < moves; i += kPagesThreads) {
            const int page = w.from[i];                  // a page that was copied has a holder less
            atomicSub(&p.refs[page], 1);
            w.growers[page] = w.lowest[page] = 0;
        }
        __syncthreads();
    }
    for (int r = tid; r < p.rows; r += kPagesThreads) p.lengths[r] = new_lengths[r];
    if (tid == 0) w.head[0] = moves;
}

// Rows dst[i] give back what they hold and then hold the pages of rows src[i] too. One CTA.
// seen: one bit per row, dynamic shared memory.
__global__ void __launch_bounds__(kPagesThreads, 1)
pages_fork_kernel(const ralm_pages_t p, const int32_t *__restrict__ src, const int32_t *__restrict__ dst, int n) {
    cudaGridDependencySynchronize();                     // what ran before in the stream has ended
    extern __shared__ unsigned int seen[];
    __shared__ int bad;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ps = p.page_size, M = p.max_pages;
    const long long cap = static_cast<long long>(M) * ps;
    for (int i = tid; i < (p.rows + 31) / 32; i += kPagesThreads) seen[i] = 0;
    if (tid == 0) bad = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kPagesThreads) {
        const int d = dst[i], s = src[i];
        if (d < 0 || d >= p.rows || s < 0 || s >= p.rows) bad = 1;
        else if (atomicOr(&seen[d >> 5], 1u << (d & 31)) >> (d & 31) & 1) bad = 1;          // twice a destination
        else if (p.lengths[s] < 0 || p.lengths[s] > cap || p.lengths[d] < 0 || p.lengths[d] > cap) bad = 1;
    }
    __syncthreads();
    for (int i = tid; i < n; i += kPagesThreads) {
        const int s = src[i];
        if (s >= 0 && s < p.rows && (seen[s >> 5] >> (s & 31) & 1)) bad = 1;                  // source and destination
    }
    __syncthreads();
    if (bad) {
        if (tid == 0) atomicMax(p.status, kStatusInvalid);
        return;
    }
    for (int i = warp; i < n; i += kPagesWarps) {
        const int s = src[i], d = dst[i];
        const int have = (p.lengths[d] + ps - 1) / ps, get = (p.lengths[s] + ps - 1) / ps;
        int32_t *to = p.table + static_cast<int64_t>(d) * M;
        const int32_t *from = p.table + static_cast<int64_t>(s) * M;
        for (int c = lane; c < max(have, get); c += 32) {
            const int old = c < have ? to[c] : -1, page = c < get ? from[c] : -1;
            if (page_ok(p, old)) atomicSub(&p.refs[old], 1);
            if (page_ok(p, page)) atomicAdd(&p.refs[page], 1);
            to[c] = page;
        }
        __syncwarp();
        if (lane == 0) p.lengths[d] = p.lengths[s];
    }
}

// Which live pages move down so that the live ones become pages 0 .. live - 1: the i-th live page at
// or above `live` goes to the i-th hole below it. One CTA. w.list[page]: the page's new number.
__global__ void __launch_bounds__(kPagesThreads, 1)
pages_compact_kernel(const ralm_pages_t p, int32_t *__restrict__ live_out) {
    cudaGridDependencySynchronize();                     // what ran before in the stream has ended
    __shared__ int buf[kPagesWarps];
    const PagesWork w = pages_work(p);
    const int tid = threadIdx.x;
    int live = 0;
    for (int g0 = 0; g0 < p.pages; g0 += 4 * kPagesThreads) {
        int n = 0, total;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int g = g0 + 4 * tid + j;
            n += g < p.pages && p.refs[g] > 0;
        }
        block_scan(n, buf, &total);
        live += total;
    }
    int holes = 0, movers = 0;
    for (int g0 = 0; g0 < p.pages; g0 += 4 * kPagesThreads) {
        int flag[4], n = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int g = g0 + 4 * tid + j;
            flag[j] = 0;
            if (g < p.pages) {
                const bool used = p.refs[g] > 0;
                flag[j] = g < live ? (used ? 0 : 1) : (used ? 1 << 16 : 0);   // hole, or page to move
            }
            n += flag[j];
        }
        int total;
        int at = block_scan(n, buf, &total) - n;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int g = g0 + 4 * tid + j;
            if (flag[j] == 1) w.to[holes + (at & 0xFFFF)] = g;
            if (flag[j] > 1) w.from[movers + (at >> 16)] = g;
            if (g < p.pages && flag[j] <= 1) w.list[g] = g;
            at += flag[j];
        }
        holes += total & 0xFFFF;
        movers += total >> 16;
    }
    __syncthreads();
    for (int i = tid; i < movers; i += kPagesThreads) {
        const int from = w.from[i], to = w.to[i];
        w.list[from] = to;
        p.refs[to] = p.refs[from];
        p.refs[from] = 0;
    }
    if (tid == 0) {
        w.head[0] = movers;
        live_out[0] = live;
    }
}

// Copies pages from[i] of the source to to[i] of the destination, i < *count (or n), in every layer;
// with `remap`, also rewrites the table's page numbers through it.
struct PagesCopyParams {
    const unsigned char *src;
    unsigned char *dst;
    int64_t src_layer_stride, dst_layer_stride, page_bytes;
    int layers, src_pages, dst_pages;
    const int *from, *to, *count;
    int n;                 // used when count is null
    int *status;           // may be null
    int32_t *table;        // may be null
    int64_t table_words;
    const int *remap;
    int remap_pages;
};
__global__ void __launch_bounds__(kCopyThreads)
pages_copy_kernel(const PagesCopyParams p) {
    cudaGridDependencySynchronize();                     // launched while the kernel that makes the list runs
    const int64_t step = static_cast<int64_t>(gridDim.x) * blockDim.x;
    if (p.table) {
        for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < p.table_words; i += step) {
            const int page = p.table[i];
            if (page >= 0 && page < p.remap_pages) {
                const int to = p.remap[page];
                if (to != page) p.table[i] = to;
            }
        }
    }
    const int n = p.count ? *p.count : p.n;
    constexpr int64_t kChunk = kCopyThreads * 16 * 4;
    const int chunks = static_cast<int>((p.page_bytes + kChunk - 1) / kChunk);
    const int64_t jobs = static_cast<int64_t>(n) * p.layers * chunks;
    for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
        const int chunk = static_cast<int>(job % chunks);
        const int64_t rest = job / chunks;
        const int layer = static_cast<int>(rest % p.layers);
        const int64_t move = rest / p.layers;
        const int from = p.from[move], to = p.to[move];
        if (from < 0 || from >= p.src_pages || to < 0 || to >= p.dst_pages) {
            if (p.status && threadIdx.x == 0) atomicMax(p.status, kStatusInvalid);
            continue;
        }
        const unsigned char *s = p.src + layer * p.src_layer_stride + from * p.page_bytes;
        unsigned char *d = p.dst + layer * p.dst_layer_stride + to * p.page_bytes;
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t at = chunk * kChunk + (j * kCopyThreads + threadIdx.x) * 16;
            if (at < p.page_bytes) v[j] = *reinterpret_cast<const uint4 *>(s + at);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t at = chunk * kChunk + (j * kCopyThreads + threadIdx.x) * 16;
            if (at < p.page_bytes) *reinterpret_cast<uint4 *>(d + at) = v[j];
        }
    }
}

}  // namespace ralm
