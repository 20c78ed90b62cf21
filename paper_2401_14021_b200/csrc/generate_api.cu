// Host side of the generator's operators declared in include/ralm.h: the KNN-LM mixture, verification
// of drafted tokens, the pages of a cache, and the 4-bit cache with its attention. Argument checks and
// launches only; nothing here allocates.
#include "../../include/ralm.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <initializer_list>
#include <utility>

#include "attend.cuh"
#include "kv4.cuh"
#include "mix.cuh"
#include "pages.cuh"
#include "verify_tokens.cuh"

using namespace ralm;

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Where the elements of a strided argument lie: runs of contiguous bytes, n[i] of them step[i] bytes apart, the longest
// step first.
struct Runs {
    int64_t at, bytes, n[3], step[3], extent[4];   // extent[i]: from the first byte to the end of dimensions i and on
    Runs(const void *p, int64_t bytes_, std::initializer_list<std::pair<int64_t, int64_t>> dims)
        : at(static_cast<int64_t>(reinterpret_cast<uintptr_t>(p))), bytes(p ? bytes_ : 0) {
        int d = 0;
        for (auto [count, stride] : dims) {
            if (count <= 0) bytes = 0;
            if (stride < 0) at += (count - 1) * stride;
            const int64_t s = stride < 0 ? -stride : stride, c = s == 0 ? 1 : count;
            int i = d++;
            for (; i > 0 && step[i - 1] < s; --i) n[i] = n[i - 1], step[i] = step[i - 1];
            n[i] = c;
            step[i] = s;
        }
        for (; d < 3; ++d) n[d] = 1, step[d] = 0;
        extent[3] = bytes;
        for (int i = 2; i >= 0; --i) extent[i] = extent[i + 1] + (n[i] - 1) * step[i];
    }
    static bool meet(const Runs &a, int i, int64_t pa, const Runs &b, int j, int64_t pb) {
        const int64_t ea = a.extent[i], eb = b.extent[j];
        if (pa + ea <= pb || pb + eb <= pa) return false;
        while (i < 3 && a.n[i] == 1) ++i;
        while (j < 3 && b.n[j] == 1) ++j;
        if (i == 3 && j == 3) return true;
        if (i < 3 && j < 3 && a.step[i] == b.step[j]) {              // side by side in every part of one buffer
            const int64_t s = a.step[i], behind = ((pb - pa) % s + s) % s;
            if (a.extent[i + 1] <= behind && behind + b.extent[j + 1] <= s) return false;
        }
        if (i == 3 || (j < 3 && eb > ea)) return meet(b, j, pb, a, i, pa);
        // those parts of a that reach into b's range
        const int64_t s = a.step[i], part = a.extent[i + 1];
        const int64_t first = pb - part - pa < 0 ? 0 : (pb - part - pa) / s + 1, last = std::min(a.n[i] - 1, (pb + eb - 1 - pa) / s);
        for (int64_t k = first; k <= last; ++k)
            if (meet(a, i + 1, pa + k * s, b, j, pb)) return true;
        return false;
    }
    // Whether the two share a byte. Arguments in different places, the usual ones, are told apart at once.
    bool overlaps(const Runs &o) const { return bytes > 0 && o.bytes > 0 && meet(*this, 0, at, o, 0, o.at); }
};
Runs dense(const void *p, int64_t bytes) { return Runs(p, bytes, {}); }

// SMs of the current device (0: none), asked once per device.
int sm_count() {
    static std::atomic<int> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
    int n = dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
        if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

// Lets a kernel use up to `most` bytes of dynamic shared memory; asked once per kernel and device.
template <auto Kernel>
bool allow_smem(int most) {
    static std::atomic<bool> done[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return false;
    if (dev < 64 && done[dev].load(std::memory_order_relaxed)) return true;
    if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    if (dev < 64) done[dev].store(true, std::memory_order_relaxed);
    return true;
}

// One cluster of `cluster` CTAs per row.
template <typename Params>
ralm_status_t launch_cluster(void (*kernel)(Params), int rows, int cluster, int threads, size_t smem, cudaStream_t st,
                             const Params &params) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows) * cluster);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, params) != cudaSuccess) {
        cudaGetLastError();
        return RALM_ERR_CUDA;
    }
    return RALM_OK;
}

// The kernel may be set up while the last blocks of the one before it in the stream run out; it waits for that
// one's end (with all that it wrote) before it reads anything.
template <typename... P, typename... A>
ralm_status_t launch(void (*kernel)(P...), int64_t blocks, int threads, size_t smem, cudaStream_t st, const A &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, P(args)...) != cudaSuccess) {
        cudaGetLastError();
        return RALM_ERR_CUDA;
    }
    return RALM_OK;
}

// A row is cut over a cluster so that a slice is about 32 KB (six CTAs then fit an SM, and one CTA's
// stores overlap another's loads), and further while there are fewer CTAs than the GPU can hold; but not
// below one vector per thread.
// The neighbours' table has twice as many slots as neighbours, up to 16 KB: half full at most it is quicker where
// one CTA per SM waits for it (1 row x 32000, 64 neighbours: 6.2 us a call, 6.7 with as many slots as
// neighbours), but 32 KB would leave room for fewer CTAs (72 rows x 50257, 1024 neighbours: 18.5 us, 16.5 with 16 KB).
constexpr int kMixSlice = 32 * 1024;
constexpr int kMixMaxStage = 160 * 1024;   // bytes of a slice that a CTA keeps in shared memory

template <typename T>
ralm_status_t launch_mix(MixParams p, int R, int sms, cudaStream_t st) {
    constexpr int64_t kVec = MixVec<T>::n;
    int cluster = 1;
    auto slice_of = [&](int c) { return ((p.V + kVec - 1 + c - 1) / c + kVec - 1) / kVec * kVec; };
    while (cluster < kMixMaxCluster &&
           (slice_of(cluster) * sizeof(T) > kMixSlice || (static_cast<int64_t>(R) * cluster < 4LL * sms && slice_of(2 * cluster) >= kVec * kMixThreads)))
        cluster *= 2;
    p.slice = static_cast<int>(slice_of(cluster));
    p.slots = 1;
    while (p.slots < std::min(2 * p.k, RALM_MAX_K)) p.slots *= 2;
    const size_t hash = p.k > 0 ? p.slots * 16 : 0, bytes = p.slice * sizeof(T);
    if (bytes > kMixMaxStage) return launch_cluster(mix_kernel<T, false>, R, cluster, kMixThreads, hash, st, p);
    if (!allow_smem<mix_kernel<T, true>>(kMixMaxStage + 16 * RALM_MAX_K)) return RALM_ERR_CUDA;
    return launch_cluster(mix_kernel<T, true>, R, cluster, kMixThreads, bytes + hash, st, p);
}

bool pages_ok(const ralm_pages_t *p) {
    return p && p->pages >= 0 && p->rows >= 0 && p->rows <= RALM_MAX_ROWS && p->max_pages >= 1 &&
           p->max_pages <= RALM_MAX_ROW_PAGES && p->page_size >= 1 &&
           static_cast<int64_t>(p->max_pages) * p->page_size < (int64_t{1} << 31) - 1 &&
           (p->rows == 0 || (p->table && p->lengths)) && (p->pages == 0 || p->refs) && p->status && p->workspace;
}
bool pool_ok(const ralm_pages_t *p) {
    return p->pool && aligned16(p->pool) && p->layers >= 1 && p->layers <= (1 << 20) && p->page_bytes >= 16 && p->page_bytes % 16 == 0 &&
           p->layer_stride % 16 == 0 && (p->layers == 1 || p->layer_stride >= p->page_bytes * p->pages);
}
ralm_status_t launch_copy(const PagesCopyParams &p, int64_t most, cudaStream_t st) {
    const int sms = sm_count();
    if (sms == 0) return RALM_ERR_CUDA;
    const int64_t jobs = most * std::max(p.layers, 1) * ((p.page_bytes + 16383) / 16384);
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(jobs, 8LL * sms));
    return launch(pages_copy_kernel, blocks, kCopyThreads, 0, st, p);
}
PagesCopyParams copy_in_pool(const ralm_pages_t &p) {
    PagesCopyParams c = {};
    c.src = c.dst = static_cast<unsigned char *>(p.pool);
    c.src_layer_stride = c.dst_layer_stride = p.layer_stride;
    c.page_bytes = p.page_bytes;
    c.layers = p.pool ? static_cast<int>(p.layers) : 0;
    c.src_pages = c.dst_pages = p.pages;
    const PagesWork w = pages_work(p);
    c.from = w.from;
    c.to = w.to;
    c.count = w.head;
    return c;
}

bool kv_ok(const ralm_kv_t *c, int32_t layer) {
    if (!c || !pages_ok(&c->pages) || !pool_ok(&c->pages)) return false;
    const ralm_pages_t &p = c->pages;
    return p.pages >= 1 && c->kv_heads >= 1 && c->kv_heads <= 4096 && (p.page_size == 16 || p.page_size == 32 || p.page_size == 64) && layer >= 0 &&
           layer < p.layers && p.page_bytes == static_cast<int64_t>(c->kv_heads) * p.page_size * (c->head_dim + 8);
}
KvParams kv_params(const ralm_kv_t &c, int32_t layer, const int32_t *rows, int batch) {
    const ralm_pages_t &p = c.pages;
    KvParams k;
    k.layer = static_cast<unsigned char *>(p.pool) + layer * p.layer_stride;
    k.page_bytes = p.page_bytes;
    k.table = p.table;
    k.lengths = p.lengths;
    k.refs = p.refs;
    k.status = p.status;
    k.table_rows = p.rows;
    k.max_pages = p.max_pages;
    k.pages = p.pages;
    k.page_size = p.page_size;
    k.page_shift = p.page_size == 16 ? 4 : p.page_size == 32 ? 5 : 6;
    k.heads = c.kv_heads;
    k.rows = rows;
    k.batch = batch;
    return k;
}

template <typename T, int D>
ralm_status_t launch_tokens(bool append, const KvParams &k, const KvTokens &t, int sms, cudaStream_t st) {
    const int64_t jobs = static_cast<int64_t>(k.batch) * kv_blocks(t.n) * k.heads;
    if (jobs >= (int64_t{1} << 31)) return RALM_ERR_UNSUPPORTED;
    const int blocks = static_cast<int>(std::min<int64_t>((jobs + kKvThreads / 32 - 1) / (kKvThreads / 32), 32LL * sms));
    return launch(append ? kv_append_kernel<T, D> : kv_read_kernel<T, D>, blocks, kKvThreads, 0, st, k, t);
}
ralm_status_t kv_tokens(bool append, const ralm_kv_t *c, int32_t layer, const ralm_kv_tokens_t *t, void *stream) {
    if (!kv_ok(c, layer) || !t || t->batch < 0 || t->n < 0 || (t->dtype != RALM_F16 && t->dtype != RALM_BF16))
        return RALM_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return RALM_ERR_UNSUPPORTED;
    if (t->batch == 0 || t->n == 0) return RALM_OK;
    if (!t->k || !t->v || !t->starts) return RALM_ERR_INVALID_ARG;
    if (!append &&                                                   // K and V of a read are both written
        Runs(t->k, 2LL * c->head_dim, {{t->batch, 2 * t->k_stride_b}, {t->n, 2 * t->k_stride_n}, {c->kv_heads, 2 * t->k_stride_h}})
            .overlaps(Runs(t->v, 2LL * c->head_dim, {{t->batch, 2 * t->v_stride_b}, {t->n, 2 * t->v_stride_n}, {c->kv_heads, 2 * t->v_stride_h}})))
        return RALM_ERR_INVALID_ARG;
    const int sms = sm_count();
    if (sms == 0) return RALM_ERR_CUDA;
    const KvParams k = kv_params(*c, layer, t->rows, t->batch);
    const KvTokens x = {t->k, t->v, t->k_stride_b, t->k_stride_n, t->k_stride_h, t->v_stride_b, t->v_stride_n, t->v_stride_h,
                        t->n, t->starts, t->count,
                        aligned16(t->k) && aligned16(t->v) && t->k_stride_b % 8 == 0 && t->k_stride_n % 8 == 0 &&
                            t->k_stride_h % 8 == 0 && t->v_stride_b % 8 == 0 && t->v_stride_n % 8 == 0 && t->v_stride_h % 8 == 0};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (t->dtype == RALM_F16)
        return c->head_dim == 64 ? launch_tokens<__half, 64>(append, k, x, sms, st) : launch_tokens<__half, 128>(append, k, x, sms, st);
    return c->head_dim == 64 ? launch_tokens<__nv_bfloat16, 64>(append, k, x, sms, st)
                             : launch_tokens<__nv_bfloat16, 128>(append, k, x, sms, st);
}

// Column blocks of 8 query rows that one pass over the keys serves: up to 4, the rows evenly cut.
int attend_nt(int64_t rows) {
    const int64_t blocks = std::max<int64_t>((rows + 31) / 32, 1);
    return static_cast<int>(std::max<int64_t>((rows + 8 * blocks - 1) / (8 * blocks), 1));
}
int64_t attend_counters(int sms) { return (sms + 63) / 64 * 64; }
int attend_workers(int nt, int head_dim, int sms) { return sms * attend_warps(nt, head_dim); }

template <typename T, int D, int NT>
ralm_status_t launch_attend(AttendParams p, int sms, cudaStream_t st) {
    constexpr int kThreads = attend_warps(NT, D) * 32;
    constexpr int kRing = attend_warps(NT, D) * attend_warp_bytes(NT, D);
    const int cum = (p.kv.batch + 1) * static_cast<int>(sizeof(int));
    if (!allow_smem<attend_kernel<T, D, NT>>(kRing + (kAttendMaxBatch + 1) * static_cast<int>(sizeof(int)))) return RALM_ERR_CUDA;
    p.workers = attend_workers(NT, D, sms);
    p.part_ml = reinterpret_cast<float *>(p.counters + attend_counters(sms));
    p.cta_ml = p.part_ml + static_cast<int64_t>(2) * p.workers * 8 * NT * 2;
    p.part = p.cta_ml + static_cast<int64_t>(2) * attend_counters(sms) * 8 * NT * 2;
    p.cta_part = p.part + static_cast<int64_t>(2) * p.workers * 8 * NT * D;
    return launch(attend_kernel<T, D, NT>, sms, kThreads, kRing + cum, st, p);
}
template <typename T, int D>
ralm_status_t launch_attend(const AttendParams &p, int nt, int sms, cudaStream_t st) {
    switch (nt) {
        case 1: return launch_attend<T, D, 1>(p, sms, st);
        case 2: return launch_attend<T, D, 2>(p, sms, st);
        case 3: return launch_attend<T, D, 3>(p, sms, st);
    }
    return launch_attend<T, D, 4>(p, sms, st);
}

}  // namespace

extern "C" {

ralm_status_t ralm_knn_mix(const void *logits, ralm_dtype_t dtype, int64_t ld_logits, int32_t R, int32_t V,
                           const int64_t *ids, const float *scores, int32_t k, ralm_metric_t metric,
                           const int32_t *values, int64_t N, float lambda, float temperature,
                           float knn_temperature, float *probs, int64_t ld_probs, void *stream) {
    if (R < 0 || V < 1 || V > RALM_MAX_VOCAB || ld_logits < V || ld_probs < V || k < 0 || k > RALM_MAX_K || N < 0)
        return RALM_ERR_INVALID_ARG;
    if (dtype != RALM_F16 && dtype != RALM_BF16 && dtype != RALM_F32) return RALM_ERR_INVALID_ARG;
    if (metric != RALM_IP && metric != RALM_L2) return RALM_ERR_INVALID_ARG;
    if (!(lambda >= 0.f && lambda <= 1.f) || !(temperature > 0.f) || !(knn_temperature > 0.f) || std::isinf(temperature) ||
        std::isinf(knn_temperature) || std::isinf(kLog2e / temperature) || std::isinf(kLog2e / knn_temperature))
        return RALM_ERR_INVALID_ARG;
    if (R == 0) return RALM_OK;
    if (!logits || !probs || (k > 0 && (!ids || !scores || (N > 0 && !values)))) return RALM_ERR_INVALID_ARG;
    const int64_t size = dtype == RALM_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % size != 0) return RALM_ERR_INVALID_ARG;
    if (static_cast<int64_t>(R) * kMixMaxCluster >= (int64_t{1} << 31)) return RALM_ERR_INVALID_ARG;
    const Runs written(probs, 4 * static_cast<int64_t>(V), {{R, 4 * ld_probs}});
    if (written.overlaps(Runs(logits, size * V, {{R, size * ld_logits}})) || written.overlaps(dense(ids, 8LL * R * k)) ||
        written.overlaps(dense(scores, 4LL * R * k)) || (k > 0 && written.overlaps(dense(values, 4 * N))))
        return RALM_ERR_INVALID_ARG;
    const int sms = sm_count();
    if (sms == 0) return RALM_ERR_CUDA;
    MixParams p;
    p.logits = logits;
    p.ld_logits = ld_logits;
    p.V = V;
    p.ids = ids;
    p.scores = scores;
    p.k = k;
    p.values = values;
    p.N = N;
    p.score_sign = metric == RALM_L2 ? -1.f : 1.f;
    p.score_scale = kLog2e / knn_temperature;
    p.logit_scale = kLog2e / temperature;
    p.lambda = lambda;
    p.probs = probs;
    p.ld_probs = ld_probs;
    p.slice = 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == RALM_F16) return launch_mix<__half>(p, R, sms, st);
    if (dtype == RALM_BF16) return launch_mix<__nv_bfloat16>(p, R, sms, st);
    return launch_mix<float>(p, R, sms, st);
}

ralm_status_t ralm_verify_tokens(const int64_t *draft_tokens, const float *draft_probs, int64_t draft_ld_r,
                                 int64_t draft_ld_s, const float *target_probs, int64_t target_ld_r,
                                 int64_t target_ld_s, const float *uniforms, const int32_t *draft_len, int32_t R,
                                 int32_t S, int32_t V, int64_t *tokens, int32_t *accepted, void *stream) {
    if (R < 0 || S < 0 || S > (1 << 20) || V < 1 || V > RALM_MAX_VOCAB) return RALM_ERR_INVALID_ARG;
    if (R == 0) return RALM_OK;
    if ((S > 0 && !draft_tokens) || !target_probs || !uniforms || !tokens || !accepted) return RALM_ERR_INVALID_ARG;
    if (static_cast<int64_t>(R) * kVtMaxCluster >= (int64_t{1} << 31)) return RALM_ERR_INVALID_ARG;
    // the CTAs of a request all read its inputs, and one of them writes its outputs while they do
    const Runs out[2] = {dense(tokens, 8LL * R * (S + 1)), dense(accepted, 4LL * R)};
    if (out[0].overlaps(out[1])) return RALM_ERR_INVALID_ARG;
    for (const Runs &o : out)
        if (o.overlaps(dense(draft_tokens, 8LL * R * S)) || o.overlaps(dense(uniforms, 4LL * R * (S + 1))) ||
            o.overlaps(dense(draft_len, 4LL * R)) ||
            o.overlaps(Runs(draft_probs, 4LL * V, {{R, 4 * draft_ld_r}, {S, 4 * draft_ld_s}})) ||
            o.overlaps(Runs(target_probs, 4LL * V, {{R, 4 * target_ld_r}, {S + 1LL, 4 * target_ld_s}})))
            return RALM_ERR_INVALID_ARG;
    const int sms = sm_count();
    if (sms == 0) return RALM_ERR_CUDA;
    VerifyTokensParams p;
    p.draft = draft_tokens;
    p.draft_probs = S > 0 ? draft_probs : nullptr;
    p.draft_ld_r = draft_ld_r;
    p.draft_ld_s = draft_ld_s;
    p.target_probs = target_probs;
    p.target_ld_r = target_ld_r;
    p.target_ld_s = target_ld_s;
    p.uniforms = uniforms;
    p.draft_len = draft_len;
    p.S = S;
    p.V = V;
    p.tokens = tokens;
    p.accepted = accepted;
    // cut over a cluster while that adds CTAs that the GPU can hold at once
    int cluster = 1;
    while (cluster < kVtMaxCluster && 2LL * R * cluster <= 2LL * sms && V / (2 * cluster) >= 2 * kVtThreads) cluster *= 2;
    p.slice = (V + cluster - 1) / cluster;
    return launch_cluster(verify_tokens_kernel, R, cluster, kVtThreads, 0, static_cast<cudaStream_t>(stream), p);
}

int64_t ralm_pages_workspace(int32_t pages) {
    return pages < 0 ? 0 : pages_workspace_words(pages) * static_cast<int64_t>(sizeof(int32_t));
}

ralm_status_t ralm_pages_resize(const ralm_pages_t *pages, const int32_t *new_lengths, void *stream) {
    if (!pages_ok(pages) || (pages->pool && !pool_ok(pages))) return RALM_ERR_INVALID_ARG;
    if (pages->rows == 0) return RALM_OK;
    if (!new_lengths) return RALM_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const ralm_status_t rs = launch(pages_resize_kernel, 1, kPagesThreads, 0, st, *pages, new_lengths);
    if (rs != RALM_OK || !pages->pool) return rs;
    return launch_copy(copy_in_pool(*pages), std::min(pages->rows, pages->pages), st);   // at most one page per row
}

ralm_status_t ralm_pages_fork(const ralm_pages_t *pages, const int32_t *src, const int32_t *dst, int32_t n, void *stream) {
    if (!pages_ok(pages) || n < 0 || n > pages->rows) return RALM_ERR_INVALID_ARG;
    if (n == 0) return RALM_OK;
    if (!src || !dst) return RALM_ERR_INVALID_ARG;
    return launch(pages_fork_kernel, 1, kPagesThreads, (pages->rows + 31) / 32 * sizeof(int), static_cast<cudaStream_t>(stream), *pages,
                  src, dst, n);
}

ralm_status_t ralm_pages_compact(const ralm_pages_t *pages, int32_t *live, void *stream) {
    if (!pages_ok(pages) || (pages->pool && !pool_ok(pages)) || !live) return RALM_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const ralm_status_t rs = launch(pages_compact_kernel, 1, kPagesThreads, 0, st, *pages, live);
    if (rs != RALM_OK) return rs;
    PagesCopyParams c = copy_in_pool(*pages);
    c.table = pages->table;
    c.table_words = static_cast<int64_t>(pages->rows) * pages->max_pages;
    c.remap = pages_work(*pages).list;
    c.remap_pages = pages->pages;
    return launch_copy(c, std::max<int64_t>(pages->pages / 2, c.table_words / (kCopyThreads * 8)), st);
}

ralm_status_t ralm_pages_copy(const ralm_pages_t *src, const int32_t *from, const ralm_pages_t *dst, const int32_t *to,
                              int32_t n, void *stream) {
    if (!src || !dst || n < 0 || !pool_ok(src) || !pool_ok(dst) || src->page_bytes != dst->page_bytes || src->layers != dst->layers)
        return RALM_ERR_INVALID_ARG;
    if (n == 0) return RALM_OK;
    if (!from || !to || !dst->status) return RALM_ERR_INVALID_ARG;
    PagesCopyParams c = {};
    c.src = static_cast<const unsigned char *>(src->pool);
    c.dst = static_cast<unsigned char *>(dst->pool);
    c.src_layer_stride = src->layer_stride;
    c.dst_layer_stride = dst->layer_stride;
    c.page_bytes = src->page_bytes;
    c.layers = static_cast<int>(src->layers);
    c.src_pages = src->pages;
    c.dst_pages = dst->pages;
    c.from = from;
    c.to = to;
    c.n = n;
    c.status = dst->status;
    return launch_copy(c, n, static_cast<cudaStream_t>(stream));
}

ralm_status_t ralm_pages_status(const ralm_pages_t *pages, void *stream) {
    if (!pages || !pages->status) return RALM_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int word = 0;
    if (cudaMemcpyAsync(&word, pages->status, sizeof(int), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaMemsetAsync(pages->status, 0, sizeof(int), st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return RALM_ERR_CUDA;
    if (word == kStatusTimeout) return RALM_ERR_TIMEOUT;
    if (word == kStatusNoPages) return RALM_ERR_OOM;
    if (word == kStatusInvalid) return RALM_ERR_INVALID_ARG;
    return word == 0 ? RALM_OK : RALM_ERR_CUDA;
}

ralm_status_t ralm_kv_append(const ralm_kv_t *cache, int32_t layer, const ralm_kv_tokens_t *tokens, void *stream) {
    return kv_tokens(true, cache, layer, tokens, stream);
}
ralm_status_t ralm_kv_read(const ralm_kv_t *cache, int32_t layer, const ralm_kv_tokens_t *tokens, void *stream) {
    return kv_tokens(false, cache, layer, tokens, stream);
}

int64_t ralm_kv_attend_workspace(int32_t kv_heads, int32_t head_dim, int32_t q_heads, int32_t n) {
    if (kv_heads < 1 || q_heads < kv_heads || q_heads % kv_heads != 0 || n < 0 || (head_dim != 64 && head_dim != 128)) return 0;
    const int64_t rows = static_cast<int64_t>(q_heads / kv_heads) * n;
    const int nt = attend_nt(rows);
    const int sms = std::max(sm_count(), 1);
    return attend_counters(sms) * static_cast<int64_t>(sizeof(int)) +
           static_cast<int64_t>(2) * (attend_workers(nt, head_dim, sms) + attend_counters(sms)) * 8 * nt * (head_dim + 2) * sizeof(float);
}

ralm_status_t ralm_kv_attend(const ralm_kv_t *cache, int32_t layer, const ralm_attend_t *a, void *stream) {
    if (!kv_ok(cache, layer) || !a || a->batch < 0 || a->batch > RALM_MAX_ATTEND_BATCH || a->n < 0 || a->q_heads < 1 ||
        a->q_heads % cache->kv_heads != 0 || (a->dtype != RALM_F16 && a->dtype != RALM_BF16) || !std::isfinite(a->scale * kLog2e))
        return RALM_ERR_INVALID_ARG;
    if (cache->head_dim != 64 && cache->head_dim != 128) return RALM_ERR_UNSUPPORTED;
    if (a->batch == 0 || a->n == 0) return RALM_OK;
    if (!a->q || !a->out || !a->workspace || !aligned16(a->workspace)) return RALM_ERR_INVALID_ARG;
    if (Runs(a->out, 2LL * cache->head_dim, {{a->batch, 2 * a->out_stride_b}, {a->n, 2 * a->out_stride_n}, {a->q_heads, 2 * a->out_stride_h}})
            .overlaps(Runs(a->q, 2LL * cache->head_dim, {{a->batch, 2 * a->q_stride_b}, {a->n, 2 * a->q_stride_n}, {a->q_heads, 2 * a->q_stride_h}})))
        return RALM_ERR_INVALID_ARG;
    const int group = a->q_heads / cache->kv_heads;
    const int64_t rows = static_cast<int64_t>(group) * a->n;
    const ralm_pages_t &pg = cache->pages;
    if (rows > (1 << 20) ||
        static_cast<int64_t>(a->batch) * ((static_cast<int64_t>(pg.max_pages) * pg.page_size + 15) / 16) >= (int64_t{1} << 31))
        return RALM_ERR_UNSUPPORTED;
    if (a->workspace_bytes < ralm_kv_attend_workspace(cache->kv_heads, cache->head_dim, a->q_heads, a->n)) return RALM_ERR_INVALID_ARG;
    const int sms = sm_count();
    if (sms == 0) return RALM_ERR_CUDA;
    const int nt = attend_nt(rows);
    AttendParams p;
    p.kv = kv_params(*cache, layer, a->rows, a->batch);
    p.q = a->q;
    p.out = a->out;
    p.q_b = a->q_stride_b;
    p.q_n = a->q_stride_n;
    p.q_h = a->q_stride_h;
    p.o_b = a->out_stride_b;
    p.o_n = a->out_stride_n;
    p.o_h = a->out_stride_h;
    p.q_len = a->q_len;
    p.n = a->n;
    p.group = group;
    p.row_blocks = static_cast<int>((rows + 8 * nt - 1) / (8 * nt));
    p.scale = a->scale * kLog2e;
    p.counters = static_cast<int *>(a->workspace);
    p.vec = aligned16(a->q) && a->q_stride_b % 8 == 0 && a->q_stride_n % 8 == 0 && a->q_stride_h % 8 == 0;
    if (static_cast<int64_t>(a->batch) * cache->kv_heads * p.row_blocks >= (int64_t{1} << 31)) return RALM_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->dtype == RALM_F16)
        return cache->head_dim == 64 ? launch_attend<__half, 64>(p, nt, sms, st) : launch_attend<__half, 128>(p, nt, sms, st);
    return cache->head_dim == 64 ? launch_attend<__nv_bfloat16, 64>(p, nt, sms, st) : launch_attend<__nv_bfloat16, 128>(p, nt, sms, st);
}

}  // extern "C"
