// Host side of the 8-bit pages (h1b_kv8_*): checks of the arguments, launch shapes, launches.
#include <algorithm>
#include <cmath>

#include <cuda_runtime.h>

#include "h1b_kv8.cuh"

using namespace h1b;

namespace {

// The device of the pool for the length of a call; the caller's current device afterwards.
struct DeviceScope {
    int before = -1;
    cudaError_t err;
    explicit DeviceScope(int device) {
        err = cudaGetDevice(&before);
        if (err == cudaSuccess && before != device) err = cudaSetDevice(device);
        else if (err == cudaSuccess) before = -1;
    }
    ~DeviceScope() { if (before >= 0) cudaSetDevice(before); }
};

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_pool(const h1b_kv8_pool *p) {
    if (!p) return report_error(H1B_ERR_NULL, "pool is NULL");
    if (p->head_dim != 64 && p->head_dim != 128)
        return report_error(H1B_ERR_UNSUPPORTED, "head_dim = %d: 64 or 128", p->head_dim);
    if (p->format != H1B_KV8_INT8 && p->format != H1B_KV8_E4M3)
        return report_error(H1B_ERR_INVALID_ARG, "unknown format %d", p->format);
    if (p->n_pages < 1 || p->n_kv_heads < 1 || p->n_kv_heads > 1024 || p->device < 0)
        return report_error(H1B_ERR_INVALID_ARG, "n_pages = %d, n_kv_heads = %d, device = %d out of range", p->n_pages,
                            p->n_kv_heads, p->device);
    if (p->page_tokens < kKv8Block || p->page_tokens % kKv8Block)
        return report_error(H1B_ERR_INVALID_ARG, "page_tokens = %d: a multiple of %d", p->page_tokens, kKv8Block);
    if ((int64_t)p->n_pages * p->n_kv_heads > (int64_t)(1u << 31) / (p->page_tokens / kKv8Block) - 1)
        return report_error(H1B_ERR_UNSUPPORTED, "%d pages of %d tokens of %d heads: 2^35 or more rows", p->n_pages, p->page_tokens,
                            p->n_kv_heads);
    if (!p->k || !p->v || !p->k_scale || !p->v_scale) return report_error(H1B_ERR_NULL, "a pool pointer is NULL");
    if (!aligned16(p->k) || !aligned16(p->v) || !aligned16(p->k_scale) || !aligned16(p->v_scale))
        return report_error(H1B_ERR_INVALID_ARG, "a pool pointer is not 16-byte aligned");
    return H1B_OK;
}

int check_batch(const h1b_kv8_pool *p, const h1b_kv8_batch *b) {
    if (!b) return report_error(H1B_ERR_NULL, "batch is NULL");
    if (b->n_seqs < 0 || b->n_seqs > 1 << 20 || b->n_rows < 0 || b->table_width < 1)
        return report_error(H1B_ERR_INVALID_ARG, "n_seqs = %d, n_rows = %d, table_width = %d out of range", b->n_seqs,
                            b->n_rows, b->table_width);
    if ((int64_t)b->table_width * p->page_tokens > (1 << 30))
        return report_error(H1B_ERR_INVALID_ARG, "table_width * page_tokens = %lld exceeds 2^30",
                            (long long)b->table_width * p->page_tokens);
    if (b->n_seqs > 0 && (!b->block_table || !b->kv_len || !b->row_start))
        return report_error(H1B_ERR_NULL, "block_table, kv_len or row_start is NULL");
    return H1B_OK;
}

int check_rows(const char *name, const h1b_kv8_rows *t, int64_t rows, int heads, int d, bool output, bool nullable) {
    if (!t) return nullable ? H1B_OK : report_error(H1B_ERR_NULL, "%s is NULL", name);
    if (rows == 0) return H1B_OK;                                // nothing is read or written
    if (!t->data) return nullable ? H1B_OK : report_error(H1B_ERR_NULL, "%s.data is NULL", name);
    if (!aligned16(t->data)) return report_error(H1B_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
    if ((rows > 1 && t->row_stride % 8) || (heads > 1 && t->head_stride % 8))
        return report_error(H1B_ERR_INVALID_ARG, "strides of %s (%lld, %lld) are not multiples of 8", name,
                            (long long)t->row_stride, (long long)t->head_stride);
    if (output) {
        const int64_t rs = std::llabs(t->row_stride), hs = std::llabs(t->head_stride);
        const bool heads_inside = (heads == 1 || hs >= d) && (rows == 1 || rs >= (heads == 1 ? d : hs * (heads - 1) + d));
        const bool rows_inside = (rows == 1 || rs >= d) && (heads == 1 || hs >= (rows == 1 ? d : rs * (rows - 1) + d));
        if (!heads_inside && !rows_inside)
            return report_error(H1B_ERR_INVALID_ARG, "rows or heads of %s overlap (strides %lld, %lld)", name,
                                (long long)t->row_stride, (long long)t->head_stride);
    }
    return H1B_OK;
}

int check_type(int dtype) {
    if (dtype != H1B_TYPE_F16 && dtype != H1B_TYPE_BF16) return report_error(H1B_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    return H1B_OK;
}

Kv8Params params_of(const h1b_kv8_pool *p, const h1b_kv8_batch *b) {
    Kv8Params P;
    P.k = static_cast<uint8_t *>(p->k); P.v = static_cast<uint8_t *>(p->v);
    P.ks = p->k_scale; P.vs = p->v_scale;
    P.table = b->block_table; P.kv_len = b->kv_len; P.row_start = b->row_start; P.status = b->status;
    P.n_pages = p->n_pages; P.hkv = p->n_kv_heads; P.page_tokens = p->page_tokens;
    P.n_seqs = b->n_seqs; P.table_width = b->table_width; P.n_rows = b->n_rows;
    P.cap = b->table_width * p->page_tokens;
    // d = page_tokens / 16 <= 2^26: with k = 26 + ceil(log2 d) and m = ceil(2^k / d), block * m exceeds block * 2^k / d by less
    // than 2^26 * d / d = a unit of 2^k / 2^ceil(log2 d), which is too little to reach the next quotient
    const uint32_t d = (uint32_t)(p->page_tokens / kKv8Block);
    int log2d = 0;
    while ((1u << log2d) < d) ++log2d;
    P.page_shift = 26 + log2d;
    P.page_mul = (uint32_t)(((1ull << P.page_shift) + d - 1) / d);
    return P;
}

#define H1B_KV8_TRY(expr)                                                                                        \
    do {                                                                                                         \
        const cudaError_t e_ = (expr);                                                                           \
        if (e_ != cudaSuccess) {                                                                                 \
            (void)cudaGetLastError(); /* reported here, and not left for somebody else to find */                \
            return report_error(H1B_ERR_CUDA, "%s: %s", #expr, cudaGetErrorString(e_));                          \
        }                                                                                                        \
    } while (0)

int check_io(const h1b_kv8_pool *pool, const h1b_kv8_batch *batch, const h1b_kv8_rows *k, const h1b_kv8_rows *v, int dtype,
             bool output) {
    int rc = check_pool(pool);
    if (rc == H1B_OK) rc = check_batch(pool, batch);
    if (rc == H1B_OK) rc = check_rows("k", k, batch->n_rows, pool->n_kv_heads, pool->head_dim, output, output);
    if (rc == H1B_OK) rc = check_rows("v", v, batch->n_rows, pool->n_kv_heads, pool->head_dim, output, output);
    if (rc == H1B_OK) rc = check_type(dtype);
    if (rc == H1B_OK && (int64_t)batch->n_rows * pool->n_kv_heads >= (int64_t)1 << 31)
        return report_error(H1B_ERR_INVALID_ARG, "n_rows * n_kv_heads reaches 2^31");
    return rc;
}

// How the attention of a batch is launched; a function of sizes only. Sequences with at most kFewPairs (row, head of the
// group) pairs go to the kernel for few rows, the others to the tensor-core tiles; both are launched only when the host
// cannot tell that one of them has nothing to do. The border, in us, few rows / tiles (32 / 8 heads of 128): 8 sequences of
// 8k tokens, 32 pairs: 97 / 109, 48 pairs: 127 / 109; one of 16k tokens: 35 / 49, 41 / 49, 64 pairs: 47 / 50; 32 sequences of
// 2k tokens: 104 / 94, 124 / 95.
constexpr int kFewPairs = 32;

struct AttnPart {
    bool used = false, cluster = false;
    int rows_per_tile = 0, tiles = 0, splits = 1, min_pairs = 1, max_pairs = 1 << 30;
    size_t lines = 0;                                            // partial results
};
struct AttnPlan {
    AttnPart few, many;
    size_t bytes = 0;
};

AttnPlan plan_of(const h1b_kv8_pool *p, const h1b_kv8_batch *b, int hq, int window, int sinks, int max_rows) {
    AttnPlan a;
    const int64_t group = hq / p->n_kv_heads, pairs = (int64_t)b->n_rows * group;
    const int64_t rows = std::min<int64_t>(std::max(max_rows, 1), b->n_rows), most = rows * group;
    const int64_t seqs = std::min(b->n_seqs, b->n_rows);
    a.many.used = most > kFewPairs;
    const int64_t cap = (int64_t)b->table_width * p->page_tokens;
    const int64_t seen = window ? std::min<int64_t>(cap, (int64_t)window + sinks + rows + 32) : cap;
    // (The kernel for few rows is also left out where the tiles of all sequences together are less work than its launches:
    // five steps of 64 tokens an SM. Four sequences of 2-132 rows over 175 tokens: 24 us with it, 16 without.)
    a.few.used = !a.many.used || (b->n_seqs > 1 && rows * b->n_seqs > b->n_rows &&
                                  (pairs / 256 + seqs) * p->n_kv_heads * seen > 148 * 5 * 64);
    if (a.few.used) {
        AttnPart &f = a.few;
        if (a.many.used) f.max_pairs = kFewPairs;
        const int64_t here = std::min<int64_t>(most, f.max_pairs);
        f.rows_per_tile = here <= 8 ? 8 : 16;
        f.tiles = (int)((here + f.rows_per_tile - 1) / f.rows_per_tile);       // of a sequence
        // Parts. The GPU holds 148 * 4 blocks of 8-row tiles at once (half as many of 16 rows). Fill it once, as far as there
        // are 128 tokens for each block (two blocks of 16 a warp); fill it up to four times, so that ragged lengths even out,
        // where each block still has 1024 tokens (more and shorter ones cost: 32 sequences with a window of 1024 tokens took
        // 24 us in seven parts and 15 in two).
        const int64_t blocks = (int64_t)b->n_seqs * f.tiles * p->n_kv_heads, slots = f.rows_per_tile == 8 ? 148 * 4 : 148 * 2;
        const int64_t fill = std::min<int64_t>(slots / blocks, (seen + 127) / 128);
        int64_t even = 0;
        for (int64_t times = 4; times >= 1 && !even; --times)
            if (times * slots / blocks <= seen / 1024) even = times * slots / blocks;
        f.splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::max(fill, even), 256));
        // Up to eight parts (the largest cluster that every GPU takes) join through each other's shared memory, others through
        // the workspace and a kernel of its own, some 2 us more (one sequence of 777 tokens: 6.7 and 8.6 us). Blocks that come
        // in several waves do better without clusters, whose parts start and end together (16 sequences of 4-8k tokens, 32
        // heads: 155 us with, 150 without).
        f.cluster = f.splits > 1 && f.splits <= 8 && blocks * f.splits <= slots;
    }
    if (a.many.used) {
        AttnPart &m = a.many;
        if (a.few.used) m.min_pairs = kFewPairs + 1;
        m.rows_per_tile = 256;
        m.tiles = (int)(pairs / 256 + std::min<int64_t>(seqs, pairs / m.min_pairs));
        // Parts only where there are too few tiles for the SMs (one block an SM): up to three times as many blocks as SMs, so
        // that ragged lengths even out, each of at least 512 tokens (six sequences with 5 to 131 rows over 1-9k tokens: 206 us
        // at one block an SM, 172, 163 and 163 at two, three and four, 180 at six).
        const int64_t blocks = (int64_t)m.tiles * p->n_kv_heads;
        m.splits = blocks >= 148 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(3 * 148 / blocks, seen / 512));
    }
    for (AttnPart *part : {&a.few, &a.many})
        if (part->used && part->splits > 1 && !part->cluster) {
            part->lines = (size_t)part->tiles * (part == &a.few ? b->n_seqs : 1) * p->n_kv_heads * part->rows_per_tile * part->splits;
            a.bytes += part->lines * (p->head_dim + 1) * sizeof(float);
        }
    return a;
}

int check_attention(const h1b_kv8_pool *pool, const h1b_kv8_batch *batch, int hq, int window, int sinks, int max_rows) {
    int rc = check_pool(pool);
    if (rc == H1B_OK) rc = check_batch(pool, batch);
    if (rc != H1B_OK) return rc;
    if (hq < 1 || hq % pool->n_kv_heads || hq / pool->n_kv_heads > 128)
        return report_error(H1B_ERR_INVALID_ARG, "%d query heads over %d KV heads: a multiple, at most 128 times", hq,
                            pool->n_kv_heads);
    if ((int64_t)batch->n_rows * hq > (1 << 30))
        return report_error(H1B_ERR_INVALID_ARG, "n_rows * n_q_heads exceeds 2^30");
    if (window < 0 || sinks < 0 || window > (1 << 30) || sinks > (1 << 30) || max_rows < 0)
        return report_error(H1B_ERR_INVALID_ARG, "window = %d, sinks = %d, max_rows = %d out of range", window, sinks, max_rows);
    return H1B_OK;
}

}  // namespace

extern "C" {

int h1b_kv8_append(const h1b_kv8_pool *pool, const h1b_kv8_batch *batch, const h1b_kv8_rows *k, const h1b_kv8_rows *v,
                   int dtype, void *stream) {
    const int rc = check_io(pool, batch, k, v, dtype, false);
    if (rc != H1B_OK) return rc;
    if (batch->n_rows == 0 || batch->n_seqs == 0) return H1B_OK;
    DeviceScope dev(pool->device);
    H1B_KV8_TRY(dev.err);
    H1B_KV8_TRY(launch_kv8_append(params_of(pool, batch), *k, *v, pool->head_dim, pool->format, dtype,
                                  static_cast<cudaStream_t>(stream)));
    return H1B_OK;
}

int h1b_kv8_read(const h1b_kv8_pool *pool, const h1b_kv8_batch *batch, const h1b_kv8_rows *k, const h1b_kv8_rows *v,
                 int dtype, void *stream) {
    const int rc = check_io(pool, batch, k, v, dtype, true);
    if (rc != H1B_OK) return rc;
    const h1b_kv8_rows none{nullptr, 0, 0};
    const h1b_kv8_rows &kk = k ? *k : none, &vv = v ? *v : none;
    if (batch->n_rows == 0 || batch->n_seqs == 0 || (!kk.data && !vv.data)) return H1B_OK;
    DeviceScope dev(pool->device);
    H1B_KV8_TRY(dev.err);
    H1B_KV8_TRY(launch_kv8_read(params_of(pool, batch), kk, vv, pool->head_dim, pool->format, dtype,
                                static_cast<cudaStream_t>(stream)));
    return H1B_OK;
}

size_t h1b_kv8_attention_bytes(const h1b_kv8_pool *pool, const h1b_kv8_batch *batch, int n_q_heads, int window, int sinks,
                               int max_rows) {
    if (check_attention(pool, batch, n_q_heads, window, sinks, max_rows) != H1B_OK) return 0;
    if (batch->n_rows == 0 || batch->n_seqs == 0) return 0;
    return plan_of(pool, batch, n_q_heads, window, sinks, max_rows).bytes;
}

int h1b_kv8_attention(const h1b_kv8_pool *pool, const h1b_kv8_batch *batch, const h1b_kv8_rows *q, const h1b_kv8_rows *out,
                      float *lse, int n_q_heads, int dtype, float scale, int window, int sinks, int max_rows,
                      void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check_attention(pool, batch, n_q_heads, window, sinks, max_rows);
    if (rc == H1B_OK) rc = check_rows("q", q, batch->n_rows, n_q_heads, pool->head_dim, false, false);
    if (rc == H1B_OK) rc = check_rows("out", out, batch->n_rows, n_q_heads, pool->head_dim, true, false);
    if (rc == H1B_OK) rc = check_type(dtype);
    if (rc != H1B_OK) return rc;
    const float scale_log2 = (float)((double)scale * 1.4426950408889634074);
    if (!std::isfinite(scale_log2)) return report_error(H1B_ERR_INVALID_ARG, "scale or scale * log2(e) is not finite");
    if (batch->n_rows == 0 || batch->n_seqs == 0) return H1B_OK;
    const AttnPlan plan = plan_of(pool, batch, n_q_heads, window, sinks, max_rows);
    if (plan.bytes && (!workspace || workspace_bytes < plan.bytes || !aligned16(workspace)))
        return report_error(H1B_ERR_WORKSPACE, "workspace needs %zu bytes, 16-byte aligned (got %zu at %p)", plan.bytes,
                            workspace ? workspace_bytes : (size_t)0, workspace);
    DeviceScope dev(pool->device);
    H1B_KV8_TRY(dev.err);
    Kv8Attn A;
    A.q = q->data; A.out = out->data; A.lse = lse;
    A.q_rs = q->row_stride; A.q_hs = q->head_stride; A.o_rs = out->row_stride; A.o_hs = out->head_stride;
    A.hq = n_q_heads; A.group = n_q_heads / pool->n_kv_heads; A.bf16 = dtype == H1B_TYPE_BF16;
    A.scale_log2 = scale_log2;
    A.window = window; A.sinks = window ? sinks : 0;
    const Kv8Params P = params_of(pool, batch);
    float *at = static_cast<float *>(workspace);
    auto take = [&](const AttnPart &part) {                      // this part's share of the workspace
        A.splits = part.splits; A.tiles = part.tiles; A.min_pairs = part.min_pairs; A.max_pairs = part.max_pairs;
        A.cluster = part.cluster;
        A.part_acc = part.lines ? at : nullptr;
        A.part_lse = part.lines ? at + part.lines * pool->head_dim : nullptr;
        if (part.lines) at += part.lines * (pool->head_dim + 1);
    };
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (plan.many.used) {
        take(plan.many);
        H1B_KV8_TRY(launch_kv8_tiles(P, A, pool->head_dim, pool->format, st));
    }
    if (plan.few.used) {
        take(plan.few);
        H1B_KV8_TRY(launch_kv8_rows(P, A, pool->head_dim, pool->format, plan.few.rows_per_tile, st));
    }
    return H1B_OK;
}

}  // extern "C"
