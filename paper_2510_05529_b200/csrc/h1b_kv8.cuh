// 8-bit pages (h1b_kv8_*): what the append / read / attention kernels share. Parameter blocks, the walk over a ragged
// batch, and the conversion of 8-bit codes to fp16 operands.
#pragma once
#include <atomic>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/h1b.h"
#include "h1b_ptx.cuh"

namespace h1b {

constexpr int kKv8Block = 16;              // tokens that are handled together; a page holds whole blocks
constexpr float kLn2 = 0.693147180559945309f;

struct Kv8Params {
    uint8_t *k, *v;
    float *ks, *vs;
    const int32_t *table, *kv_len, *row_start;
    int32_t *status;
    int n_pages, hkv, page_tokens;
    int n_seqs, table_width, n_rows;
    int cap;                               // table_width * page_tokens
    uint32_t page_mul;                     // block / (page_tokens / 16) = block * page_mul >> page_shift, exactly, for
    int page_shift;                        // block < 2^26 (all that 2^30 tokens have)
};

struct Kv8Attn {
    const void *q;
    void *out;
    float *lse;
    int64_t q_rs, q_hs, o_rs, o_hs;
    int hq, group;                         // query heads, query heads per KV head
    int bf16;
    float scale_log2;                      // scale * log2(e)
    int window, sinks;
    int splits;                            // most parts a tile's tokens are dealt into
    int tiles;                             // few rows: tiles of a sequence that have a block each; many: the most tiles there are
    int min_pairs;                         // sequences with fewer (row, head of the group) pairs are another kernel's ...
    int max_pairs;                         // ... and those with more
    int cluster;                           // few rows: the parts of a tile are a cluster and join by themselves
    float *part_acc, *part_lse;            // [tiles][hkv][pairs of a tile][splits] times [d], and alone (log2)
};

__device__ __forceinline__ void kv8_report(const Kv8Params &P, int code) {
    if (P.status) *P.status = code;        // any one of several stays: the host asks whether there was one
}

// The entry of a sequence's table that block `block` (of 16 tokens) lies in.
__device__ __forceinline__ int kv8_page_of(const Kv8Params &P, int block) {
    return (int)((uint64_t)(uint32_t)block * P.page_mul >> P.page_shift);
}

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

struct Kv8Seq {
    int b, start, n, kv;                   // sequence, its first row, rows, cached tokens
};

// Whole warp: the rows of sequence `i` (n = 0 beyond the last). Whatever row_start holds, rows stay inside the tensors.
__device__ __forceinline__ Kv8Seq kv8_seq(const Kv8Params &P, int i) {
    Kv8Seq s{i, 0, 0, 0};
    if (i < P.n_seqs) {
        const int st = P.row_start[i], en = P.row_start[i + 1], kv = P.kv_len[i];
        s.start = clampi(st, 0, P.n_rows);
        s.n = clampi(en, s.start, P.n_rows) - s.start;
        s.kv = clampi(kv, 0, 1 << 30);
        if (s.start != st || s.start + s.n != en || kv < 0) kv8_report(P, H1B_ERR_INVALID_ARG);
        else if (kv > P.cap) kv8_report(P, H1B_ERR_CAPACITY);
    }
    return s;
}

__device__ __forceinline__ Kv8Seq kv8_seq_from_lane(const Kv8Seq &s, int b, int src) {
    return {b, __shfl_sync(~0u, s.start, src), __shfl_sync(~0u, s.n, src), __shfl_sync(~0u, s.kv, src)};
}

// Whole warp `first` of `step`: a share of the sequences is looked at for what does not fit. (Up to 32 are looked at by every
// warp that walks over them; of more, those without rows might be passed over by all.)
__device__ __forceinline__ void kv8_check_batch(const Kv8Params &P, uint32_t first, uint32_t step, int lane) {
    if (P.n_seqs <= 32 || !P.status) return;
    for (uint64_t i = first; i * 32 < (uint32_t)P.n_seqs; i += step) (void)kv8_seq(P, (int)i * 32 + lane);
}

// Whole warp: the sequence that row r belongs to; false if it is nobody's. row_start is searched 32 entries at a time.
__device__ __forceinline__ bool kv8_seq_of_row(const Kv8Params &P, int r, int lane, Kv8Seq *out) {
    int base = 0, count = P.n_seqs;
    while (count > 32) {
        const int step = (count + 31) / 32, i = base + lane * step;
        const int below = __popc(__ballot_sync(~0u, i < base + count && P.row_start[min(i, P.n_seqs)] <= r));
        if (below == 0) return false;
        const int next = base + (below - 1) * step;
        count = min(step, base + count - next);
        base = next;
    }
    const Kv8Seq s = kv8_seq(P, lane < count ? base + lane : P.n_seqs);
    const unsigned hit = __ballot_sync(~0u, r >= s.start && r < s.start + s.n);
    if (!hit) return false;
    const int src = __ffs(hit) - 1;
    *out = kv8_seq_from_lane(s, base + src, src);
    return true;
}

// Whole warp: tile `idx` of the batch. The (row, head of the group) pairs of a sequence, pair = row * group + head, are cut
// into tiles of R; sequences outside [min_pairs, max_pairs] have none. False if there are not that many tiles.
__device__ __forceinline__ bool kv8_find_tile(const Kv8Params &P, const Kv8Attn &A, int idx, int R, int lane, Kv8Seq *out,
                                              int *tile) {
    int before = 0;
    for (int base = 0; base < P.n_seqs; base += 32) {
        const Kv8Seq s = kv8_seq(P, base + lane);
        const int pairs = s.n * A.group;
        int upto = pairs >= A.min_pairs && pairs <= A.max_pairs ? (pairs + R - 1) / R : 0;
        const int own = upto;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(~0u, upto, o);
            if (lane >= o) upto += x;
        }
        const unsigned hit = __ballot_sync(~0u, idx - before < upto);
        if (hit) {
            const int src = __ffs(hit) - 1;
            *out = kv8_seq_from_lane(s, base + src, src);
            *tile = idx - before - __shfl_sync(~0u, upto - own, src);
            return true;
        }
        before += __shfl_sync(~0u, upto, 31);
    }
    return false;
}

// The tokens that a tile's rows see, in blocks of 16: the sinks' blocks, then the window's (without a window: all).
struct Kv8Span {
    int lo, hi;                            // a token is seen by some row of the tile iff lo <= t <= hi or t < sinks
    int sinks;                             // 0 when the sinks are part of lo .. hi
    int sink_blocks, first, count;
    __device__ __forceinline__ int token(int j) const {
        return (j < sink_blocks ? j : first + j - sink_blocks) * kKv8Block;
    }
};
__device__ __forceinline__ Kv8Span kv8_span(const Kv8Params &P, const Kv8Attn &A, int pos_first, int pos_last) {
    Kv8Span s;
    s.hi = min(pos_last, P.cap - 1);
    s.lo = A.window ? max(0, pos_first - A.window + 1) : 0;
    s.sinks = min(A.sinks, s.lo);
    if (s.sinks > s.hi + 1) s.sinks = max(0, s.hi + 1);
    s.first = s.lo / kKv8Block;
    const int body = s.hi >= s.lo ? s.hi / kKv8Block - s.first + 1 : 0;
    s.sink_blocks = min((s.sinks + kKv8Block - 1) / kKv8Block, s.first);
    s.count = s.sink_blocks + body;
    return s;
}

// Four 8-bit codes -> two fp16 pairs, exactly. int8: 1024 + 128 + code assembled in the mantissa, minus 1152 (five
// instructions); e4m3: the conversion instruction, which takes a pair from the lower half of a register (three). A NaN
// pattern of e4m3, which no row that was appended holds, stays one.
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t w) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)w));
    return r;
}
template <int FMT>
__device__ __forceinline__ void kv8_codes4(uint32_t w, uint32_t &h01, uint32_t &h23) {
    if (FMT == H1B_KV8_INT8) {
        w ^= 0x80808080u;
        h01 = sub_f16x2(__byte_perm(w, 0x64646464u, 0x4140), 0x64806480u);
        h23 = sub_f16x2(__byte_perm(w, 0x64646464u, 0x4342), 0x64806480u);
    } else {
        h01 = e4m3x2_to_f16x2(w);
        h23 = e4m3x2_to_f16x2(w >> 16);
    }
}
// Codes of the same four channels of two tokens a, b -> pairs (a_i, b_i), i = 0 .. 3.
template <int FMT>
__device__ __forceinline__ void kv8_codes4x2(uint32_t a, uint32_t b, uint32_t (&h)[4]) {
    kv8_codes4<FMT>(__byte_perm(a, b, 0x5140), h[0], h[1]);
    kv8_codes4<FMT>(__byte_perm(a, b, 0x7362), h[2], h[3]);
}

__device__ __forceinline__ float2 pair_to_float2(uint32_t w, int bf16) {
    if (bf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    return half2_bits_to_float2(w);
}
__device__ __forceinline__ uint32_t float2_to_pair(float a, float b, int bf16) {
    if (!bf16) return pack_f16x2(a, b);
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }   // -126 <= e <= 127

// Two fp32 numbers in one register pair, and the packed operations on them.
__device__ __forceinline__ uint64_t pack2(uint32_t lo, uint32_t hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ uint64_t pack2f(float lo, float hi) { return pack2(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ float2 unpack2(uint64_t v) {
    uint32_t lo, hi;
    asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(v));
    return make_float2(__uint_as_float(lo), __uint_as_float(hi));
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// A query row is handed to the tensor cores as fp16 whatever its type: multiplied by 2^-e so that its largest number
// lies in [2^14, 2^15). fp16 then holds every bit of it down to 2^-28 of that number, and numbers below to 2^-39 of it.
__device__ __forceinline__ int kv8_row_exponent(float amax) {
    if (!(amax > 0.f) || !(amax <= 3.402823466e38f)) return 0;
    const int e = (int)(__float_as_uint(amax) >> 23) - 127 - 14;   // (a subnormal amax: -141, clamped)
    return clampi(e, -100, 113);
}

// A kernel's launch attribute, set once on each device (again if two threads meet: it is the same value).
struct Kv8Once {
    std::atomic<uint64_t> done{0};
    cudaError_t shared_memory(const void *kernel, int bytes) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const uint64_t bit = dev < 64 ? 1ull << dev : 0;
        if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
        return e;
    }
};

cudaError_t launch_kv8_append(const Kv8Params &P, const h1b_kv8_rows &k, const h1b_kv8_rows &v, int d, int fmt, int bf16,
                              cudaStream_t st);
cudaError_t launch_kv8_read(const Kv8Params &P, const h1b_kv8_rows &k, const h1b_kv8_rows &v, int d, int fmt, int bf16,
                            cudaStream_t st);
cudaError_t launch_kv8_rows(const Kv8Params &P, const Kv8Attn &A, int d, int fmt, int rows_per_tile, cudaStream_t st);

cudaError_t launch_kv8_tiles(const Kv8Params &P, const Kv8Attn &A, int d, int fmt, cudaStream_t st);
cudaError_t launch_kv8_join(const Kv8Params &P, const Kv8Attn &A, int d, int rows_per_tile, int unit_blocks, int min_blocks,
                            cudaStream_t st);

// A launch whose error is its own (and not one that somebody left behind).
template <class Kernel, class... Args>
cudaError_t kv8_launch(Kernel kernel, dim3 grid, int threads, int smem, cudaStream_t st, const Args &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

int report_error(int code, const char *fmt, ...);      // h1b_api.cu: the text behind h1b_last_error(NULL)

}  // namespace h1b
