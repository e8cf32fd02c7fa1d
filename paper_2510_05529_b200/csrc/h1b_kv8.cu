// 8-bit pages: quantise-and-append, read-back, and attention for few rows per sequence (decode steps, short chunks).
#include <type_traits>

#include "h1b_kv8.cuh"

namespace h1b {

namespace {

// ------------------------------------------------------------------------------------------------------------------
// Append and read. A row of d numbers is handled by d / 16 lanes (8 numbers of each half of the row, so that neighbouring
// lanes read and write neighbouring bytes), the keys and values of two (d = 128) or four heads side by side in one warp; a
// warp takes `heads` KV heads of one row, so the walk over the batch and the page table is done once for all of them, and the
// next heads' loads are under way while it works on these. A token of a head is 2 * 2 d bytes on one side and 2 (d + 4) on
// the other. Read is bound by memory: 8 sequences of 2-4k tokens, 32 heads of 128, 99 us = 6.1 TB/s, 94 % of the copy
// bandwidth. Append is bound by instruction issue (75 % of the slots; some 14 instructions a number): 8192 tokens of 32 heads
// of 128, 41.6 us = 4.9 TB/s, 74 %; with a division for each number it was 82, with a lane's addresses computed for each head
// 44.7. A grid of as many blocks as run at once, each looping over rows, took longer (append 2 us, read 30).
// ------------------------------------------------------------------------------------------------------------------
struct Kv8Io {
    Kv8Params P;
    h1b_kv8_rows k, v;
    int heads, groups;                     // heads per warp, warps per row
};

// Where row r's token lives: its place in the pool, in tokens of one KV head ((page * hkv + head) * page_tokens + offset
// with head = 0), or -1.
__device__ __forceinline__ int64_t kv8_place(const Kv8Params &P, const Kv8Seq &s, int r) {
    const int pos = s.kv - s.n + (r - s.start);
    if (pos < 0) { kv8_report(P, H1B_ERR_INVALID_ARG); return -1; }
    if (pos >= P.cap) { kv8_report(P, H1B_ERR_CAPACITY); return -1; }
    const int col = kv8_page_of(P, pos / kKv8Block), page = P.table[(int64_t)s.b * P.table_width + col];
    if (page < 0 || page >= P.n_pages) { kv8_report(P, H1B_ERR_BOUNDS); return -1; }
    return (int64_t)page * P.hkv * P.page_tokens + (pos - col * P.page_tokens);
}

// The codes of 16 numbers f and their row's amax. A code is the exact quotient TOP x / amax rounded once. TOP / amax,
// off by 2^-22 of itself at most, is moved up and down by 2^-21, so the exact quotient lies between the two products: where
// both round to the same code, that is the one. Elsewhere (one number in 5000, most of them ties) the lane divides: TOP x is
// exact in fp32 (7 + 11 bits), the division is correctly rounded, and a quotient of such numbers that is not on a border
// between two codes lies at least 2^-16 of itself away from it, so fp32 cannot put it there or across.
constexpr float kMagic = 12582912.f;                             // 1.5 * 2^23: the integer nearest to x lands in the low byte of x + kMagic
template <int FMT>
__device__ __forceinline__ uint32_t kv8_quantise4(float x, float y, float z, float w, float up, float dn, uint32_t &differ) {
    if (FMT == H1B_KV8_INT8) {
        const uint64_t f[2] = {pack2f(x, y), pack2f(z, w)}, magic = pack2f(kMagic, kMagic);
        uint32_t r[4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float2 a = unpack2(fma2(f[j], pack2f(up, up), magic)), b = unpack2(fma2(f[j], pack2f(dn, dn), magic));
            r[2 * j] = __float_as_uint(a.x);
            r[2 * j + 1] = __float_as_uint(a.y);
            differ |= (r[2 * j] ^ __float_as_uint(b.x)) | (r[2 * j + 1] ^ __float_as_uint(b.y));
        }
        return __byte_perm(__byte_perm(r[0], r[1], 0x0040), __byte_perm(r[2], r[3], 0x0040), 0x5410);
    }
    uint16_t a, b, c, d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(a) : "f"(y * up), "f"(x * up));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(y * dn), "f"(x * dn));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(w * up), "f"(z * up));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(w * dn), "f"(z * dn));
    differ |= (uint32_t)(a ^ b) | (uint32_t)(c ^ d);
    return a | (uint32_t)c << 16;
}
template <int FMT>
__device__ __forceinline__ uint4 kv8_quantise16(const float (&f)[16], float amax) {
    constexpr float TOP = FMT == H1B_KV8_INT8 ? 127.f : 448.f;
    const float by = __fdividef(TOP, amax), up = by * (1.f + 0x1p-21f), dn = by * (1.f - 0x1p-21f);   // (off by 2 ulp at most)
    uint32_t c[4], differ = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = kv8_quantise4<FMT>(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3], up, dn, differ);
    const bool wide = !(amax >= 0x1p-100f && amax <= 0x1p100f);  // where the quotient above is not that exact
    if (differ || wide) {
        const float down = amax > 1e30f ? 0x1p-16f : 1.f, m = amax * down;   // TOP * x stays finite
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {                            // a word at a time: the others are right
            float x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = i == 0 ? f[j] : i == 1 ? f[4 + j] : i == 2 ? f[8 + j] : f[12 + j];
            uint32_t again = 0, r;
            (void)kv8_quantise4<FMT>(x[0], x[1], x[2], x[3], up, dn, again);
            if (!again && !wide) continue;
            float q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] = __fdiv_rn(x[j] * down * TOP, m);
            if (FMT == H1B_KV8_INT8) {
                r = ((uint32_t)__float2int_rn(q[0]) & 255u) | ((uint32_t)__float2int_rn(q[1]) & 255u) << 8 |
                    ((uint32_t)__float2int_rn(q[2]) & 255u) << 16 | (uint32_t)__float2int_rn(q[3]) << 24;
            } else {
                uint16_t a, b;
                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(a) : "f"(q[1]), "f"(q[0]));
                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(q[3]), "f"(q[2]));
                r = a | (uint32_t)b << 16;
            }
            if (i == 0) c[0] = r; else if (i == 1) c[1] = r; else if (i == 2) c[2] = r; else c[3] = r;
        }
    }
    return make_uint4(c[0], c[1], c[2], c[3]);
}

// amax / TOP, rounded once. The product with 1 / TOP, corrected by its remainder, is the correctly rounded quotient (P. Markstein,
// IA-64 and Elementary Functions, 2000; all 1024 mantissas that an amax may have were compared); not where a term is subnormal.
template <int FMT>
__device__ __forceinline__ float kv8_scale(float amax) {
    constexpr float TOP = FMT == H1B_KV8_INT8 ? 127.f : 448.f, BY = 1.f / TOP;
    if (amax < 0x1p-80f) return __fdiv_rn(amax, TOP);
    const float q = amax * BY;
    return fmaf(fmaf(-q, TOP, amax), BY, q);
}

// The largest magnitude; NaN if there is one.
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float r;
    asm("{\n\t.reg .f32 b, c;\n\tabs.f32 b, %2;\n\tabs.f32 c, %3;\n\tmax.NaN.f32 %0, %1, b, c;\n\t}" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

template <int D, int FMT, bool BF16>
__global__ void __launch_bounds__(256) kv8_append_kernel(const Kv8Io io) {
    constexpr int LANES = D / 16, VECS = 32 / LANES;             // lanes per vector, vectors (key or value rows) per warp
    const Kv8Params &P = io.P;
    const int lane = threadIdx.x & 31, sub = lane % LANES;
    const uint32_t unit = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const int r = unit / io.groups;
    if (r >= P.n_rows) return;                                   // (whole warps)
    const int h0 = (int)(unit - (uint32_t)r * io.groups) * io.heads, h1 = min(h0 + io.heads, P.hkv);
    // A lane has the keys (val: the values) of head h, then of the head HEADS further on ...
    constexpr int HEADS = VECS / 2;
    const bool val = (lane / LANES) & 1;
    int h = h0 + lane / (2 * LANES);
    const int64_t hop = (val ? io.v.head_stride : io.k.head_stride) * HEADS;
    const uint16_t *src = static_cast<const uint16_t *>(val ? io.v.data : io.k.data) +
                          (int64_t)r * (val ? io.v.row_stride : io.k.row_stride) +
                          (int64_t)h * (val ? io.v.head_stride : io.k.head_stride) + sub * 8;
    auto load = [&](uint4 (&w)[2]) {
        w[0] = __ldcs(reinterpret_cast<const uint4 *>(src));
        w[1] = __ldcs(reinterpret_cast<const uint4 *>(src + D / 2));
    };
    uint4 next[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (h < h1) load(next);                                      // (nobody's rows lie in the tensors too)
    kv8_check_batch(P, unit, P.n_rows * io.groups, lane);
    Kv8Seq s;
    if (!kv8_seq_of_row(P, r, lane, &s)) return;
    const int64_t at = kv8_place(P, s, r);
    if (at < 0) return;
    const int64_t row = at + (int64_t)h * P.page_tokens, next_row = (int64_t)HEADS * P.page_tokens;
    uint8_t *to = (val ? P.v : P.k) + row * D + sub * 8;
    float *scale = (val ? P.vs : P.ks) + row;
#pragma unroll 1
    for (int hb = h0; hb < h1; hb += HEADS, h += HEADS, to += next_row * D, scale += next_row) {
        const uint32_t w[8] = {next[0].x, next[0].y, next[0].z, next[0].w, next[1].x, next[1].y, next[1].z, next[1].w};
        src += hop;
        if (h + HEADS < h1) load(next);
        float f[16], amax = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 p = pair_to_float2(w[i], BF16);
            f[2 * i] = p.x; f[2 * i + 1] = p.y;
            amax = max_abs(amax, p.x, p.y);
        }
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) amax = max_abs(amax, amax, __shfl_xor_sync(~0u, amax, o));
        const bool odd = !(amax <= 3.402823466e38f);             // the row holds an infinity or a NaN
        uint4 c = make_uint4(0, 0, 0, 0);
        if (!odd && amax > 0.f) c = kv8_quantise16<FMT>(f, amax);
        if (h < h1) {
            *reinterpret_cast<uint2 *>(to) = make_uint2(c.x, c.y);
            *reinterpret_cast<uint2 *>(to + D / 2) = make_uint2(c.z, c.w);
            if (sub == 0) *scale = odd ? __int_as_float(0x7FC00000) : kv8_scale<FMT>(amax);
        }
        __syncwarp();
    }
}

template <int D, int FMT, bool BF16>
__global__ void __launch_bounds__(256) kv8_read_kernel(const Kv8Io io) {
    constexpr int LANES = D / 16, VECS = 32 / LANES;
    const Kv8Params &P = io.P;
    const int lane = threadIdx.x & 31, sub = lane % LANES;
    const uint32_t unit = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const int r = unit / io.groups;
    if (r >= P.n_rows) return;
    const int h0 = (int)(unit - (uint32_t)r * io.groups) * io.heads, h1 = min(h0 + io.heads, P.hkv);
    kv8_check_batch(P, unit, P.n_rows * io.groups, lane);
    Kv8Seq s;
    if (!kv8_seq_of_row(P, r, lane, &s)) return;
    const int64_t at = kv8_place(P, s, r);
    auto load = [&](int x, uint4 &c, float &sc) {
        c = make_uint4(0, 0, 0, 0);
        sc = 0.f;                                                // (a token that is nowhere reads as zeros)
        if (at < 0 || (x >> 1) >= h1) return;
        const int64_t row = at + (int64_t)(x >> 1) * P.page_tokens;
        const uint8_t *from = ((x & 1) ? P.v : P.k) + row * D + sub * 8;
        const uint2 a = __ldcs(reinterpret_cast<const uint2 *>(from)), b = __ldcs(reinterpret_cast<const uint2 *>(from + D / 2));
        c = make_uint4(a.x, a.y, b.x, b.y);
        sc = ((x & 1) ? P.vs : P.ks)[row];
    };
    constexpr int AHEAD = 4;                                     // loads under way
    uint4 c[AHEAD];
    float sc[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load(h0 * 2 + i * VECS + lane / LANES, c[i], sc[i]);
#pragma unroll 1
    for (int x0 = h0 * 2; x0 < h1 * 2; x0 += AHEAD * VECS)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int x = x0 + i * VECS + lane / LANES, h = x >> 1;
            const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
            const float by = sc[i];
            load(x + AHEAD * VECS, c[i], sc[i]);
            const h1b_kv8_rows &dst = (x & 1) ? io.v : io.k;
            if (h >= h1 || !dst.data) continue;
            uint32_t out[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t a, b;
                kv8_codes4<FMT>(w[j], a, b);
                const float2 p = half2_bits_to_float2(a), q = half2_bits_to_float2(b);
                out[2 * j] = float2_to_pair(p.x * by, p.y * by, BF16);
                out[2 * j + 1] = float2_to_pair(q.x * by, q.y * by, BF16);
            }
            uint4 *to = reinterpret_cast<uint4 *>(static_cast<uint16_t *>(dst.data) + (int64_t)r * dst.row_stride +
                                                  (int64_t)h * dst.head_stride + sub * 8);
            to[0] = make_uint4(out[0], out[1], out[2], out[3]);
            to[D / 16] = make_uint4(out[4], out[5], out[6], out[7]);
        }
}

template <bool APPEND>
cudaError_t launch_io(const Kv8Params &P, const h1b_kv8_rows &k, const h1b_kv8_rows &v, int d, int fmt, int bf16,
                      cudaStream_t st) {
    Kv8Io io;
    io.P = P; io.k = k; io.v = v;
    // few rows: as few heads a warp as it has lanes for (latency); many: up to sixteen (8 sequences of
    // 2-4k tokens of 32 heads read back: 97 us, 102 with up to eight, 101 with 32; appended the difference is 1 %)
    io.heads = 32 / (d / 16) / 2;
    while (io.heads < 16 && (int64_t)P.n_rows * ((P.hkv + io.heads - 1) / io.heads) > 148 * 64) io.heads *= 2;
    io.groups = (P.hkv + io.heads - 1) / io.heads;
    const int64_t warps = (int64_t)P.n_rows * io.groups;
    // (smaller blocks even append's warps out, some of which divide: 8192 tokens 41.6 us, 42.4 with eight warps; read 100 and 99)
    const int warps_per_block = warps < 148 * 8 ? 1 : APPEND ? 4 : 8;
    const unsigned grid = (unsigned)((warps + warps_per_block - 1) / warps_per_block);
#define H1B_KV8_IO(D, F, B)                                                                                            \
    kv8_launch(APPEND ? kv8_append_kernel<D, F, B> : kv8_read_kernel<D, F, B>, dim3(grid), warps_per_block * 32, 0, st, io)
#define H1B_KV8_IO2(D, F) (bf16 ? H1B_KV8_IO(D, F, true) : H1B_KV8_IO(D, F, false))
    if (d == 128) return fmt == H1B_KV8_INT8 ? H1B_KV8_IO2(128, H1B_KV8_INT8) : H1B_KV8_IO2(128, H1B_KV8_E4M3);
    return fmt == H1B_KV8_INT8 ? H1B_KV8_IO2(64, H1B_KV8_INT8) : H1B_KV8_IO2(64, H1B_KV8_E4M3);
#undef H1B_KV8_IO2
#undef H1B_KV8_IO
}

// ------------------------------------------------------------------------------------------------------------------
// Attention, few rows. A block of four warps takes one tile (up to 8 * NB (row, head of the group) pairs of a sequence
// that share a KV head) and one part of the tokens that the tile sees; the warps take its blocks of 16 tokens in turn,
// each through a ring of its own in shared memory that 16-byte asynchronous copies fill, so nothing in the loop is
// block-wide.
//   S^T = K Q^T    (16 tokens x 8 NB rows)   mma m16n8k16, A = the codes as exact fp16 numbers, B = the query rows
//   w   = 2^(S ks - m) vs / sigma            softmax weights, online; the value's scale goes into the weight
//   O^T += V^T w   (d channels x 8 NB rows)  A = the codes again, B = the weights in fp16
// m and sigma (a power of two) are references that follow the row's largest score and the largest value scale lazily:
// the accumulators are only rescaled when a score exceeds m by 2 (in log2) or a scale exceeds 4 sigma, so the weights,
// carried times 2^11, stay below 2^15 and keep fp16's full precision down to 2^-25 of the largest one. One rounding to fp16
// (2^-12 on average) vanishes beside that of a bf16 result, but would add as much again to an fp16 result's: there (SPLIT)
// a second product carries what the rounding left, w = hi + lo to 2^-22, at no cost in time where the loads are the bound.
// Bound by memory where there is enough of it: 16 sequences of 4-8k tokens, 32 heads of 128 (int8, fp16): 150 us = 5.7 TB/s,
// 87 % of the copy bandwidth, the arithmetic pipe that unpacks codes busy 53 % of the time; 8 of 32k, 32 / 8 heads (e4m3,
// bf16): 97 us, 86 %. tcgen05 has no place here: its smallest tile is 64 rows, and codes would pass shared memory twice.
// ------------------------------------------------------------------------------------------------------------------
constexpr int kRowsStages = 3;
constexpr int kRowsWarps = 4;
constexpr float kLazy = 2.f;
constexpr float kWeightUnit = 2048.f;
constexpr float kPartShare = 0x1p-8f;                            // parts (256 at most) join with weights up to this: large results do not overflow

__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// Block p of this block's cluster: the number at the place where this block has `addr`.
__device__ __forceinline__ uint32_t cluster_at(uint32_t addr, int p) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(p));
    return r;
}
__device__ __forceinline__ float cluster_load(uint32_t addr, int p) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_at(addr, p)) : "memory");
    return v;
}
__device__ __forceinline__ float2 cluster_load2(uint32_t addr, int p) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(cluster_at(addr, p)) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int D>
__host__ __device__ constexpr int rows_stage_bytes() { return 32 * D + 128; }
template <int D, int NB>
__host__ __device__ constexpr int rows_smem_bytes() {
    const int ring = kRowsWarps * kRowsStages * rows_stage_bytes<D>(), merge = kRowsWarps * 8 * NB * (D + 2) * 4 + 8 * NB * (D + 1) * 4;
    return ring > merge ? ring : merge;
}

template <int D, int FMT, int NB, bool SPLIT>
__global__ void __launch_bounds__(kRowsWarps * 32, NB == 1 ? 4 : 2) kv8_rows_kernel(const Kv8Params P, const Kv8Attn A) {
    extern __shared__ __align__(128) unsigned char smem[];
    constexpr int R = 8 * NB, STAGE = rows_stage_bytes<D>();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int gi = lane >> 2, tj = lane & 3;                     // row of A / column of B, and the pair of k, of this lane
    const int kvh = blockIdx.y, split = blockIdx.z;
    const uint32_t ring = smem_addr(smem) + warp * kRowsStages * STAGE;

    // Blocks x * tiles .. + tiles - 1 belong to sequence x, one for each of its tiles; if it has more than the host said, they
    // take those too, undivided.
    const Kv8Seq s = kv8_seq(P, blockIdx.x / A.tiles);
    if (s.n * A.group < A.min_pairs || s.n * A.group > A.max_pairs) return;
    const int first_tile = blockIdx.x % A.tiles;
    for (int tile = first_tile; tile * R < s.n * A.group; tile += A.tiles) {
        const bool extra = tile != first_tile;
        const int splits = extra ? 1 : A.splits;
        const int pair0 = tile * R, pairs = min(R, s.n * A.group - pair0);
        const int tok0 = pair0 / A.group, tok1 = (pair0 + pairs - 1) / A.group;
        const int pos0 = s.kv - s.n + tok0, pos1 = s.kv - s.n + tok1;
        if (pos0 < 0 && split == 0) kv8_report(P, H1B_ERR_INVALID_ARG);
        const Kv8Span span = kv8_span(P, A, pos0, pos1);
        // the tile's blocks in parts of `per`, a multiple of four (one per warp) and at least two per warp
        const int per = extra ? span.count + 1 : max((((span.count + splits - 1) / splits) + 3) & ~3, 2 * kRowsWarps);
        const int parts = max(1, (span.count + per - 1) / per);
        if (split >= parts && (parts == 1 || !A.cluster)) continue;
        const int j0 = min(split * per, span.count), j1 = min(j0 + per, span.count);
        const int n_mine = j1 - j0 > warp ? (j1 - j0 - warp + kRowsWarps - 1) / kRowsWarps : 0;

        // ---- the copies: block i of this warp into stage i % 3; where the blocks lie is looked up 32 blocks at a time ----
        const int32_t *table = P.table + (int64_t)s.b * P.table_width;
        const uint8_t *kp = P.k + lane * 16, *vp = P.v + lane * 16;
        const float *sp = (lane < 4 ? P.ks : P.vs) + (lane & 3) * 4;
        int at_lane = -1;                                        // block i + lane of the warp: its number in the pool, or -1
        auto issue = [&](int i, int stage) -> int {              // -> the block's first token, or -1: nobody sees it
            int t = -1;
            if (i < n_mine) {
                if ((i & 31) == 0) {
                    at_lane = -1;
                    if (i + lane < n_mine) {
                        const int blk = span.token(j0 + warp + (i + lane) * kRowsWarps) / kKv8Block, col = kv8_page_of(P, blk);
                        const int page = table[col], per_page = P.page_tokens / kKv8Block;
                        if (page >= 0 && page < P.n_pages) at_lane = (page * P.hkv + kvh) * per_page + blk - col * per_page;
                        else kv8_report(P, H1B_ERR_BOUNDS);
                    }
                }
                const int at = __shfl_sync(~0u, at_lane, i & 31);
                if (at >= 0) {
                    t = span.token(j0 + warp + i * kRowsWarps);
                    const uint32_t st = ring + stage * STAGE;
                    const uint8_t *ks = kp + (int64_t)at * (16 * D), *vs = vp + (int64_t)at * (16 * D);
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        const int x = lane + 32 * c, r = x / (D / 16), ch = x % (D / 16);
                        const uint32_t kd = D == 128 ? r * 128 + ((ch ^ ((r & 1) << 2)) << 4) : x << 4;
                        const uint32_t vd = D == 128 ? r * 128 + ((ch ^ (r & 7)) << 4)
                                                     : (r >> 1) * 128 + (((((r & 1) << 2) | ch) ^ (((r >> 1) & 3) << 1)) << 4);
                        cp_async_16(st + kd, ks + c * 512, 16);
                        cp_async_16(st + 16 * D + vd, vs + c * 512, 16);
                    }
                    if (lane < 8) cp_async_16(st + 32 * D + lane * 16, sp + (int64_t)at * kKv8Block, 16);
                }
            }
            cp_async_commit();
            return t;
        };
        int t_now = issue(0, 0), t_next = issue(1, 1);

        // ---- the query rows, as B operands: lane (n = gi, k pair tj) holds channels 16 (tj + 4 c) .. + 15 of row gi ----
        uint32_t qf[NB][D / 16][2];
        float qs[NB][2];                                         // what turns a dot product of codes into a score, rows 2 tj, + 1
        int pos[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int x = nb * 8 + gi, tok = (pair0 + x) / A.group, head = kvh * A.group + (pair0 + x) % A.group;
            const bool live = x < pairs;
            const uint16_t *qp = static_cast<const uint16_t *>(A.q) + (int64_t)(s.start + tok) * A.q_rs + (int64_t)head * A.q_hs;
            float2 f[D / 16][2];
            float amax = 0.f;
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                uint4 u[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
                if (live) {
                    u[0] = *reinterpret_cast<const uint4 *>(qp + 16 * (tj + 4 * c));
                    u[1] = *reinterpret_cast<const uint4 *>(qp + 16 * (tj + 4 * c) + 8);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 &uu = u[i >> 1];
                    f[c * 4 + i][0] = pair_to_float2((i & 1) ? uu.z : uu.x, A.bf16);
                    f[c * 4 + i][1] = pair_to_float2((i & 1) ? uu.w : uu.y, A.bf16);
#pragma unroll
                    for (int y = 0; y < 2; ++y)
                        amax = fmaxf(amax, fmaxf(fabsf(f[c * 4 + i][y].x), fabsf(f[c * 4 + i][y].y)));
                }
            }
            amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
            const int e = kv8_row_exponent(amax);
            const float up = A.scale_log2 < 0.f ? -pow2i(-e) : pow2i(-e);   // (so that qs >= 0)
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int y = 0; y < 2; ++y) qf[nb][i][y] = pack_f16x2(f[i][y].x * up, f[i][y].y * up);
            const float unit = fabsf(A.scale_log2) * pow2i(e);
            const int t0 = s.kv - s.n + tok;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                qs[nb][y] = __shfl_sync(~0u, unit, (2 * tj + y) * 4);
                pos[nb][y] = __shfl_sync(~0u, t0, (2 * tj + y) * 4);
            }
        }

        float o[NB][D / 16][4], nm[NB][2], l[NB][2];             // nm: -m
        float sigma = 0.f, wscale = 0.f;                         // wscale = kWeightUnit / sigma
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[nb][i][0] = o[nb][i][1] = o[nb][i][2] = o[nb][i][3] = 0.f;
            nm[nb][0] = nm[nb][1] = INFINITY;
            l[nb][0] = l[nb][1] = 0.f;
        }

        int stage = 0;
        for (int i = 0; i < n_mine; ++i) {
            cp_async_wait_group<kRowsStages - 2>();
            __syncwarp();                                        // every lane's copies of block i are there; block i - 1 is read
            const int t = t_now;
            const unsigned char *st = smem + (warp * kRowsStages + stage) * STAGE;
            t_now = t_next;
            t_next = issue(i + 2, stage == 0 ? 2 : stage - 1);
            stage = stage == 2 ? 0 : stage + 1;
            if (t < 0) continue;
            // ---- scores ----
            float c[NB][4];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) c[nb][0] = c[nb][1] = c[nb][2] = c[nb][3] = 0.f;
#pragma unroll
            for (int h = 0; h < D / 64; ++h) {
                const int ch = D == 128 ? (tj + 4 * h) ^ ((gi & 1) << 2) : tj;
                const uint4 ka = *reinterpret_cast<const uint4 *>(st + gi * D + ch * 16);
                const uint4 kb = *reinterpret_cast<const uint4 *>(st + (gi + 8) * D + ch * 16);
                const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    uint32_t a0, a1, a2, a3;
                    kv8_codes4<FMT>(wa[x], a0, a2);
                    kv8_codes4<FMT>(wb[x], a1, a3);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        mma_f16_16816(c[nb], a0, a1, a2, a3, qf[nb][h * 4 + x][0], qf[nb][h * 4 + x][1]);
                }
            }
            const float *sc = reinterpret_cast<const float *>(st + 32 * D);
            const float ks0 = sc[gi], ks1 = sc[gi + 8];
            float vs0 = sc[16 + gi], vs1 = sc[16 + gi + 8];
            // all rows of the tile see all 16 tokens, or each pair is looked at
            const bool whole = t + 15 <= pos0 && (!A.window || t > pos1 - A.window || t + 15 < A.sinks);
            uint32_t hidden = 0;                                 // bit 4 nb + y: token gi (+ 8 for y >= 2) is not seen by row 2 tj + y % 2
            float over = -INFINITY;                              // how far a score lies above its row's reference
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int y = 0; y < 4; ++y) c[nb][y] *= (y & 2) ? ks1 : ks0;
            if (!whole) {
                const int t0 = t + gi, t1 = t0 + 8;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const int tt = (y & 2) ? t1 : t0, p = pos[nb][y & 1];
                        if (tt <= p && (!A.window || tt > p - A.window || tt < A.sinks)) continue;
                        hidden |= 1u << (4 * nb + y);
                        c[nb][y] = -INFINITY;
                    }
                // scales of tokens that no row sees say nothing
                if (!(t0 <= span.hi && (t0 >= span.lo || t0 < span.sinks))) vs0 = 0.f;
                if (!(t1 <= span.hi && (t1 >= span.lo || t1 < span.sinks))) vs1 = 0.f;
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int y = 0; y < 2; ++y) over = fmaxf(over, fmaf(fmaxf(c[nb][y], c[nb][y + 2]), qs[nb][y], nm[nb][y]));
            if (__any_sync(~0u, over > kLazy || fmaxf(vs0, vs1) > 4.f * sigma)) {
                float mx = fmaxf(vs0 <= 3.402823466e38f ? vs0 : 0.f, vs1 <= 3.402823466e38f ? vs1 : 0.f);
#pragma unroll
                for (int x = 1; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, x));
                float turn = 1.f;                                // old sigma / new sigma
                if (mx > 4.f * sigma) {
                    const int e = clampi((int)(__float_as_uint(mx) >> 23) - 126, -115, 126);   // 2^e > mx
                    const float next = pow2i(e);
                    turn = sigma / next;
                    sigma = next;
                    wscale = kWeightUnit * pow2i(-e);
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        float top = fmaxf(c[nb][y], c[nb][y + 2]);
                        top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
                        top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
                        top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
                        if (top != -INFINITY) top *= qs[nb][y];
                        const float m = -nm[nb][y];
                        const bool up = top > m;
                        const float f = up ? ex2_approx(m - top) : 1.f;   // (from -inf: 0)
                        if (up) nm[nb][y] = -top;
                        l[nb][y] *= f;
#pragma unroll
                        for (int x = 0; x < D / 16; ++x) { o[nb][x][y] *= f * turn; o[nb][x][y + 2] *= f * turn; }
                    }
            }
            // ---- weights: fp16, rounded once; a token that a row does not see gets weight zero whatever its scale holds ----
            const float g0 = vs0 * wscale, g1 = vs1 * wscale;
            uint32_t b[NB][2], b_lo[NB][2];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float p[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) p[y] = ex2_approx(fmaf(c[nb][y], qs[nb][y & 1], nm[nb][y & 1]));
                if (!whole) {
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if (hidden >> (4 * nb + y) & 1) p[y] = 0.f;
                }
                l[nb][0] += p[0] + p[2];
                l[nb][1] += p[1] + p[3];
#pragma unroll
                for (int y = 0; y < 4; ++y) p[y] *= (y & 2) ? g1 : g0;
                if (!whole) {
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if (hidden >> (4 * nb + y) & 1) p[y] = 0.f;
                }
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t hi = pack_f16x2(p[2 * y], p[2 * y + 1]);
                    b[nb][y] = movmatrix_trans(hi);
                    if (SPLIT) {
                        const float2 back = half2_bits_to_float2(hi);
                        b_lo[nb][y] = movmatrix_trans(pack_f16x2(p[2 * y] - back.x, p[2 * y + 1] - back.y));
                    }
                }
            }
            // ---- values: lane (m = gi, k pair tj) holds channels (D / 8) gi .. of tokens 2 tj, 2 tj + 1, + 8, + 9 ----
            const unsigned char *vst = st + 16 * D;
            uint32_t w[4][D / 32];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int r = 2 * tj + (y & 1) + (y & 2) * 4;
                if (D == 128) {
                    const uint4 u = *reinterpret_cast<const uint4 *>(vst + r * 128 + ((gi ^ (r & 7)) << 4));
                    w[y][0] = u.x; w[y][1] = u.y; w[y][D / 32 - 2] = u.z; w[y][D / 32 - 1] = u.w;
                } else {
                    const uint2 u = *reinterpret_cast<const uint2 *>(
                        vst + (r >> 1) * 128 + (((((r & 1) << 2) | (gi >> 1)) ^ (((r >> 1) & 3) << 1)) << 4) + (gi & 1) * 8);
                    w[y][0] = u.x; w[y][1] = u.y;
                }
            }
            if (!whole) {                                        // codes that no row sees may be NaN patterns: zero times NaN is none
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int tt = t + 2 * tj + (y & 1) + (y & 2) * 4;
                    if (tt <= span.hi && (tt >= span.lo || tt < span.sinks)) continue;
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) w[y][x] = 0;
                }
            }
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                uint32_t lo[4], hi[4];
                kv8_codes4x2<FMT>(w[0][x], w[1][x], lo);
                kv8_codes4x2<FMT>(w[2][x], w[3][x], hi);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    mma_f16_16816(o[nb][2 * x], lo[0], lo[1], hi[0], hi[1], b[nb][0], b[nb][1]);
                    mma_f16_16816(o[nb][2 * x + 1], lo[2], lo[3], hi[2], hi[3], b[nb][0], b[nb][1]);
                    if (SPLIT) {
                        mma_f16_16816(o[nb][2 * x], lo[0], lo[1], hi[0], hi[1], b_lo[nb][0], b_lo[nb][1]);
                        mma_f16_16816(o[nb][2 * x + 1], lo[2], lo[3], hi[2], hi[3], b_lo[nb][0], b_lo[nb][1]);
                    }
                }
            }
        }
        cp_async_wait_group<0>();
        launch_dependents();

        // ---- the four warps' results meet in shared memory: [warp][row][d], then m and l [warp][row] ----
        __syncthreads();
        float *acc = reinterpret_cast<float *>(smem), *ml = acc + kRowsWarps * R * D;
        float *res = ml + kRowsWarps * R * 2, *res_lse = res + R * D;   // this part's result, for the cluster
        const float unit = sigma * (1.f / kWeightUnit);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int row = nb * 8 + 2 * tj + y;
                float sum = l[nb][y];
                sum += __shfl_xor_sync(~0u, sum, 4);
                sum += __shfl_xor_sync(~0u, sum, 8);
                sum += __shfl_xor_sync(~0u, sum, 16);
                // (divided by the warp's own sum first: a sum over many tokens of large numbers is beyond fp32)
                const float inv = sum > 0.f ? 1.f / sum : sum;
                float *a = acc + (warp * R + row) * D + gi * (D / 8);
#pragma unroll
                for (int x = 0; x < D / 16; ++x) {
                    a[2 * x] = o[nb][x][y] * inv * unit;
                    a[2 * x + 1] = o[nb][x][y + 2] * inv * unit;
                }
                // (a row whose every score is NaN has no maximum, and is not an empty row)
                if (gi == 0) { ml[(warp * R + row) * 2] = sum != sum ? sum : -nm[nb][y]; ml[(warp * R + row) * 2 + 1] = sum; }
            }
        __syncthreads();
        constexpr int PER = D / 2;                               // channel pairs of a row
        for (int x = threadIdx.x; x < pairs * PER; x += kRowsWarps * 32) {
            const int row = x / PER, ch = (x % PER) * 2;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kRowsWarps; ++w) {
                const float mw = ml[(w * R + row) * 2];
                top = (mw > top || mw != mw) ? mw : top;
            }
            float f[kRowsWarps], sum = 0.f, a0 = 0.f, a1 = 0.f;
#pragma unroll
            for (int w = 0; w < kRowsWarps; ++w) {
                const float mw = ml[(w * R + row) * 2];
                f[w] = mw == -INFINITY ? 0.f : ex2_approx(mw - top) * ml[(w * R + row) * 2 + 1];
                sum += f[w];
            }
            const bool empty = top == -INFINITY;
            const float inv = empty ? 0.f : 1.f / sum;
#pragma unroll
            for (int w = 0; w < kRowsWarps; ++w) {
                a0 += f[w] * inv * acc[(w * R + row) * D + ch];
                a1 += f[w] * inv * acc[(w * R + row) * D + ch + 1];
            }
            const int tok = (pair0 + row) / A.group, head = kvh * A.group + (pair0 + row) % A.group;
            const float lse2 = empty ? -INFINITY : top + log2f(sum);
            if (parts == 1) {
                *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(A.out) + (int64_t)(s.start + tok) * A.o_rs +
                                              (int64_t)head * A.o_hs + ch) = float2_to_pair(a0, a1, A.bf16);
                if (A.lse && ch == 0) A.lse[(int64_t)(s.start + tok) * A.hq + head] = lse2 * kLn2;
            } else if (A.cluster) {
                *reinterpret_cast<float2 *>(res + row * D + ch) = make_float2(a0, a1);
                if (ch == 0) res_lse[row] = lse2;
            } else {
                const int64_t part = (((int64_t)blockIdx.x * P.hkv + kvh) * R + row) * A.splits + split;
                *reinterpret_cast<float2 *>(A.part_acc + part * D + ch) = make_float2(a0, a1);
                if (ch == 0) A.part_lse[part] = lse2;
            }
        }
        if (A.cluster && parts > 1) {
            // The parts of a tile are a cluster: they join in each other's shared memory, every block a share of the numbers.
            // (All blocks of a cluster come through here for the same tiles.)
            cluster_sync();
            const uint32_t at = smem_addr(res), at_lse = smem_addr(res_lse);
            for (int x = split * kRowsWarps * 32 + threadIdx.x; x < pairs * PER; x += A.splits * kRowsWarps * 32) {
                const int row = x / PER, ch = (x % PER) * 2;
                float top = -INFINITY, sum = 0.f, a0 = 0.f, a1 = 0.f;
                bool nan = false;
                for (int p = 0; p < parts; ++p) {
                    const float y = cluster_load(at_lse + row * 4, p);
                    top = fmaxf(top, y);
                    nan |= y != y;
                }
                for (int p = 0; p < parts; ++p) {
                    const float y = cluster_load(at_lse + row * 4, p), f = y == -INFINITY ? 0.f : kPartShare * ex2_approx(y - top);
                    const float2 v = cluster_load2(at + (row * D + ch) * 4, p);
                    sum += f;
                    a0 += f * v.x;
                    a1 += f * v.y;
                }
                const bool empty = top == -INFINITY && !nan;
                const int tok = (pair0 + row) / A.group, head = kvh * A.group + (pair0 + row) % A.group;
                *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(A.out) + (int64_t)(s.start + tok) * A.o_rs +
                                              (int64_t)head * A.o_hs + ch) = empty ? 0u : float2_to_pair(a0 / sum, a1 / sum, A.bf16);
                if (A.lse && ch == 0)
                    A.lse[(int64_t)(s.start + tok) * A.hq + head] = empty ? -INFINITY : (top + log2f(sum * (1.f / kPartShare))) * kLn2;
            }
            cluster_sync();                                      // nobody's results are overwritten or gone while another reads them
        }
        __syncthreads();                                         // the ring is free for the next tile's copies
    }
}

// Joins the parts of the rows whose tokens were dealt into more than one: out = sum_s 2^(lse_s - lse) out_s. Up to eight
// parts: a warp for two rows of a tile. WIDE, more parts (then there are few rows): a block for each row, whose four warps
// take the parts in turn (one sequence of 16k tokens, 64 parts: 33 -> 19 us; but 13 us more for 8192 rows of two parts).
// DIRECT: the blocks of the few-rows kernel (a number of tiles for each sequence), else those of the tiles kernel.
template <int D, bool DIRECT, bool WIDE>
__global__ void __launch_bounds__(128) kv8_join_kernel(const Kv8Params P, const Kv8Attn A, const int R, const int unit_blocks,
                                                       const int min_blocks) {
    __shared__ float sums[4][D + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int idx = blockIdx.x / P.hkv, kvh = blockIdx.x % P.hkv;
    grid_dependency_wait();                                      // launched while the attention kernel's last blocks run
    Kv8Seq s;
    int tile;
    if (DIRECT) {
        s = kv8_seq(P, idx / A.tiles);
        tile = idx % A.tiles;
        if (s.n * A.group < A.min_pairs || s.n * A.group > A.max_pairs || tile * R >= s.n * A.group) return;
    } else if (!kv8_find_tile(P, A, idx, R, lane, &s, &tile)) {
        return;
    }
    // the same split of the same tile as the attention kernel's
    const int pair0 = tile * R, pairs = min(R, s.n * A.group - pair0);
    const Kv8Span span = kv8_span(P, A, s.kv - s.n + pair0 / A.group, s.kv - s.n + (pair0 + pairs - 1) / A.group);
    const int per = max(((span.count + A.splits - 1) / A.splits + unit_blocks - 1) / unit_blocks * unit_blocks, min_blocks);
    const int parts = max(1, (span.count + per - 1) / per);
    if (parts == 1) return;
    const int row0 = WIDE ? blockIdx.y : blockIdx.y * 8 + warp, row1 = WIDE ? row0 + 1 : blockIdx.y * 8 + 8;
    for (int row = row0; row < min(pairs, row1); row += 4) {
        const int64_t part = (((int64_t)idx * P.hkv + kvh) * R + row) * A.splits;
        const float *pl = A.part_lse + part, *pa = A.part_acc + part * D;
        float top = -INFINITY;
        bool nan = false;
        for (int i = lane; i < parts; i += 32) { top = fmaxf(top, pl[i]); nan |= pl[i] != pl[i]; }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
        nan = __any_sync(~0u, nan);
        float sum = 0.f, a[D / 32];
#pragma unroll
        for (int x = 0; x < D / 32; ++x) a[x] = 0.f;
#pragma unroll 4
        for (int i = WIDE ? warp : 0; i < parts; i += WIDE ? 4 : 1) {
            const float f = pl[i] == -INFINITY ? 0.f : kPartShare * ex2_approx(pl[i] - top);
            sum += f;
#pragma unroll
            for (int x = 0; x < D / 64; ++x) {
                const float2 v = *reinterpret_cast<const float2 *>(pa + (int64_t)i * D + x * 64 + lane * 2);
                a[2 * x] += f * v.x;
                a[2 * x + 1] += f * v.y;
            }
        }
        if (WIDE) {
#pragma unroll
            for (int x = 0; x < D / 32; ++x) sums[warp][(x >> 1) * 64 + lane * 2 + (x & 1)] = a[x];
            if (lane == 0) sums[warp][D] = sum;
            __syncthreads();
            if (warp != 0) return;
            sum = sums[0][D] + sums[1][D] + sums[2][D] + sums[3][D];
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                const int ch = (x >> 1) * 64 + lane * 2 + (x & 1);
                a[x] = sums[0][ch] + sums[1][ch] + sums[2][ch] + sums[3][ch];
            }
        }
        const bool empty = top == -INFINITY && !nan;
        const int tok = (pair0 + row) / A.group, head = kvh * A.group + (pair0 + row) % A.group;
        uint16_t *op = static_cast<uint16_t *>(A.out) + (int64_t)(s.start + tok) * A.o_rs + (int64_t)head * A.o_hs;
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
            *reinterpret_cast<uint32_t *>(op + x * 64 + lane * 2) =
                empty ? 0u : float2_to_pair(a[2 * x] / sum, a[2 * x + 1] / sum, A.bf16);
        if (A.lse && lane == 0)
            A.lse[(int64_t)(s.start + tok) * A.hq + head] = empty ? -INFINITY : (top + log2f(sum * (1.f / kPartShare))) * kLn2;
    }
}

template <int D, int FMT, int NB, bool SPLIT>
cudaError_t launch_rows_of(const Kv8Params &P, const Kv8Attn &A, cudaStream_t st) {
    constexpr int bytes = rows_smem_bytes<D, NB>();
    static Kv8Once once;
    const cudaError_t e = once.shared_memory(reinterpret_cast<const void *>(kv8_rows_kernel<D, FMT, NB, SPLIT>), bytes);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 1;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = (unsigned)A.splits;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)P.n_seqs * (unsigned)A.tiles, (unsigned)P.hkv, (unsigned)A.splits);
    cfg.blockDim = dim3(kRowsWarps * 32);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = A.cluster ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kv8_rows_kernel<D, FMT, NB, SPLIT>, P, A);
}

}  // namespace

cudaError_t launch_kv8_append(const Kv8Params &P, const h1b_kv8_rows &k, const h1b_kv8_rows &v, int d, int fmt, int bf16,
                              cudaStream_t st) {
    return launch_io<true>(P, k, v, d, fmt, bf16, st);
}
cudaError_t launch_kv8_read(const Kv8Params &P, const h1b_kv8_rows &k, const h1b_kv8_rows &v, int d, int fmt, int bf16,
                            cudaStream_t st) {
    return launch_io<false>(P, k, v, d, fmt, bf16, st);
}

cudaError_t launch_kv8_rows(const Kv8Params &P, const Kv8Attn &A, int d, int fmt, int rows_per_tile, cudaStream_t st) {
    cudaError_t e;
#define H1B_KV8_ROWS(D, F)                                                                                        \
    e = rows_per_tile == 8 ? (A.bf16 ? launch_rows_of<D, F, 1, false> : launch_rows_of<D, F, 1, true>)(P, A, st) \
                           : (A.bf16 ? launch_rows_of<D, F, 2, false> : launch_rows_of<D, F, 2, true>)(P, A, st)
    if (d == 128 && fmt == H1B_KV8_INT8) { H1B_KV8_ROWS(128, H1B_KV8_INT8); }
    else if (d == 128) { H1B_KV8_ROWS(128, H1B_KV8_E4M3); }
    else if (fmt == H1B_KV8_INT8) { H1B_KV8_ROWS(64, H1B_KV8_INT8); }
    else { H1B_KV8_ROWS(64, H1B_KV8_E4M3); }
#undef H1B_KV8_ROWS
    if (e != cudaSuccess || A.splits == 1 || A.cluster) return e;
    return launch_kv8_join(P, A, d, rows_per_tile, kRowsWarps, 2 * kRowsWarps, st);
}

cudaError_t launch_kv8_join(const Kv8Params &P, const Kv8Attn &A, int d, int rows_per_tile, int unit_blocks, int min_blocks,
                            cudaStream_t st) {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    const bool direct = rows_per_tile <= 16, wide = direct && A.splits > 8;
    cfg.gridDim = dim3((unsigned)A.tiles * (direct ? (unsigned)P.n_seqs : 1u) * (unsigned)P.hkv, (unsigned)(wide ? rows_per_tile : rows_per_tile / 8));
    cfg.blockDim = dim3(128);
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    auto pick = [&](auto head_dim) {
        constexpr int D = decltype(head_dim)::value;
        return !direct ? kv8_join_kernel<D, false, false> : wide ? kv8_join_kernel<D, true, true> : kv8_join_kernel<D, true, false>;
    };
    return cudaLaunchKernelEx(&cfg, d == 128 ? pick(std::integral_constant<int, 128>()) : pick(std::integral_constant<int, 64>()),
                              P, A, rows_per_tile, unit_blocks, min_blocks);
}

}  // namespace h1b
