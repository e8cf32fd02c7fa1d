// 8-bit pages: attention for many rows per sequence (prompts and chunks of them) on the 5th-generation tensor cores.
//
// One block of 13 warps takes 256 (row, head of the group) pairs of a sequence that share a KV head, as two tiles of 128
// pairs, and one part of the tokens they see, 128 tokens at a time (eight blocks of 16, whichever blocks the span lists:
// sinks and window need not be neighbours). The roles hand each other operands through mbarriers; nothing in the loop is
// block-wide:
//   warps 8-11   convert: codes come from the pages in 16-byte loads, one tile ahead in registers, become exact fp16
//                numbers ONCE for all 256 pairs and go to shared memory as the matrix operands of keys and values (two
//                of each, 128-byte swizzle; keys K-major, values with the channels contiguous, so nothing is transposed);
//   warp 12      issues every contraction: S = Q K^T into tensor memory, O += P V with P read from tensor memory;
//   warps 0-3    softmax of tile A, warps 4-7 of tile B, one pair (row of S) per thread: scores S * ks * qs, the row's
//                reference, weights w = 2^(score - m) * vs / sigma in fp16, written over the scores they came from.
// While one tile's softmax runs the tensor cores work for the other tile. m and sigma follow lazily (as in the kernel for
// few rows): O is rescaled only when a score exceeds m by 4 (in log2) or a value scale exceeds 4 sigma; weights are
// carried times 2^9. For fp16 results (SPLIT) a second contraction adds what rounding the weights left over.
// Every wait is bounded; a role that gives up records the time-out and leaves, and the block releases its tensor memory.
#include "h1b_kv8.cuh"

namespace h1b {

namespace {

constexpr int kTlRows = 128, kTlKeys = 128;
constexpr int kTlThreads = 13 * 32;
constexpr unsigned long long kTlWaitNs = 2000000000ull;
constexpr float kTlLazy = 4.f, kTlWeightUnit = 512.f;
constexpr int kTlHidden = 1 << 30;                             // "first token" of a block that nobody sees: beyond every position
constexpr int kTlScaleStages = 4;

template <int D>
struct TlSmem {
    static constexpr int kQ1 = kTlRows * D * 2, kKV1 = kTlKeys * D * 2;
    static constexpr int kQ = 0, kK = 2 * kQ1, kV = kK + 2 * kKV1, kScales = kV + 2 * kKV1;
    // per scale stage: ks [128], vs' [128], blocks' first tokens [8], {first token if all 128 are in a row, else -1; turn}
    static constexpr int kStage = 1024 + 64;
    static constexpr int kBars = kScales + kTlScaleStages * kStage;
    static constexpr int kTotal = kBars + 256 + 1024;            // + slack to align the operands to 1024 bytes
};
enum { kBarQ = 0, kBarKFull = 1, kBarKFree = 3, kBarVFull = 5, kBarVFree = 7, kBarScales = 9, kBarS = 13, kBarP = 15, kBarO = 17,
       kBarCount = 18 };

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

// An operand with the channels contiguous (MN-major): rows of 128 bytes (64 channels) per token, 128-byte swizzle, eight
// tokens 1024 bytes apart, the next 64 channels 16384 bytes on.
__device__ __forceinline__ uint64_t umma_desc_mn_sw128(uint32_t addr) {
    uint64_t d = 0;
    d |= (uint64_t)((addr >> 4) & 0x3FFFu);
    d |= (uint64_t)(16384 >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
__device__ __forceinline__ void tmem_st_16cols_issue(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) {
    return __all_sync(~0u, mbar_wait_bounded(bar, parity, kTlWaitNs));
}

// Where the weights of contraction step ks (16 tokens) lie within the tile's 128 columns: 32 columns of scores become 16
// columns of weights (two to a column) and 16 of their remainders.
__device__ __forceinline__ uint32_t weight_column(int ks) { return (ks >> 1) * 32 + (ks & 1) * 8; }

template <int D, int FMT, bool SPLIT>
__global__ void __launch_bounds__(kTlThreads, 1) kv8_tiles_kernel(const Kv8Params P, const Kv8Attn A) {
    using M = TlSmem<D>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ uint32_t tmem_base_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t sm = smem_addr(smem), bars = sm + M::kBars;
    auto bar = [&](int i) { return bars + 8u * i; };

    // the last tiles of a prompt see the most tokens: they go first
    const int idx = A.tiles - 1 - (int)(blockIdx.x / P.hkv), kvh = blockIdx.x % P.hkv, split = blockIdx.z;
    Kv8Seq s;
    int tile;
    if (!kv8_find_tile(P, A, idx, 2 * kTlRows, lane, &s, &tile)) return;
    const int pair0 = tile * 2 * kTlRows, pairs = min(2 * kTlRows, s.n * A.group - pair0);
    const int seq_pos = s.kv - s.n;                              // position of the sequence's first row
    const int pos0 = seq_pos + pair0 / A.group, pos1 = seq_pos + (pair0 + pairs - 1) / A.group;
    if (pos0 < 0 && split == 0) kv8_report(P, H1B_ERR_INVALID_ARG);
    const Kv8Span span = kv8_span(P, A, pos0, pos1);
    const int per = max(((span.count + A.splits - 1) / A.splits + 7) & ~7, 16);
    const int parts = max(1, (span.count + per - 1) / per);
    if (split >= parts) return;
    const int j0 = split * per, j1 = min(j0 + per, span.count);
    const int n_tiles = (j1 - j0 + 7) / 8, n_q = pairs > kTlRows ? 2 : 1;

    if (warp == 12) tmem_alloc(smem_addr(&tmem_base_s), 512);
    if (tid == 0) {
        const int counts[kBarCount] = {8, 4, 4, 1, 1, 4, 4, 1, 1, 4, 4, 4, 4, 1, 1, 4, 4, 1};
#pragma unroll
        for (int i = 0; i < kBarCount; ++i) mbar_init(bar(i), counts[i]);
        mbar_fence_init();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_base_s;
    bool failed = false;

    if (warp < 8) {
        // ---------------------------------------------------------------------------------------- softmax
        const int qt = warp >> 2, row = tid & 127, pair = pair0 + qt * kTlRows + row;
        const bool live = qt * kTlRows + row < pairs;
        const int tok = pair / A.group, head = kvh * A.group + pair % A.group, pos = seq_pos + tok;
        float qs;
        {   // the query row: fp16 multiplied by 2^-e, negated if the scale is negative, into the K-major operand
            const uint16_t *qp = static_cast<const uint16_t *>(A.q) + (int64_t)(s.start + tok) * A.q_rs + (int64_t)head * A.q_hs;
            uint32_t w[D / 2];
            float amax = 0.f;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                uint4 u = make_uint4(0, 0, 0, 0);
                if (live) u = *reinterpret_cast<const uint4 *>(qp + c * 8);
                w[4 * c] = u.x; w[4 * c + 1] = u.y; w[4 * c + 2] = u.z; w[4 * c + 3] = u.w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = pair_to_float2(w[4 * c + i], A.bf16);
                    amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
                }
            }
            const int e = kv8_row_exponent(amax);
            const float up = A.scale_log2 < 0.f ? -pow2i(-e) : pow2i(-e);
            unsigned char *dst = smem + M::kQ + qt * M::kQ1;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                uint32_t h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = pair_to_float2(w[4 * c + i], A.bf16);
                    h[i] = pack_f16x2(f.x * up, f.y * up);
                }
                *reinterpret_cast<uint4 *>(dst + (c >> 3) * (kTlRows * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4)) =
                    make_uint4(h[0], h[1], h[2], h[3]);
            }
            qs = fabsf(A.scale_log2) * kv8_unit<FMT>() * pow2i(e);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kBarQ));

        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t t_s = t_lane + qt * kTlKeys, t_o = t_lane + 2 * kTlKeys + qt * D;
        const int qpos0 = seq_pos + (pair0 + qt * kTlRows) / A.group;          // smallest and largest position of this tile
        const int qpos1 = seq_pos + min(pair0 + pairs - 1, pair0 + qt * kTlRows + kTlRows - 1) / A.group;
        float m = -INFINITY, l = 0.f;
        if (qt < n_q) {
            for (int i = 0; i < n_tiles; ++i) {
                if (!warp_wait(bar(kBarScales + (i & 3)), (i >> 2) & 1) || !warp_wait(bar(kBarS + qt), i & 1)) { failed = true; break; }
                tc_fence_after_sync();
                const unsigned char *stage = smem + M::kScales + (i & 3) * M::kStage;
                const float *ks = reinterpret_cast<const float *>(stage), *vs = ks + 128;
                const int *first = reinterpret_cast<const int *>(stage + 1024);
                const int t0 = first[8];
                const float turn = reinterpret_cast<const float *>(stage + 1024)[9];
                const bool whole = t0 >= 0 && t0 + kTlKeys - 1 <= qpos0 && (!A.window || t0 > qpos1 - A.window || t0 + kTlKeys - 1 < A.sinks);
                // which of 32 columns this row sees, as bits
                auto seen = [&](int c) -> uint32_t {
                    uint32_t bits = 0;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int t = first[2 * c + h];
                        if (t > pos) continue;
                        // tokens t .. t + 15: those <= pos, and of them those > pos - window or < sinks
                        uint32_t b = pos - t >= 15 ? 0xFFFFu : (2u << (pos - t)) - 1u;
                        if (A.window) {
                            const int cut = pos - A.window - t;                // bits 0 .. cut lie before the window
                            const uint32_t in = cut >= 15 ? 0u : cut < 0 ? 0xFFFFu : ~((2u << cut) - 1u);
                            const int left = A.sinks - t;                      // bits 0 .. left - 1 are sinks
                            b &= in | (left >= 16 ? 0xFFFFu : left <= 0 ? 0u : (1u << left) - 1u);
                        }
                        bits |= (b & 0xFFFFu) << (16 * h);
                    }
                    return bits;
                };
                // ---- the row's largest score (before qs >= 0) ----
                float top = -INFINITY;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t sv[32];
                    tmem_ld_32cols(t_s + c * 32, sv);
                    const uint32_t bits = whole ? ~0u : seen(c);
#pragma unroll
                    for (int x = 0; x < 32; x += 4) {
                        const float4 kk = *reinterpret_cast<const float4 *>(ks + c * 32 + x);
                        float z0 = __uint_as_float(sv[x]) * kk.x, z1 = __uint_as_float(sv[x + 1]) * kk.y;
                        float z2 = __uint_as_float(sv[x + 2]) * kk.z, z3 = __uint_as_float(sv[x + 3]) * kk.w;
                        if (!whole) {
                            if (!(bits >> x & 1)) z0 = -INFINITY;
                            if (!(bits >> (x + 1) & 1)) z1 = -INFINITY;
                            if (!(bits >> (x + 2) & 1)) z2 = -INFINITY;
                            if (!(bits >> (x + 3) & 1)) z3 = -INFINITY;
                        }
                        top = fmaxf(top, fmaxf(fmaxf(z0, z1), fmaxf(z2, z3)));
                    }
                }
                top = top == -INFINITY ? top : top * qs;
                const bool move = top > m + kTlLazy;
                if (__any_sync(~0u, move) || turn != 1.f) {
                    const float next = move ? top : m, f = (move ? ex2_approx(m - next) : 1.f) * turn;
                    l *= move ? ex2_approx(m - next) : 1.f;
                    m = next;
                    if (i > 0) {                                  // O holds the tiles before this one: they are done (S was issued after)
#pragma unroll 1
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t ov[32];
                            tmem_ld_32cols(t_o + c * 32, ov);
#pragma unroll
                            for (int x = 0; x < 32; ++x) ov[x] = __float_as_uint(__uint_as_float(ov[x]) * f);
                            tmem_st_32cols(t_o + c * 32, ov);
                        }
                    }
                }
                // ---- weights, over the scores they come from ----
                const uint64_t qs2 = pack2f(qs, qs), nm2 = pack2f(-m, -m);
                uint64_t sum2 = 0;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t sv[32], hi[16], lo[16];
                    tmem_ld_32cols(t_s + c * 32, sv);
                    const uint32_t bits = whole ? ~0u : seen(c);
#pragma unroll
                    for (int x = 0; x < 32; x += 4) {
                        const ulonglong2 kk = *reinterpret_cast<const ulonglong2 *>(ks + c * 32 + x);
                        const ulonglong2 vv = *reinterpret_cast<const ulonglong2 *>(vs + c * 32 + x);
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const int at = x + 2 * y;
                            const float2 z = unpack2(fma2(mul2(pack2(sv[at], sv[at + 1]), y ? kk.y : kk.x), qs2, nm2));
                            float p0 = ex2_approx(z.x), p1 = ex2_approx(z.y);
                            if (!whole) {
                                if (!(bits >> at & 1)) p0 = 0.f;
                                if (!(bits >> (at + 1) & 1)) p1 = 0.f;
                            }
                            const uint64_t pp = pack2f(p0, p1);
                            sum2 = add2(sum2, pp);
                            float2 w = unpack2(mul2(pp, y ? vv.y : vv.x));
                            if (!whole) {                         // (a hidden token's scale may be anything)
                                if (!(bits >> at & 1)) w.x = 0.f;
                                if (!(bits >> (at + 1) & 1)) w.y = 0.f;
                            }
                            hi[at / 2] = pack_f16x2(w.x, w.y);
                            if (SPLIT) {
                                const float2 back = half2_bits_to_float2(hi[at / 2]);
                                lo[at / 2] = pack_f16x2(w.x - back.x, w.y - back.y);
                            }
                        }
                    }
                    tmem_st_16cols_issue(t_s + c * 32, hi);
                    if (SPLIT) tmem_st_16cols_issue(t_s + c * 32 + 16, lo);
                }
                const float2 sum = unpack2(sum2);
                l += sum.x + sum.y;
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kBarP + qt));
            }
            // ---- the result ----
            if (!failed && n_tiles > 0 && !warp_wait(bar(kBarO), 0)) failed = true;
            tc_fence_after_sync();
            if (!failed) {
                float sigma = 0.f;
                if (n_tiles > 0) sigma = reinterpret_cast<const float *>(smem + M::kScales + ((n_tiles - 1) & 3) * M::kStage + 1024)[10];
                const bool empty = l == 0.f;
                const float inv = empty ? 0.f : 1.f / l * (kv8_unit<FMT>() / kTlWeightUnit) * sigma;
                const float lse2 = empty ? -INFINITY : m + log2f(l);
                const int64_t part = ((((int64_t)idx * P.hkv + kvh) * 2 + qt) * kTlRows + row) * A.splits + split;
                uint16_t *op = static_cast<uint16_t *>(A.out) + (int64_t)(s.start + tok) * A.o_rs + (int64_t)head * A.o_hs;
                float *pa = A.part_acc + part * D;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t ov[32];
                    if (n_tiles > 0) tmem_ld_32cols(t_o + c * 32, ov);
#pragma unroll
                    for (int x = 0; x < 32; ++x) ov[x] = empty ? 0u : __float_as_uint(__uint_as_float(ov[x]) * inv);
                    if (live && parts == 1) {
#pragma unroll
                        for (int x = 0; x < 32; x += 8) {
                            uint32_t h[4];
#pragma unroll
                            for (int y = 0; y < 4; ++y)
                                h[y] = float2_to_pair(__uint_as_float(ov[x + 2 * y]), __uint_as_float(ov[x + 2 * y + 1]), A.bf16);
                            *reinterpret_cast<uint4 *>(op + c * 32 + x) = make_uint4(h[0], h[1], h[2], h[3]);
                        }
                    } else if (live) {
#pragma unroll
                        for (int x = 0; x < 32; x += 4)
                            *reinterpret_cast<uint4 *>(pa + c * 32 + x) = make_uint4(ov[x], ov[x + 1], ov[x + 2], ov[x + 3]);
                    }
                    __syncwarp();
                }
                if (live) {
                    if (parts > 1) A.part_lse[part] = lse2;
                    else if (A.lse) A.lse[(int64_t)(s.start + tok) * A.hq + head] = lse2 * kLn2;
                }
            }
        }
    } else if (warp < 12) {
        // ---------------------------------------------------------------------------------------- convert
        const int cw = warp - 8;
        constexpr int ROWS_IT = D == 128 ? 4 : 8, ITS = 32 / ROWS_IT;          // rows per 512 bytes, loads per thread and tile
        // lane -> (row, 16 channels) such that eight neighbouring lanes write 128 different bytes of the swizzled operand
        const int grp = D == 128 ? (lane & 3) | ((lane >> 3) & 1) << 2 : lane & 3;
        const int rr = D == 128 ? ((lane >> 2) & 1) | ((lane >> 4) & 1) << 1 : lane >> 2;
        const int32_t *table = P.table + (int64_t)s.b * P.table_width;
        // lane's block of a tile: lane / 4. Its page (-1: nobody sees it).
        auto page_of = [&](int i) -> int {
            const int j = j0 + i * 8 + (lane >> 2);
            if (i >= n_tiles || j >= j1) return -1;
            const int page = table[span.token(j) / P.page_tokens];
            if (page >= 0 && page < P.n_pages) return page;
            kv8_report(P, H1B_ERR_BOUNDS);
            return -1;
        };
        auto place_of = [&](int i, int page) -> int64_t {                      // token slot of the lane's block, or -1
            if (page < 0) return -1;
            const int t = span.token(j0 + i * 8 + (lane >> 2));
            return ((int64_t)page * P.hkv + kvh) * P.page_tokens + t % P.page_tokens;
        };
        auto load = [&](const uint8_t *base, int64_t place, uint4 (&r)[ITS]) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {                                      // the warp's rows are two of the tile's blocks
                const int64_t at = __shfl_sync(~0u, place, (2 * cw + h) * 4);
#pragma unroll
                for (int it = 0; it < ITS / 2; ++it)
                    r[h * (ITS / 2) + it] = at < 0 ? make_uint4(0, 0, 0, 0)
                                                   : *reinterpret_cast<const uint4 *>(base + (at + it * ROWS_IT + rr) * D + grp * 16);
            }
        };
        auto convert = [&](unsigned char *dst, const uint4 (&r)[ITS]) {
#pragma unroll
            for (int it = 0; it < ITS; ++it) {
                const int rw = 32 * cw + it * ROWS_IT + rr, slab = grp >> 2, c0 = (grp & 3) * 2;
                uint32_t a[8];
                kv8_codes4<FMT>(r[it].x, a[0], a[1]);
                kv8_codes4<FMT>(r[it].y, a[2], a[3]);
                kv8_codes4<FMT>(r[it].z, a[4], a[5]);
                kv8_codes4<FMT>(r[it].w, a[6], a[7]);
                unsigned char *line = dst + slab * 16384 + rw * 128;
                *reinterpret_cast<uint4 *>(line + ((c0 ^ (rw & 7)) << 4)) = make_uint4(a[0], a[1], a[2], a[3]);
                *reinterpret_cast<uint4 *>(line + (((c0 + 1) ^ (rw & 7)) << 4)) = make_uint4(a[4], a[5], a[6], a[7]);
            }
        };
        auto load_scales = [&](const float *base, int64_t place) -> float4 {  // lane's four tokens: block lane / 4, 4 (lane % 4) ..
            return place < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4 *>(base + place + (lane & 3) * 4);
        };
        uint4 kr[ITS], vr[ITS];
        float sigma = 0.f;
        int page = page_of(0), page_next = page_of(1);
        int64_t place = place_of(0, page);
        load(P.k, place, kr);
        float4 ks = load_scales(P.ks, place), vs = load_scales(P.vs, place);
        for (int i = 0; i < n_tiles; ++i) {
            const int st = i & 1;
            load(P.v, place, vr);
            // scales of the tile's 128 tokens (every warp has all of them), those that no row sees cleared
            const int jb = j0 + i * 8 + (lane >> 2), t = jb < j1 ? span.token(jb) : kTlHidden;
            {
                float *kf = &ks.x, *vf = &vs.x;
                float mx = 0.f;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int tt = t + (lane & 3) * 4 + x;
                    if (!(tt <= span.hi && (tt >= span.lo || tt < span.sinks))) kf[x] = vf[x] = 0.f;
                    mx = fmaxf(mx, vf[x] <= 3.402823466e38f ? vf[x] : 0.f);
                }
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, o));
                float turn = 1.f;
                if (mx > 4.f * sigma) {
                    const float next = pow2i(clampi((int)(__float_as_uint(mx) >> 23) - 126, -117, 126));   // > mx
                    turn = sigma / next;
                    sigma = next;
                }
                const float g = sigma > 0.f ? kTlWeightUnit / sigma : 0.f;
                // stage i % 4: its last readers were the softmax warps of tile i - 4, whose weights were contracted before
                // the scores of tile i - 2, which the wait below (or, before it, tile i - 1's) has seen completed
                if (i >= 2 && !warp_wait(bar(kBarKFree + st), ((i >> 1) - 1) & 1)) { failed = true; break; }
                unsigned char *stage = smem + M::kScales + (i & 3) * M::kStage;
                if ((lane >> 3) == cw) {                                       // this warp's 32 tokens
                    *reinterpret_cast<float4 *>(stage + lane * 16) = ks;
                    *reinterpret_cast<float4 *>(stage + 512 + lane * 16) = make_float4(vs.x * g, vs.y * g, vs.z * g, vs.w * g);
                }
                const int shown = page >= 0 ? t : kTlHidden;
                const int t_first = __shfl_sync(~0u, shown, 0), t_last = __shfl_sync(~0u, shown, 28);
                const bool row = __all_sync(~0u, shown != kTlHidden) && t_last - t_first == 112;
                if (cw == 0) {
                    if ((lane & 3) == 0) *reinterpret_cast<int *>(stage + 1024 + lane) = shown;
                    if (lane == 0) {
                        *reinterpret_cast<int *>(stage + 1024 + 32) = row ? t_first : -1;
                        *reinterpret_cast<float *>(stage + 1024 + 36) = turn;
                        *reinterpret_cast<float *>(stage + 1024 + 40) = sigma;
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kBarScales + (i & 3)));
            }
            convert(smem + M::kK + st * M::kKV1, kr);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kBarKFull + st));
            page = page_next;
            page_next = page_of(i + 2);
            place = place_of(i + 1, page);
            if (i + 1 < n_tiles) {
                load(P.k, place, kr);
                ks = load_scales(P.ks, place);
                vs = load_scales(P.vs, place);
            }
            if (i >= 2 && !warp_wait(bar(kBarVFree + st), ((i >> 1) - 1) & 1)) { failed = true; break; }
            convert(smem + M::kV + st * M::kKV1, vr);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kBarVFull + st));
        }
    } else if (lane == 0 && n_tiles > 0) {
        // ---------------------------------------------------------------------------------------- issue
        const uint32_t idesc_s = umma_idesc_f16_m128(kTlKeys), idesc_o = umma_idesc_f16_m128(D) | 1u << 16;   // B: channels contiguous
        auto scores = [&](int qt, int i) {
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const uint32_t off = (ks >> 2) * 16384 + (ks & 3) * 32;
                umma_f16(tmem + qt * kTlKeys, umma_desc_k_sw128(sm + M::kQ + qt * M::kQ1 + off),
                         umma_desc_k_sw128(sm + M::kK + (i & 1) * M::kKV1 + off), idesc_s, ks ? 1u : 0u);
            }
            umma_commit(bar(kBarS + qt));
        };
        auto values = [&](int qt, int i) {
            const uint32_t v = sm + M::kV + (i & 1) * M::kKV1, p = tmem + qt * kTlKeys, o = tmem + 2 * kTlKeys + qt * D;
#pragma unroll
            for (int ks = 0; ks < kTlKeys / 16; ++ks) {
                umma_f16_ta(o, p + weight_column(ks), umma_desc_mn_sw128(v + ks * 2048), idesc_o, (i | ks) ? 1u : 0u);
                if (SPLIT) umma_f16_ta(o, p + weight_column(ks) + 16, umma_desc_mn_sw128(v + ks * 2048), idesc_o, 1u);
            }
        };
        auto wait = [&](int b, uint32_t parity) {
            if (!failed && !mbar_wait_bounded(bar(b), parity, kTlWaitNs)) failed = true;
            return !failed;
        };
        if (wait(kBarQ, 0) && wait(kBarKFull, 0)) {
            tc_fence_after_sync();
            for (int qt = 0; qt < n_q; ++qt) scores(qt, 0);
            umma_commit(bar(kBarKFree));
            for (int i = 0; i < n_tiles && !failed; ++i) {
                if (!wait(kBarVFull + (i & 1), (i >> 1) & 1)) break;
                for (int qt = 0; qt < n_q; ++qt) {
                    if (!wait(kBarP + qt, i & 1)) break;
                    tc_fence_after_sync();
                    values(qt, i);
                    if (qt == n_q - 1) umma_commit(bar(kBarVFree + (i & 1)));
                    if (i + 1 < n_tiles) {
                        if (qt == 0 && !wait(kBarKFull + ((i + 1) & 1), ((i + 1) >> 1) & 1)) break;
                        tc_fence_after_sync();
                        scores(qt, i + 1);
                        if (qt == n_q - 1) umma_commit(bar(kBarKFree + ((i + 1) & 1)));
                    }
                }
            }
        }
        umma_commit(bar(kBarO));
        (void)mbar_wait_bounded(bar(kBarO), 0, kTlWaitNs);       // nothing is in flight when the tensor memory is released
    }
    if (failed) kv8_report(P, H1B_ERR_TIMEOUT);
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 12) { tc_fence_after_sync(); tmem_dealloc(tmem, 512); }
}

template <int D, int FMT, bool SPLIT>
cudaError_t launch_of(const Kv8Params &P, const Kv8Attn &A, cudaStream_t st) {
    constexpr int bytes = TlSmem<D>::kTotal;
    const cudaError_t e = cudaFuncSetAttribute(kv8_tiles_kernel<D, FMT, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)A.tiles * (unsigned)P.hkv, 1, (unsigned)A.splits);
    kv8_tiles_kernel<D, FMT, SPLIT><<<grid, kTlThreads, bytes, st>>>(P, A);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv8_tiles(const Kv8Params &P, const Kv8Attn &A, int d, int fmt, cudaStream_t st) {
    cudaError_t e;
#define H1B_KV8_TILES(D, F) (A.bf16 ? launch_of<D, F, false> : launch_of<D, F, true>)(P, A, st)
    if (d == 128) e = fmt == H1B_KV8_INT8 ? H1B_KV8_TILES(128, H1B_KV8_INT8) : H1B_KV8_TILES(128, H1B_KV8_E4M3);
    else e = fmt == H1B_KV8_INT8 ? H1B_KV8_TILES(64, H1B_KV8_INT8) : H1B_KV8_TILES(64, H1B_KV8_E4M3);
#undef H1B_KV8_TILES
    if (e != cudaSuccess || A.splits == 1) return e;
    return launch_kv8_join(P, A, d, 2 * kTlRows, 8, 16, st);
}

}  // namespace h1b
