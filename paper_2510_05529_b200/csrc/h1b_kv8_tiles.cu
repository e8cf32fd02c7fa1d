// 8-bit pages: attention for many rows per sequence (prompts and chunks of them) on the 5th-generation tensor cores.
//
// One block of 27 warps (and one that only hands over its registers) takes 256 (row, head of the group) pairs of a sequence
// that share a KV head, as two tiles of 128 pairs, and one part of the tokens they see, 64 tokens at a time (four blocks of
// 16, whichever blocks the span lists: sinks and window need not be neighbours). The roles hand each other operands through
// mbarriers; nothing in the loop is block-wide:
//   warps 0-7    softmax of tile A, warps 8-15 of tile B, 16 rows a warp: scores S * ks * qs, the rows' references,
//                weights w = 2^(score - m) * vs / sigma in fp16, written over the scores they came from;
//   warps 16-23  convert (four warps the keys, four the values): codes come from the pages in 16-byte copies, two
//                steps ahead, become exact fp16 numbers ONCE for all 256 pairs and go to shared memory as matrix
//                operands (three of each, 128-byte swizzle; keys K-major, values with the channels contiguous, so nothing
//                is transposed);
//   warps 24, 25 issue the contractions of tile A and of tile B: S = Q K^T into tensor memory, O += P V with P read from
//                tensor memory;
//   warp 26      brings the tokens' scales and says what of a step needs masks.
// Tensor memory holds two sets of scores for each tile, so the scores of the next step are there when a softmax warp has
// finished with this one. m and sigma follow lazily (as in the kernel for few rows): O is rescaled only when a score exceeds
// m by 4 (in log2) or a value scale exceeds 4 sigma; weights are carried times 2^9. For fp16 results (SPLIT) a second
// contraction adds what rounding the weights left over.
//
// What bounds it: instruction issue (66 % of the slots; the tensor cores are busy 40 % of the time). A prompt of 8192 tokens,
// 32 heads of 128, takes 825 us = 668 TFLOP/s, 40 % of the measured bf16 rate; a softmax warp spends some 290 instructions on
// a step, half of them the arithmetic of its 16 x 64 scores. Steps on the way there (the same prompt): one thread issuing
// for both tiles, a single set of scores and 128 tokens a step 1194 us (the roles' loops together did not fit the instruction
// cache: 85 % hits), two threads, two sets, 64 tokens 935 (99 % hits), copies two steps ahead and a warp for the scales 873,
// sixteen softmax warps of 16 rows instead of eight of 32 (more warps to hide each other's latencies) 841, the masks' flags
// made by the scales' warp 825.
// Every wait is bounded; a role that gives up records the time-out and leaves, and the block releases its tensor memory.
#include <type_traits>

#include "h1b_kv8.cuh"

namespace h1b {

namespace {

constexpr int kTlRows = 128, kTlKeys = 64, kTlBlocks = kTlKeys / kKv8Block;
constexpr int kTlSoftmax = 16;                                 // softmax warps, then 8 convert, 2 issue, 1 scales; the last
constexpr int kTlThreads = (kTlSoftmax + 12) * 32;             // only hands over its registers
constexpr int kTlRegsLaunch = 72, kTlRegsSoftmax = 88, kTlRegsConvert = 48, kTlRegsIssue = 56;
static_assert(kTlSoftmax * 32 * kTlRegsSoftmax + 256 * kTlRegsConvert + 128 * kTlRegsIssue <= kTlThreads * kTlRegsLaunch,
              "more registers than a block is launched with");
constexpr float kTlLazy = 4.f, kTlWeightUnit = 512.f;
constexpr int kTlHidden = 1 << 30;                             // "first token" of a block that nobody sees: beyond every position
constexpr int kTlUnit = kTlBlocks, kTlMinBlocks = 16;         // a part is whole steps, and 256 tokens at least
constexpr int kTlStages = 3, kTlScaleStages = 4, kTlRawStages = 3;

// What a block works on, in shared memory: each role reads what it needs where it needs it. (Kept in registers across the
// roles' branches it was spilled, and a reload from local memory, whose lines the codes push out of the small L1, held up
// the issuing thread for longer than its contractions took.)
struct TlWork {
    int64_t part0;                                               // index of (first row, this part) among the partial results
    int go, seq, start, seq_pos, pair0, pairs, parts, lo, hi, sinks, sink_blocks, first, j0, j1, n_tiles, n_q;
    uint32_t tmem;
};

template <int D>
struct TlSmem {
    static constexpr int kQ1 = kTlRows * D * 2, kKV1 = kTlKeys * D * 2, kRaw1 = 2 * kTlKeys * D;
    static constexpr int kQ = 0, kK = 2 * kQ1, kV = kK + kTlStages * kKV1, kRaw = kV + kTlStages * kKV1;
    static constexpr int kScales = kRaw + kTlRawStages * kRaw1;
    // per scale stage: ks [64], vs / sigma [64], blocks' first tokens [4], {turn, sigma}, {for tiles A and B: bit 0 every row
    // sees all 64 tokens, bit 1 turn is not 1}
    static constexpr int kVs = kTlKeys * 4, kFirst = 2 * kTlKeys * 4, kStage = kFirst + 32;
    static constexpr int kRows = kScales + kTlScaleStages * kStage;              // qs [256], positions [256]
    static constexpr int kBars = kRows + 2 * kTlRows * 8;
    static constexpr int kTotal = kBars + 512 + 1024;            // + slack to align the operands to 1024 bytes
};
enum { kBarQ = 0, kBarFull = 1, kBarKFree = 4, kBarVFree = 7, kBarScales = 10, kBarS = 14, kBarP = 18, kBarPV = 22, kBarO = 26,
       kBarCount = 28 };

// Matrix descriptors of operands in shared memory, 128-byte swizzle: the lower word is the start address (16-byte units) and
// the leading offset, the upper word the stride between groups of eight rows (1024 bytes), the version and the layout. Only
// the address changes from one contraction to the next, so the one issuing thread, which has some 50 cycles for each, adds
// to a lower word and does nothing else.
//   K-major: rows of 128 bytes (64 numbers along K), the leading offset is unused.
//   MN-major (channels contiguous): rows of 128 bytes (64 channels) per token; the next 64 channels `lead` bytes on.
constexpr uint32_t kDescHi = (1024u >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lead) { return (addr >> 4) | (lead >> 4) << 16; }
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"((uint32_t)add), "n"(kDescHi) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}"
        ::"r"(d), "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"((uint32_t)add), "n"(kDescHi) : "memory");
}
// Tensor memory in the layout of a matrix fragment: 16 lanes (rows) x 32 columns; register 4 b + 2 y + x of lane l holds row
// 8 y + l / 4, column 8 b + 2 (l % 4) + x. A lane then meets 8 of 32 columns instead of all, so what belongs to a column (its
// token's scales) is read from shared memory a quarter as often as with one row per lane: with that, the reads took most
// of the time that shared memory has beside the contractions' operands.
__device__ __forceinline__ void tmem_ld_frag_issue(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_tie16(uint32_t (&r)[16]) {
    asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
}
// The store of the same fragment.
__device__ __forceinline__ void tmem_st_frag_f32(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// 16 rows x 4 N columns of 32 bits: register 2 b + y of lane l is row 8 y + l / 4, column 4 b + l % 4.
__device__ __forceinline__ void tmem_st_frag16(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tmem_st_frag32(uint32_t taddr, const uint32_t (&r)[8], const uint32_t (&s)[8]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(s[0]), "r"(s[1]), "r"(s[2]), "r"(s[3]), "r"(s[4]), "r"(s[5]), "r"(s[6]), "r"(s[7]) : "memory");
}
// A bounded wait: a look, then at most 2^20 looks that may each park the warp for about 2 us while the phase is incomplete
// (a second or two). It is written out at each place it is used, so it is short: the loops of the three roles have to stay
// in the instruction cache together (when they did not, instruction fetches bound the kernel).
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity) {
    if (mbar_try_wait(bar, parity)) return true;
#pragma unroll 1
    for (int i = 0; i < 1 << 20; ++i)
        if (mbar_try_wait_parked(bar, parity, H1B_WAIT_PARK_NS)) return true;
    return false;
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) { return __all_sync(~0u, wait_phase(bar, parity)); }
// Two at once (a look takes 100 cycles and more when shared memory is busy).
__device__ __forceinline__ bool warp_wait2(uint32_t bar0, uint32_t parity0, uint32_t bar1, uint32_t parity1) {
    const bool a = mbar_try_wait(bar0, parity0), b = mbar_try_wait(bar1, parity1);
    return __all_sync(~0u, a && b) || (warp_wait(bar0, parity0) && warp_wait(bar1, parity1));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Where the weights of contraction step ks (16 tokens) lie within a set of scores' 64 columns: 32 columns of scores become 16
// columns of weights (two to a column) and 16 of their remainders.
__device__ __forceinline__ uint32_t weight_column(int ks) { return (ks >> 1) * 32 + (ks & 1) * 8; }

template <int D, int FMT, bool SPLIT>
__global__ void __launch_bounds__(kTlThreads, 1) kv8_tiles_kernel(const Kv8Params P, const Kv8Attn A) {
    using M = TlSmem<D>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ TlWork work_s;
    const volatile TlWork &W = work_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t sm = smem_addr(smem), bars = sm + M::kBars;
    auto bar = [&](int i) { return bars + 8u * i; };

    if (warp == 0) {
        // the last tiles of a prompt see the most tokens: they go first
        const int idx = A.tiles - 1 - (int)(blockIdx.x / P.hkv), split = blockIdx.z;
        Kv8Seq s;
        int tile;
        bool go = kv8_find_tile(P, A, idx, 2 * kTlRows, lane, &s, &tile);
        if (go) {
            const int pair0 = tile * 2 * kTlRows, pairs = min(2 * kTlRows, s.n * A.group - pair0);
            const int seq_pos = s.kv - s.n;                      // position of the sequence's first row
            const int pos0 = seq_pos + pair0 / A.group, pos1 = seq_pos + (pair0 + pairs - 1) / A.group;
            if (pos0 < 0 && split == 0) kv8_report(P, H1B_ERR_INVALID_ARG);
            const Kv8Span span = kv8_span(P, A, pos0, pos1);
            const int per = max(((span.count + A.splits - 1) / A.splits + kTlUnit - 1) / kTlUnit * kTlUnit, kTlMinBlocks);
            const int parts = max(1, (span.count + per - 1) / per);
            go = split < parts;
            if (lane == 0) {
                const int j0 = split * per, j1 = min(j0 + per, span.count);
                work_s.part0 = (((int64_t)idx * P.hkv + (int)(blockIdx.x % P.hkv)) * 2 * kTlRows) * A.splits + split;
                work_s.seq = s.b; work_s.start = s.start; work_s.seq_pos = seq_pos;
                work_s.pair0 = pair0; work_s.pairs = pairs; work_s.parts = parts;
                work_s.lo = span.lo; work_s.hi = span.hi; work_s.sinks = span.sinks;
                work_s.sink_blocks = span.sink_blocks; work_s.first = span.first;
                work_s.j0 = j0; work_s.j1 = j1;
                work_s.n_tiles = (j1 - j0 + kTlBlocks - 1) / kTlBlocks;
                work_s.n_q = pairs > kTlRows ? 2 : 1;
            }
        }
        if (lane == 0) work_s.go = go;
    } else if (warp == 1 && blockIdx.z == 0) {
        kv8_check_batch(P, blockIdx.x, gridDim.x, lane);
    }
    __syncthreads();
    if (!W.go) return;
    if (warp == kTlSoftmax + 8) tmem_alloc(smem_addr(&work_s.tmem), 512);
    if (tid == 0) {
        for (int i = 0; i < kBarCount; ++i) {                    // arrivals: one a warp, or one commit
            int n = 1;
            if (i == kBarQ) n = kTlSoftmax;
            else if (i >= kBarFull && i < kBarKFree) n = 8;
            else if (i >= kBarP && i < kBarPV) n = kTlSoftmax / 2;
            else if (i >= kBarKFree && i < kBarScales) n = W.n_q;
            mbar_init(bar(i), n);
        }
        mbar_fence_init();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    bool failed = false;

    if (warp < kTlSoftmax) {
        more_registers<kTlRegsSoftmax>();
        // ---------------------------------------------------------------------------------------- softmax
        // A warp has 16 rows of a tile in fragment layout: rows gi and gi + 8 of them are this lane's, four lanes to a row.
        // (A warp reaches the quarter of tensor memory of its number % 4.)
        const int qt = warp / (kTlSoftmax / 2), gi = lane >> 2, tj = lane & 3;
        const int row0 = (warp & 3) * 32 + (warp & 4) * 4;
        // the query rows, two threads to a row: fp16 multiplied by 2^-e, negated if the scale is negative, into the K-major
        // operand
#pragma unroll 1
        for (int r = tid >> 1; r < 2 * kTlRows; r += kTlSoftmax * 16) {
            const int half = tid & 1;
            const int pair = W.pair0 + r, tok = pair / A.group, head = (int)(blockIdx.x % P.hkv) * A.group + pair % A.group;
            const bool live = r < W.pairs;
            const uint16_t *qp = static_cast<const uint16_t *>(A.q) + (int64_t)(W.start + tok) * A.q_rs + (int64_t)head * A.q_hs + half * (D / 2);
            uint32_t w[D / 4];
            float amax = 0.f;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                uint4 u = make_uint4(0, 0, 0, 0);
                if (live) u = *reinterpret_cast<const uint4 *>(qp + c * 8);
                w[4 * c] = u.x; w[4 * c + 1] = u.y; w[4 * c + 2] = u.z; w[4 * c + 3] = u.w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = pair_to_float2(w[4 * c + i], A.bf16);
                    amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
                }
            }
            amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
            const int e = kv8_row_exponent(amax);
            const float up = A.scale_log2 < 0.f ? -pow2i(-e) : pow2i(-e);
            unsigned char *dst = smem + M::kQ + (r >> 7) * M::kQ1 + (r & 127) * 128;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                uint32_t h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = pair_to_float2(w[4 * c + i], A.bf16);
                    h[i] = pack_f16x2(f.x * up, f.y * up);
                }
                const int ch = half * (D / 16) + c;
                *reinterpret_cast<uint4 *>(dst + (ch >> 3) * (kTlRows * 128) + (((ch & 7) ^ (r & 7)) << 4)) =
                    make_uint4(h[0], h[1], h[2], h[3]);
            }
            if (half == 0) {
                reinterpret_cast<float *>(smem + M::kRows)[r] = fabsf(A.scale_log2) * pow2i(e);
                reinterpret_cast<int *>(smem + M::kRows)[2 * kTlRows + r] = W.seq_pos + tok;
            }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kBarQ));
        if (!warp_wait(bar(kBarQ), 0)) failed = true;            // (the rows of a warp came through others)

        const uint32_t t_lane = W.tmem + ((uint32_t)row0 << 16), t_o = t_lane + 4 * kTlKeys + qt * D;
        const int n_tiles = W.n_tiles;
        uint64_t qs2[2], nm2[2], l2[2];                              // of each row, twice: qs, -m, and the two halves of the sum
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const float qs = reinterpret_cast<const float *>(smem + M::kRows)[qt * kTlRows + row0 + 8 * q + gi];
            qs2[q] = pack2f(qs, qs);
            nm2[q] = pack2f(INFINITY, INFINITY);
            l2[q] = 0;
        }
        const int *row_pos = reinterpret_cast<const int *>(smem + M::kRows) + 2 * kTlRows + qt * kTlRows + row0 + gi;
        if (qt < W.n_q) {
            for (int i = 0; i < n_tiles && !failed; ++i) {
                if (!warp_wait2(bar(kBarScales + (i & 3)), (i >> 2) & 1, bar(kBarS + qt * 2 + (i & 1)), (i >> 1) & 1)) {
                    failed = true;
                    break;
                }
                tc_fence_after_sync();
                const uint32_t t_s = t_lane + (qt * 2 + (i & 1)) * kTlKeys;
                uint32_t sv[2][16];                              // [32 columns]
#pragma unroll
                for (int c = 0; c < 2; ++c) tmem_ld_frag_issue(t_s + c * 32, sv[c]);
                const unsigned char *stage = smem + M::kScales + (i & 3) * M::kStage;
                const unsigned char *ks = stage + tj * 8, *vs = ks + M::kVs;   // pairs of columns 8 b + 2 tj, + 1
                const int *first = reinterpret_cast<const int *>(stage + M::kFirst);
                const int how = first[6 + qt];
                const bool whole = how & 1;
                // bit 2 b + x of seen[q]: row q of the lane sees column 8 b + 2 tj + x
                uint32_t seen[2] = {};
                if (!whole) {
#pragma unroll 1
                    for (int b = 7; b >= 0; --b) {
                        const int t = first[b >> 1] + (b & 1) * 8 + 2 * tj;
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const int pos = row_pos[8 * q];
                            const bool s0 = t <= pos && (!A.window || t > pos - A.window || t < A.sinks);
                            const bool s1 = t + 1 <= pos && (!A.window || t + 1 > pos - A.window || t + 1 < A.sinks);
                            seen[q] = seen[q] << 2 | (uint32_t)s0 | (uint32_t)s1 << 1;
                        }
                    }
                }
                tmem_ld_wait();
#pragma unroll
                for (int c = 0; c < 2; ++c) tmem_tie16(sv[c]);
                // ---- scores times the keys' scales, and the rows' largest (before qs >= 0) ----
                float top[2];
#pragma unroll
                for (int q = 0; q < 2; ++q) top[q] = -INFINITY;
#pragma unroll
                for (int b = 0; b < 8; ++b) {
                    const uint64_t kk = *reinterpret_cast<const uint64_t *>(ks + b * 32);
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        uint32_t *r = &sv[b >> 2][(b & 3) * 4 + q * 2];
                        const float2 z = unpack2(mul2(pack2(r[0], r[1]), kk));
                        r[0] = __float_as_uint(z.x);
                        r[1] = __float_as_uint(z.y);
                    }
                }
                if (!whole) {
#pragma unroll
                    for (int b = 0; b < 8; ++b)
#pragma unroll
                        for (int q = 0; q < 2; ++q)
#pragma unroll
                            for (int x = 0; x < 2; ++x)
                                if (!(seen[q] >> (2 * b + x) & 1)) sv[b >> 2][(b & 3) * 4 + q * 2 + x] = 0xFF800000u;
                }
#pragma unroll
                for (int b = 0; b < 8; ++b)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const uint32_t *r = &sv[b >> 2][(b & 3) * 4 + q * 2];
                        top[q] = max3(top[q], __uint_as_float(r[0]), __uint_as_float(r[1]));
                    }
                float over = -INFINITY;                           // how far a score lies above its row's reference
#pragma unroll
                for (int q = 0; q < 2; ++q) over = fmaxf(over, fmaf(top[q], unpack2(qs2[q]).x, unpack2(nm2[q]).x));
                if (__any_sync(~0u, over > kTlLazy) || (how & 2)) {
                    const float turn = reinterpret_cast<const float *>(first)[4];
                    float f[2];
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const float m = -unpack2(nm2[q]).x;
                        float x = top[q] == -INFINITY ? top[q] : top[q] * unpack2(qs2[q]).x;
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 2));
                        const bool up = x > m + kTlLazy;
                        const float g = up ? ex2_approx(m - x) : 1.f;
                        l2[q] = mul2(l2[q], pack2f(g, g));
                        if (up) nm2[q] = pack2f(-x, -x);
                        f[q] = g * turn;
                    }
                    if (i > 0) {
                        // O holds the steps before this one, and the last of them may still be running (the step before that
                        // one with the same barrier is long done: the scores of step i - 1 were issued after it)
                        if (!warp_wait(bar(kBarPV + qt * 2 + ((i - 1) & 1)), ((i - 1) >> 1) & 1)) { failed = true; break; }
                        tc_fence_after_sync();
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            uint32_t ov[16];
                            tmem_ld_frag_issue(t_o + c, ov);
                            tmem_ld_wait();
                            tmem_tie16(ov);
#pragma unroll
                            for (int x = 0; x < 16; ++x) ov[x] = __float_as_uint(__uint_as_float(ov[x]) * f[(x >> 1) & 1]);
                            tmem_st_frag_f32(t_o + c, ov);
                        }
                        tmem_st_wait();
                    }
                }
                // ---- weights, over the scores they come from ----
                auto weigh = [&](auto masked) {
                    constexpr bool MASK = decltype(masked)::value;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t hi[8], lo[8];
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            const uint64_t vv = *reinterpret_cast<const uint64_t *>(vs + (c * 4 + b) * 32);
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const uint32_t *r = &sv[c][b * 4 + q * 2];
                                const float2 z = unpack2(fma2(pack2(r[0], r[1]), qs2[q], nm2[q]));
                                float p0 = ex2_approx(z.x), p1 = ex2_approx(z.y);
                                const bool s0 = !MASK || (seen[q] >> (8 * c + 2 * b) & 1);
                                const bool s1 = !MASK || (seen[q] >> (8 * c + 2 * b + 1) & 1);
                                if (MASK) {
                                    if (!s0) p0 = 0.f;
                                    if (!s1) p1 = 0.f;
                                }
                                const uint64_t pp = pack2f(p0, p1);
                                l2[q] = add2(l2[q], pp);
                                uint64_t ww = mul2(pp, vv);
                                if (MASK) {                       // (a hidden token's scale may be anything)
                                    float2 w = unpack2(ww);
                                    if (!s0) w.x = 0.f;
                                    if (!s1) w.y = 0.f;
                                    ww = pack2f(w.x, w.y);
                                }
                                const float2 w = unpack2(ww);
                                uint32_t &h = hi[b * 2 + q];
                                h = pack_f16x2(w.x, w.y);
                                if (SPLIT) {
                                    const float2 back = half2_bits_to_float2(h);
                                    const float2 rest = unpack2(fma2(pack2f(back.x, back.y), pack2f(-1.f, -1.f), ww));
                                    lo[b * 2 + q] = pack_f16x2(rest.x, rest.y);
                                }
                            }
                        }
                        if (SPLIT) tmem_st_frag32(t_s + c * 32, hi, lo);
                        else tmem_st_frag16(t_s + c * 32, hi);
                    }
                };
                if (whole) weigh(std::false_type()); else weigh(std::true_type());
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kBarP + qt * 2 + (i & 1)));
            }
            // ---- the result ----
            if (!failed && n_tiles > 0 && !warp_wait(bar(kBarO + qt), 0)) failed = true;
            tc_fence_after_sync();
            if (!failed) {
                float unit = 0.f;                                // sigma / kTlWeightUnit; a factor of its own: with 1 / l it may be subnormal
                if (n_tiles > 0)
                    unit = reinterpret_cast<const float *>(smem + M::kScales + ((n_tiles - 1) & 3) * M::kStage + M::kFirst)[5] * (1.f / kTlWeightUnit);
                const int parts = W.parts;
                float inv[2];
                bool live[2];
                uint16_t *op[2];
                float *pa[2];
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const float2 x = unpack2(l2[q]);
                    float l = x.x + x.y;
                    l += __shfl_xor_sync(~0u, l, 1);
                    l += __shfl_xor_sync(~0u, l, 2);
                    const bool empty = l == 0.f;
                    inv[q] = empty ? 0.f : 1.f / l;
                    const float lse2 = empty ? -INFINITY : log2f(l) - unpack2(nm2[q]).x;
                    const int r = qt * kTlRows + row0 + 8 * q + gi, pair = W.pair0 + r, tok = W.start + pair / A.group;
                    const int head = (int)(blockIdx.x % P.hkv) * A.group + pair % A.group;
                    live[q] = r < W.pairs;
                    op[q] = static_cast<uint16_t *>(A.out) + (int64_t)tok * A.o_rs + (int64_t)head * A.o_hs + 2 * tj;
                    const int64_t part = W.part0 + (int64_t)r * A.splits;
                    pa[q] = A.part_acc + part * D + 2 * tj;
                    if (live[q] && tj == 0) {
                        if (parts > 1) A.part_lse[part] = lse2;
                        else if (A.lse) A.lse[(int64_t)tok * A.hq + head] = lse2 * kLn2;
                    }
                }
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t ov[16];
                    if (n_tiles > 0) {
                        tmem_ld_frag_issue(t_o + c, ov);
                        tmem_ld_wait();
                        tmem_tie16(ov);
                    }
#pragma unroll
                    for (int b = 0; b < 4; ++b)
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            if (!live[q]) continue;
                            const float u = n_tiles > 0 ? __uint_as_float(ov[b * 4 + q * 2]) * inv[q] * unit : 0.f;
                            const float v = n_tiles > 0 ? __uint_as_float(ov[b * 4 + q * 2 + 1]) * inv[q] * unit : 0.f;
                            if (parts == 1) *reinterpret_cast<uint32_t *>(op[q] + c + b * 8) = float2_to_pair(u, v, A.bf16);
                            else *reinterpret_cast<float2 *>(pa[q] + c + b * 8) = make_float2(u, v);
                        }
                    __syncwarp();
                }
            }
        }
    } else if (warp < kTlSoftmax + 8) {
        fewer_registers<kTlRegsConvert>();
        // ---------------------------------------------------------------------------------------- convert
        const bool keys = warp < kTlSoftmax + 4;
        const int cw = warp & 3;
        constexpr int ROWS_IT = D == 128 ? 4 : 8, ITS = 16 / ROWS_IT;          // rows per 512 bytes, loads per thread and step
        // A warp converts one block of each step. lane -> (row, 16 channels) such that eight neighbouring lanes write 128
        // different bytes of the swizzled operand. The codes come to shared memory with asynchronous copies two steps ahead; a
        // lane converts the very bytes that it copied, so nobody else has to know.
        const int grp = D == 128 ? (lane & 3) | ((lane >> 3) & 1) << 2 : lane & 3;
        const int rr = D == 128 ? ((lane >> 2) & 1) | ((lane >> 4) & 1) << 1 : lane >> 2;
        const uint8_t *codes = (keys ? P.k : P.v) + (int64_t)(blockIdx.x % P.hkv) * P.page_tokens * D + rr * D + grp * 16;
        const int32_t *table = P.table + (int64_t)W.seq * P.table_width;
        const uint32_t raw = sm + M::kRaw + (warp - kTlSoftmax) * 16 * D + lane * 16;
        const int n_tiles = W.n_tiles, j_first = W.j0 + cw, j1 = W.j1, sink_blocks = W.sink_blocks, skip = W.first - sink_blocks;
        const int lo = W.lo, hi = W.hi, sinks = W.sinks;
        int offset = 0, page = -1;                                              // asked for last: the block's place in its page, the page
        auto block_of = [&](int i) { const int j = j_first + i * kTlBlocks; return j < sink_blocks ? j : j + skip; };
        auto look_up = [&](int i) {
            page = -1;
            if (j_first + i * kTlBlocks >= j1) return;
            const int blk = block_of(i), col = kv8_page_of(P, blk);
            offset = blk * kKv8Block - col * P.page_tokens;
            page = table[col];
        };
        auto fetch = [&](int stage) {                                           // the copies of the step looked up
            const bool ok = page >= 0 && page < P.n_pages;                      // (a block that nobody sees: zeros)
            const uint8_t *src = codes + ((int64_t)(ok ? page : 0) * P.hkv * P.page_tokens + offset) * D;
#pragma unroll
            for (int it = 0; it < ITS; ++it)
                cp_async_16(raw + stage * M::kRaw1 + it * 512, src + it * ROWS_IT * D, ok ? 16 : 0);
            cp_async_commit();
        };
        look_up(0);
        fetch(0);
        look_up(1);
        fetch(1);
        look_up(2);
        int st = 0, phase = 1;                                                  // i % 3, and i / 3 - 1 as a parity
#pragma unroll 1
        for (int i = 0; i < n_tiles; ++i) {
            fetch(st == 0 ? 2 : st - 1);                                        // step i + 2 into (i + 2) % 3, which was read in step i - 1
            look_up(i + 3);
            if (i >= kTlStages && !warp_wait(bar((keys ? kBarKFree : kBarVFree) + st), phase)) { failed = true; break; }
            cp_async_wait_group<2>();                                           // this step's copies
            unsigned char *line = smem + (keys ? M::kK : M::kV) + st * M::kKV1 + (grp >> 2) * (kTlKeys * 128) + (16 * cw + rr) * 128;
            unsigned char *src = smem + (raw - sm) + st * M::kRaw1;
            if (FMT == H1B_KV8_E4M3 && !keys) {
                // codes that no row sees may be NaN patterns, and their weight zero times NaN is none: they become zeros (a key's
                // only reach a score that is hidden)
                const int t = block_of(i) * kKv8Block;
                if (!(t + 15 <= hi && (t >= lo || t + 15 < sinks))) {
#pragma unroll 1
                    for (int it = 0; it < ITS; ++it) {
                        const int tt = t + it * ROWS_IT + rr;
                        if (!(tt <= hi && (tt >= lo || tt < sinks))) *reinterpret_cast<uint4 *>(src + it * 512) = make_uint4(0, 0, 0, 0);
                    }
                }
            }
#pragma unroll
            for (int it = 0; it < ITS; ++it) {
                const int rw = it * ROWS_IT + rr, c0 = (grp & 3) * 2;          // (row % 8: the block's first row is a multiple of 16)
                const uint4 r = *reinterpret_cast<const uint4 *>(src + it * 512);
                uint32_t a[8];
                kv8_codes4<FMT>(r.x, a[0], a[1]);
                kv8_codes4<FMT>(r.y, a[2], a[3]);
                kv8_codes4<FMT>(r.z, a[4], a[5]);
                kv8_codes4<FMT>(r.w, a[6], a[7]);
                *reinterpret_cast<uint4 *>(line + it * ROWS_IT * 128 + ((c0 ^ (rw & 7)) << 4)) = make_uint4(a[0], a[1], a[2], a[3]);
                *reinterpret_cast<uint4 *>(line + it * ROWS_IT * 128 + (((c0 + 1) ^ (rw & 7)) << 4)) = make_uint4(a[4], a[5], a[6], a[7]);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kBarFull + st));
            if (++st == kTlStages) { st = 0; phase ^= 1; }
        }
        cp_async_wait_group<0>();
    } else {
        fewer_registers<kTlRegsIssue>();
        // ---------------------------------------------------------------------------------------- issue
        // A thread for each of the two tiles: a wait that need not wait still takes it some 200 cycles, and one thread for
        // both had no time left to keep the tensor cores busy.
        const int qt = warp - (kTlSoftmax + 8);
        if (qt == 2) {
            // ------------------------------------------------------------------------------------ scales
            // Lanes 4 x .. 4 x + 3 look after block x % 4 of a step: its first token, its page, and the scales of tokens
            // 4 (lane % 4) .. + 3 of it, the keys' (lanes 0 - 15) or the values' (16 - 31). The table is read two steps ahead,
            // the scales one.
            const bool keys = lane < 16;
            const float *scales = (keys ? P.ks : P.vs) + (int64_t)(blockIdx.x % P.hkv) * P.page_tokens + (lane & 3) * 4;
            const int32_t *table = P.table + (int64_t)W.seq * P.table_width;
            const int n_tiles = W.n_tiles, j_first = W.j0 + ((lane >> 2) & 3), j1 = W.j1, sink_blocks = W.sink_blocks, skip = W.first - sink_blocks;
            const int lo = W.lo, hi = W.hi, sinks = W.sinks;
            // the smallest and largest position of tile A (lane 0) and B (lane 1)
            const int pos0 = W.seq_pos + (W.pair0 + (lane & 1) * kTlRows) / A.group;
            const int pos1 = W.seq_pos + (W.pair0 + min(W.pairs, (lane & 1) * kTlRows + kTlRows) - 1) / A.group;
            int t_next = kTlHidden, offset = 0, page = -1;
            auto look_up = [&](int i) {
                const int j = j_first + i * kTlBlocks;
                t_next = kTlHidden;
                if (j >= j1) return;
                const int blk = j < sink_blocks ? j : j + skip, col = kv8_page_of(P, blk);
                t_next = blk * kKv8Block;
                offset = t_next - col * P.page_tokens;
                page = table[col];
            };
            int t;
            float4 sc;
            auto fetch = [&]() {                                                // the scales of the step looked up
                t = t_next;
                if (t != kTlHidden && (page < 0 || page >= P.n_pages)) {
                    kv8_report(P, H1B_ERR_BOUNDS);
                    t = kTlHidden;
                }
                sc = make_float4(0.f, 0.f, 0.f, 0.f);
                if (t != kTlHidden) sc = __ldcg(reinterpret_cast<const float4 *>(scales + (int64_t)page * P.hkv * P.page_tokens + offset));
            };
            look_up(0);
            fetch();
            look_up(1);
            float sigma = 0.f;
            int st = 0, phase = 1;
#pragma unroll 1
            for (int i = 0; i < n_tiles; ++i) {
                // Stage i % 4 was last read in step i - 4, whose weights had been contracted before those of step i - 3.
                if (i >= kTlStages && !warp_wait(bar(kBarVFree + st), phase)) { failed = true; break; }
                unsigned char *stage = smem + M::kScales + (i & 3) * M::kStage;
                float *f = &sc.x;
                float mx = 0.f;
#pragma unroll
                for (int y = 0; y < 4; ++y) {                                   // what no row sees may be anything
                    const int tt = t + (lane & 3) * 4 + y;
                    if (!(tt <= hi && (tt >= lo || tt < sinks))) f[y] = 0.f;
                    mx = fmaxf(mx, !keys && f[y] <= 3.402823466e38f ? f[y] : 0.f);
                }
                float turn = 1.f;                                               // old sigma / new sigma
                if (__any_sync(~0u, mx > 4.f * sigma)) {
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, o));
                    const float next = pow2i(clampi((int)(__float_as_uint(mx) >> 23) - 126, -117, 126));       // > mx
                    turn = sigma / next;
                    sigma = next;
                }
                const float g = keys ? 1.f : sigma > 0.f ? kTlWeightUnit / sigma : 0.f;
                *reinterpret_cast<float4 *>(stage + lane * 16) = make_float4(sc.x * g, sc.y * g, sc.z * g, sc.w * g);
                const int t_first = __shfl_sync(~0u, t, 0), t_last = __shfl_sync(~0u, t, 12);
                const bool row = __all_sync(~0u, t != kTlHidden) && t_last - t_first == kTlKeys - 16;
                if (keys && (lane & 3) == 0) *reinterpret_cast<int *>(stage + M::kFirst + lane) = t;
                if (lane < 2) {                                                 // a lane for each tile
                    const bool whole = row && t_last + 15 <= pos0 && (!A.window || t_first > pos1 - A.window || t_last + 15 < A.sinks);
                    reinterpret_cast<int *>(stage + M::kFirst)[6 + lane] = (int)whole | (turn != 1.f ? 2 : 0);
                    reinterpret_cast<float *>(stage + M::kFirst)[4 + lane] = lane ? sigma : turn;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kBarScales + (i & 3)));
                fetch();
                look_up(i + 2);
                if (++st == kTlStages) { st = 0; phase ^= 1; }
            }
        } else if (qt < W.n_q && lane == 0 && W.n_tiles > 0) {
            const uint32_t s_at = W.tmem + qt * 2 * kTlKeys, o_at = W.tmem + 4 * kTlKeys + qt * D;
            const int n_tiles = W.n_tiles;
            const uint32_t idesc_s = umma_idesc_f16_m128(kTlKeys), idesc_o = umma_idesc_f16_m128(D) | 1u << 16;   // B: channels contiguous
            const uint32_t q_lo = desc_lo(sm + M::kQ + qt * M::kQ1, 16), k_lo = desc_lo(sm + M::kK, 16);
            const uint32_t v_lo = desc_lo(sm + M::kV, kTlKeys * 128);
            auto wait = [&](int b, uint32_t parity) {
                if (!failed && !wait_phase(bar(b), parity)) failed = true;
                return !failed;
            };
            int k_st = 0, k_turn = 0, v_st = 0;                     // stage and phase of the next scores, stage of the next values
            auto scores = [&](int i) {                             // (the keys and values of a step become full together)
                if (!wait(kBarFull + k_st, k_turn)) return;
                tc_fence_after_sync();
                const uint32_t k = k_lo + k_st * (M::kKV1 >> 4), to = s_at + (i & 1) * kTlKeys;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    mma_ss(to, q_lo + (ks >> 2) * (kTlRows * 128 >> 4) + (ks & 3) * 2, k + (ks >> 2) * (kTlKeys * 128 >> 4) + (ks & 3) * 2,
                           idesc_s, ks != 0);
                umma_commit(bar(kBarS + qt * 2 + (i & 1)));
                umma_commit(bar(kBarKFree + k_st));
                if (++k_st == kTlStages) { k_st = 0; k_turn ^= 1; }
            };
            // Scores run two steps ahead of the values: step i + 2's go where step i's weights were, after the contraction that
            // reads those (this thread issues both, and they execute in order).
            if (wait(kBarQ, 0))
                for (int i = 0; i < 2 && i < n_tiles && !failed; ++i) scores(i);
#pragma unroll 1
            for (int i = 0; i < n_tiles && !failed; ++i) {
                if (!wait(kBarP + qt * 2 + (i & 1), (i >> 1) & 1)) break;
                tc_fence_after_sync();
                const uint32_t v = v_lo + v_st * (M::kKV1 >> 4), p = s_at + (i & 1) * kTlKeys;
#pragma unroll
                for (int ks = 0; ks < kTlKeys / 16; ++ks) {
                    mma_ts(o_at, p + weight_column(ks), v + ks * (2048 >> 4), idesc_o, ks != 0 || i != 0);
                    if (SPLIT) mma_ts(o_at, p + weight_column(ks) + 16, v + ks * (2048 >> 4), idesc_o, true);
                }
                umma_commit(bar(kBarPV + qt * 2 + (i & 1)));
                umma_commit(bar(kBarVFree + v_st));
                if (++v_st == kTlStages) v_st = 0;
                if (i + 2 < n_tiles) scores(i + 2);
            }
            umma_commit(bar(kBarO + qt));
            (void)wait_phase(bar(kBarO + qt), 0);  // nothing is in flight when the tensor memory is released
        }
    }
    if (failed) kv8_report(P, H1B_ERR_TIMEOUT);
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    if (warp == kTlSoftmax + 8) { tc_fence_after_sync(); tmem_dealloc(W.tmem, 512); }
}

template <int D, int FMT, bool SPLIT>
cudaError_t launch_of(const Kv8Params &P, const Kv8Attn &A, cudaStream_t st) {
    constexpr int bytes = TlSmem<D>::kTotal;
    static Kv8Once once;
    const cudaError_t e = once.shared_memory(reinterpret_cast<const void *>(kv8_tiles_kernel<D, FMT, SPLIT>), bytes);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)A.tiles * (unsigned)P.hkv, 1, (unsigned)A.splits);
    return kv8_launch(kv8_tiles_kernel<D, FMT, SPLIT>, grid, kTlThreads, bytes, st, P, A);
}

}  // namespace

cudaError_t launch_kv8_tiles(const Kv8Params &P, const Kv8Attn &A, int d, int fmt, cudaStream_t st) {
    cudaError_t e;
#define H1B_KV8_TILES(D, F) (A.bf16 ? launch_of<D, F, false> : launch_of<D, F, true>)(P, A, st)
    if (d == 128) e = fmt == H1B_KV8_INT8 ? H1B_KV8_TILES(128, H1B_KV8_INT8) : H1B_KV8_TILES(128, H1B_KV8_E4M3);
    else e = fmt == H1B_KV8_INT8 ? H1B_KV8_TILES(64, H1B_KV8_INT8) : H1B_KV8_TILES(64, H1B_KV8_E4M3);
#undef H1B_KV8_TILES
    if (e != cudaSuccess || A.splits == 1) return e;
    return launch_kv8_join(P, A, d, 2 * kTlRows, kTlUnit, kTlMinBlocks, st);
}

}  // namespace h1b
