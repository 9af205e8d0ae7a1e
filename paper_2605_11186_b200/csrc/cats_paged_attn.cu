// Attention of one new token per sequence over the paged cache (include/cats.h: cats_paged_attention):
//   out[s][h] = sum_t softmax_t(q[s][h] . k[t][g] scale) v[t][g],   g = h / (n_heads / n_kv_heads)
//
// Bound by reading K and V once.  The query heads of a group share every row, so both products are matrix products whose small
// side is the group: S^T = K Q^T (16 rows x head_dim x 8 heads per instruction) and O^T = V^T P^T.  mma.sync takes the cache's
// rows as its 16-row operand straight from the registers they were loaded into, 16 bytes at a time: both products may run over
// channels and rows in any order, so a thread's 16 bytes are 8 (int8: 16) neighbouring channels of a row, and nothing of K or V
// passes through shared memory.  (tcgen05 would want a tile of 128 rows in shared memory for 8 columns of work; at the rate
// HBM delivers rows the 8-column products take a tenth of the issue slots.)
//
// One pass with a running maximum and sum per head and warp.  Probabilities enter the second product as two bf16 parts (16
// bits) over a bf16 cache.  An int8 cache's bytes are whole numbers in fp16, exact; the row's scale is part of the weight
// w = p scale_v, which enters as two fp16 parts (22 bits, and 11 at 2^-28 of the largest) with a running exponent of its own (fit).  Groups of up to four heads have room for both parts
// in the columns of one product: their queries stand there twice (48 sequences of up to 1500 rows, 40 heads over 40: 102 us; with a second
// product, as larger groups take it, 108; with one part of 11 bits 100, and outputs 4e-4 to 1e-3 from those of fp32 weights instead of 3e-5 to 2e-4).
//
// Work: the rows of every (sequence, head group) are cut into units of 4 tiles; all units in one line are dealt out evenly to the
// blocks, three per SM (12 warps with 8 KB of rows in flight each; HBM needs about 45 KB per SM).  A block of four warps takes
// its units sequence by sequence, the warps tile by tile, and joins its warps through shared memory.  What one block has of a
// head group that others have rows of goes to the workspace; the last to arrive (a counter) adds the parts in order of their rows,
// so the result does not depend on who that is.  More than kGroup parts are added in two steps.  No block ever waits for another.
// Measured: 64 sequences of up to 8191 rows, 32 heads over 8 in bf16 165 us (6.5 TB/s, the copy rate); one of 131071 in int8 54 us (5.1 TB/s; loads alone 50, 49
// without the scales); 48 of up to 1500, 40 heads over 40 in int8 102 us: loads alone 74 (of it 10 because 1920 head groups each start and end, at four
// times the length they run at the copy rate; 3 because pages of 24 rows break tiles, 2 for the scales), the rest a tile's chain of dependent
// instructions in three warps a scheduler, which leaves 46 % of the issue slots empty; one of 513 8.5 us, a chain of latencies; one of 131071 with 16 heads over 1 in
// bf16 34 us (2.0 TB/s): two blocks an SM, the same chain for two halves of the heads.
#include <atomic>

#include "cats_paged.cuh"

namespace cats {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kBlocksPerSm = 3, kMaxBlocks = 148 * kBlocksPerSm;
constexpr int kGroup = 24;          // parts added at once; kGroup^2 >= kMaxBlocks
constexpr int kMaxHeads = 16;       // query heads per block
constexpr int kMaxLen = INT32_MAX - 1023;       // a tile's rows behind the last one are still numbers
constexpr uint32_t kNoRow = 0xFFFFFFFFu;
static_assert(kGroup * kGroup >= kMaxBlocks, "two steps have to do");
constexpr float kLowest = -110.f;   // int8: of the weights' exponent `up`; 2^(15 - up) is a number

// Workspace: two part slots per block (a head group that began before its first unit, one that goes on behind its last), then counters.  A
// block is the first of at most one head group that goes on in the next, and a later one of at most one: a counter each.
constexpr size_t kSlotFloats = (size_t)kMaxHeads * (128 + 4);
typedef float4 Part;            // of a head: reference of its probabilities, exponent of its weights (int8), sum of its probabilities
struct Slots {
    float* values;
    int* counters;              // zero between calls
    __device__ __forceinline__ int* first(int block) const { return counters + block; }                       // parts that begin with a first block's
    __device__ __forceinline__ int* later(int block) const { return counters + kMaxBlocks + block; }          // with a later one's
    __device__ __forceinline__ int* groups(int block) const { return counters + 2 * kMaxBlocks + block; }     // sums of kGroup parts, by first block
    __device__ __forceinline__ float* o(int slot) const { return values + (size_t)slot * kSlotFloats; }
    __device__ __forceinline__ Part* part_of(int slot) const { return reinterpret_cast<Part*>(values + (size_t)slot * kSlotFloats + kMaxHeads * 128); }
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two bf16 with infinities as the largest number of their sign (NaN as some number)
__device__ __forceinline__ uint32_t finite(uint32_t a) {
    uint32_t r;
    asm("min.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(0x7F7F7F7Fu));
    return r;
}
__device__ __forceinline__ float lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
template <bool I8> __device__ __forceinline__ void mma(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (I8)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float f16_low(uint32_t a) {
    float x;
    asm("{ .reg .b16 l, h; mov.b32 {l, h}, %1; cvt.f32.f16 %0, l; }" : "=f"(x) : "r"(a));
    return x;
}
__device__ __forceinline__ float f16_high(uint32_t a) {
    float x;
    asm("{ .reg .b16 l, h; mov.b32 {l, h}, %1; cvt.f32.f16 %0, h; }" : "=f"(x) : "r"(a));
    return x;
}
// Bytes 0 and 1 (which = 0x4140) or 2 and 3 (0x4342) of w, each 128 more than the number it stands for, as fp16: 0x6400 + b is 1024 + b
__device__ __forceinline__ uint32_t f16_of_bytes(uint32_t w, uint32_t which) {
    uint32_t r, x = __byte_perm(w, 0x64646464u, which);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0x64806480u));
    return r;
}
__device__ __forceinline__ uint32_t word_of(const uint4& a, int i) { return i == 0 ? a.x : (i == 1 ? a.y : (i == 2 ? a.z : a.w)); }

// A run of units of one head group.
struct Segment {
    int s, kvh, head0, heads;       // sequence, head of the cache, query heads
    int t0, t1;                     // rows
    int unit, units;                // first unit, and units of the whole head group
    __device__ __forceinline__ int tiles(int first, int step) const { return first < t1 ? (t1 - first + step - 1) / step : 0; }
};

// BOTH (int8, groups of up to four): columns 4 to 7 of both products are those of 0 to 3 once more, and the second parts of their weights stand there.
template <int HD, bool I8, int NT, bool BOTH> struct Attn {
    static_assert(!BOTH || (I8 && NT == 1), "two parts of each weight, in the columns of one product");
    static constexpr int kTile = I8 || HD == 64 ? 32 : 16;      // rows per warp and step
    static constexpr int kUnit = kTile * kWarps;
    static constexpr int kBlk = kTile / 16;
    static constexpr int RB = HD * (I8 ? 1 : 2);            // bytes of a row
    static constexpr int RP = RB / 16, kPerCopy = 32 / RP;  // its 16-byte pieces, rows per copy of a warp
    static constexpr int kCopies = kTile / kPerCopy;
    static constexpr int KI = RB / 64;                      // 16-byte pieces of a K row per thread
    static constexpr int VI = I8 ? 1 : HD / 64;             // and of a V row (int8, 64 channels: 8 bytes)
    static constexpr int MT = HD / 16;                      // 16-channel tiles of O^T
    static constexpr int QV = HD / 32;                      // 16-byte pieces of the queries per thread and 8 heads
    static constexpr int kPad = HD + 4;
    // Half of a warp's ring: a tile of K, one of V, and (int8) a scale of each per row; or, after a segment, the warp's O.
    static constexpr int kV = kTile * RB, kScales = 2 * kV, kO = NT * 8 * kPad * 4;
    static constexpr int kStage = (kScales + (I8 ? 256 : 0)) > kO ? kScales + (I8 ? 256 : 0) : kO;
    struct Shared {
        uint8_t ring[kWarps][2][kStage];
        uint4 raw[NT * 8 * HD / 8];                         // the queries of the next segment, as they are
        uint4 q[2][NT][QV][32];                             // and as the second operand of K Q^T, of this segment and the next
        float qf[2][NT * 8];                                // factors of the scores
        Part part[kWarps][NT * 8];
        int o_at[kWarps];                                   // which half of its ring a warp's O is in
        long long total, before;        // units of all sequences, and of those in front of `seq`
        int seq, last;
        long long warp_sum[kWarps];
    };

    const PagedDev& c;
    const PagedAttn& a;
    Shared& sh;
    const int lane, warp, g, j;
    float acc[NT][MT][4];
    float m[NT][2], l[NT][2], qf[NT][2];       // heads 2j and 2j + 1 of each 8: reference, sum, factor of the scores
    float up[NT][2], times[NT][2];             // int8: the weights' exponent and 2^(15 - up)

    __device__ __forceinline__ Attn(const PagedDev& c_, const PagedAttn& a_, Shared& s_)
        : c(c_), a(a_), sh(s_), lane(threadIdx.x & 31), warp(threadIdx.x >> 5), g((threadIdx.x & 31) >> 2), j(threadIdx.x & 3) {}

    // A row of a tile per lane: where it lies; kNoRow: nowhere, zeros are taken for it.
    struct Row {
        uint32_t at;
        uint32_t s;
    };
    __device__ __forceinline__ Row row_of(int s, int t, int t1) const {
        Row r = {kNoRow, 0};
        PagedDev::Row p;
        if ((kTile == 32 || lane < kTile) && t + lane < t1) {
            if (c.locate(s, t + lane, p)) r = {p.at, p.s};
            else report(a.d_status, CATS_ERR_INVALID_ARG);
        }
        return r;
    }
    template <int N> static __device__ __forceinline__ void copy(uint32_t to, const void* from, bool there) {
        if (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(N), "r"(there ? N : 0) : "memory");
    }
    // Where piece `piece` of row `row` of a tile lies.  Rows follow each other; the pieces within 128 bytes change places so that neither the
    // reads of K (rows 2p, 2p + 1 and four pieces at a time) nor those of V (rows 0, 2, 4, 6 and two pieces) meet in a bank.
    static __device__ __forceinline__ int k_at(int row, int piece) { return row * RB + ((RB >= 128 ? piece ^ ((row & 1) << 2) : piece) << 4); }
    static __device__ __forceinline__ int v_at(int row, int piece) {
        const int x = row * RP + piece;
        return (x ^ (((row >> 1) & 3) << 1)) << 4;
    }
    // Requests the tile whose rows are `row`: 512 bytes of whole rows per instruction.  (Rows in pieces of 64 bytes, as the threads
    // use them, asked L2 for every line twice: 4.85 instead of 6.05 TB/s.)
    __device__ __forceinline__ void request(uint32_t stage, const Row& row, int kvh) const {
        const uint8_t* const k = c.k + (size_t)kvh * c.head16 * 16 + (lane % RP) * 16;
        const uint8_t* const v = c.v + (size_t)kvh * c.head16 * 16 + (lane % RP) * 16;
        if (I8) {
            copy<4>(stage + kScales + lane * 4, c.ks + (size_t)kvh * c.s_head + row.s, row.at != kNoRow);
            copy<4>(stage + kScales + 128 + lane * 4, c.vs + (size_t)kvh * c.s_head + row.s, row.at != kNoRow);
        }
        const uint32_t at0 = __shfl_sync(0xffffffffu, row.at, 0);
        if (__all_sync(0xffffffffu, (kTile < 32 && lane >= kTile) || (row.at != kNoRow && lies_behind(at0, row.at, lane * RP)))) {      // rows that follow each other
#pragma unroll
            for (int n = 0; n < kCopies; ++n) {
                const int r = n * kPerCopy + lane / RP;
                copy<16>(stage + k_at(r, lane % RP), k + (size_t)at0 * 16 + lane / RP * RB + n * 512, true);
                copy<16>(stage + kV + v_at(r, lane % RP), v + (size_t)at0 * 16 + lane / RP * RB + n * 512, true);
            }
        } else {
#pragma unroll
            for (int n = 0; n < kCopies; ++n) {
                const int r = n * kPerCopy + lane / RP;
                const uint32_t at = __shfl_sync(0xffffffffu, row.at, r);
                copy<16>(stage + k_at(r, lane % RP), k + (at != kNoRow ? (size_t)at * 16 : 0), at != kNoRow);
                copy<16>(stage + kV + v_at(r, lane % RP), v + (at != kNoRow ? (size_t)at * 16 : 0), at != kNoRow);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // Requests the queries of a segment.
    __device__ __forceinline__ void request_q(const Segment& g) const {
        const uint16_t* const q = a.q + g.s * a.ldq + (size_t)g.head0 * HD;
        for (int i = threadIdx.x; i < NT * 8 * HD / 8; i += kThreads) {
            const bool there = i < g.heads * (HD / 8);
            copy<16>(smem_u32(&sh.raw[i]), q + (there ? i * 8 : 0), there);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    static __device__ __forceinline__ uint4 lds16(uint32_t p) {
        uint4 x;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(p) : "memory");
        return x;
    }
    static __device__ __forceinline__ float lds_float(uint32_t p) {
        float x;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(p) : "memory");
        return x;
    }
    __device__ __forceinline__ uint4 k_piece(uint32_t stage, int b, int i) const { return lds16(stage + k_at(b * 8 + g, i * 4 + j)); }
    __device__ __forceinline__ uint4 v_piece(uint32_t stage, int n, int i) const {
        const int row = (n >> 2) * 16 + ((n & 2) ? 8 : 0) + 2 * j + (n & 1);
        if (!I8 || HD == 128) return lds16(stage + kV + v_at(row, i * 8 + g));
        uint4 x = make_uint4(0, 0, 0, 0);
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(stage + kV + v_at(row, g >> 1) + (g & 1) * 8) : "memory");
        return x;
    }

    // The queries that have arrived as the second operand of K Q^T, by one warp: thread (g, j) makes of head g the channels that thread
    // (any, j) holds of a K row.  int8: as fp16, times a power of two that brings the head's largest to 2^14: exact down to 2^-28 of it.
    __device__ __forceinline__ void make_q(int to) {
        const float base = a.scale * 1.4426950408889634f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            uint4 x[QV];
#pragma unroll
            for (int i = 0; i < QV; ++i) x[i] = sh.raw[(nt * 8 + (BOTH ? g & 3 : g)) * (HD / 8) + (I8 ? (i >> 1) * 8 + j * 2 + (i & 1) : i * 4 + j)];
            float mine = base;
            if (I8) {
                uint32_t mx = 0;
#pragma unroll
                for (int i = 0; i < QV; ++i)
#pragma unroll
                    for (int w = 0; w < 4; ++w) mx = max(mx, max((word_of(x[i], w) << 16) & 0x7FFF0000u, word_of(x[i], w) & 0x7FFF0000u));
                mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                const int e = (int)(mx >> 23);                      // biased exponent; zero and subnormals, infinities and NaN: factor 1
                const int up = e > 0 && e < 255 ? 141 - e : 0;      // e - 127 + up = 14
                // 2^up in two factors: up reaches 140
                const float f0 = __int_as_float((127 + up / 2) << 23), f1 = __int_as_float((127 + up - up / 2) << 23);
#pragma unroll
                for (int i = 0; i < QV; ++i) {
                    uint32_t o[4];
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t y = word_of(x[i], w);
                        o[w] = pack_f16x2(__uint_as_float(y << 16) * f0 * f1, __uint_as_float(y & 0xFFFF0000u) * f0 * f1);
                    }
                    x[i] = make_uint4(o[0], o[1], o[2], o[3]);
                }
                mine = base / f0 / f1;
            }
#pragma unroll
            for (int i = 0; i < QV; ++i) sh.q[to][nt][i][lane] = x[i];
            if (j == 0) sh.qf[to][nt * 8 + g] = mine;
        }
    }

    static __device__ __forceinline__ float over_rows(float x) {       // the largest of the lanes that have rows of the same heads
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
        return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
    }
    __device__ __forceinline__ void rescale(const float (&keep)[NT][2]) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[nt][t][e] *= keep[nt][e & 1];
    }
    // int8.  A probability is relative to 2^m, m a whole number a little above the largest score so far; a weight p scale_v has a factor of its own, 2^(15 - up).
    // (One reference, the maximum of score + log2 scale_v, for both: probabilities of rows with a small scale, or next to a row with a
    // large one, leave the range of fp32, and the sum loses them.)  O^T is in units of 2^(m + up - 15).
    // The largest weight when `up` is set becomes 2^14 to 2^15: what is 2^-28 of it is still a normal number of fp16.  Most tiles change neither m nor
    // `up`: their scores are below m, and the largest score's probability times the largest scale is a number of fp16, so the weights are.
    __device__ __forceinline__ void fit(const float (&s)[NT][kBlk][4], const float (&sv)[kBlk][2], bool first) {
        float x[NT][2], size = 0.f;
        bool over = false;
#pragma unroll
        for (int b = 0; b < kBlk; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) size = fmaxf(size, fabsf(sv[b][h]));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                x[nt][e] = s[nt][0][e];
#pragma unroll
                for (int b = 0; b < kBlk; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h) x[nt][e] = fmaxf(x[nt][e], s[nt][b][h * 2 + e]);
                over |= x[nt][e] > m[nt][e] || size * times[nt][e] * ex2(x[nt][e] - m[nt][e]) > 65504.f;
            }
        if (!__any_sync(0xffffffffu, over)) return;
        // the largest score and the largest score + log2 scale_v, the second relative to the first, so that large scores leave the logarithms their bits
        float lg[kBlk][2], keep[NT][2];
        bool changed = false;
#pragma unroll
        for (int b = 0; b < kBlk; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) lg[b][h] = lg2(fabsf(sv[b][h]));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = x[nt][e], most = (s[nt][0][e] - top) + lg[0][0];
#pragma unroll
                for (int b = 0; b < kBlk; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h) most = fmaxf(most, (s[nt][b][h * 2 + e] - top) + lg[b][h]);
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    const float x1 = __shfl_xor_sync(0xffffffffu, top, d), z1 = __shfl_xor_sync(0xffffffffu, most, d), larger = fmaxf(top, x1);
                    most = fmaxf(most + (top - larger), z1 + (x1 - larger));
                    top = larger;
                }
                const float to = top > m[nt][e] ? ceilf(top) + 2.f : m[nt][e];
                const float by = m[nt][e] == to ? 0.f : m[nt][e] - to, from = up[nt][e] + by, need = most + (top - to);
                const float with = fmaxf(need > from + 0.99f ? ceilf(need) : from, kLowest);
                keep[nt][e] = ex2(from - with);
                changed |= with != from;
                l[nt][e] *= ex2(by);
                up[nt][e] = with;
                times[nt][e] = ex2(15.f - with);
                m[nt][e] = to;
            }
        if (!first && __any_sync(0xffffffffu, changed)) rescale(keep);
    }

    // One tile: scores, weights, O^T.  left: rows of the sequence from the tile's first on; first: nothing has been added to O^T yet.
    __device__ __forceinline__ void step(uint32_t stage, int left, int parity, bool first) {
        float s[NT][kBlk][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int b = 0; b < kBlk; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nt][b][e] = 0.f;
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            uint4 kr[kBlk * 2];
#pragma unroll
            for (int b = 0; b < kBlk * 2; ++b) kr[b] = k_piece(stage, b, i);
            if (I8) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
#pragma unroll
                    for (int b = 0; b < kBlk; ++b) {
                        const uint32_t x = word_of(kr[2 * b], w) ^ 0x80808080u, y = word_of(kr[2 * b + 1], w) ^ 0x80808080u;
                        const uint32_t a0 = f16_of_bytes(x, 0x4140), a1 = f16_of_bytes(y, 0x4140), a2 = f16_of_bytes(x, 0x4342), a3 = f16_of_bytes(y, 0x4342);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint4 q = sh.q[parity][nt][i * 2 + (w >> 1)][lane];
                            mma<I8>(s[nt][b], a0, a1, a2, a3, w & 1 ? q.z : q.x, w & 1 ? q.w : q.y);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint4 q = sh.q[parity][nt][i][lane];
#pragma unroll
                    for (int b = 0; b < kBlk; ++b) {
                        mma<I8>(s[nt][b], kr[2 * b].x, kr[2 * b + 1].x, kr[2 * b].y, kr[2 * b + 1].y, q.x, q.y);
                        mma<I8>(s[nt][b], kr[2 * b].z, kr[2 * b + 1].z, kr[2 * b].w, kr[2 * b + 1].w, q.z, q.w);
                    }
                }
            }
        }
        // scores in log2
        float vs[kBlk][2];
#pragma unroll
        for (int b = 0; b < kBlk; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = b * 16 + h * 8 + g;
                const float none = row < left ? 0.f : -INFINITY;
                float ks = 1.f;
                vs[b][h] = 1.f;
                if (I8) {
                    ks = lds_float(stage + kScales + row * 4);
                    vs[b][h] = lds_float(stage + kScales + 128 + row * 4);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) s[nt][b][h * 2 + e] = s[nt][b][h * 2 + e] * qf[nt][e] * ks + none;
            }
        // weights, turned into the second operand of V^T P^T: heads along the lanes' groups, rows along a thread
        uint32_t p[NT][kBlk][2], lo[NT][kBlk][2];
        if constexpr (I8) {
            fit(s, vs, first);
            const float second = j < 2 ? 0.f : -1.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float m0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], m1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1], f0 = times[nt][0], f1 = times[nt][1];
#pragma unroll
                for (int b = 0; b < kBlk; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float p0 = ex2(s[nt][b][h * 2] - m0), p1 = ex2(s[nt][b][h * 2 + 1] - m1);
                        l[nt][0] += p0;
                        l[nt][1] += p1;
                        const float w0 = p0 * vs[b][h] * f0, w1 = p1 * vs[b][h] * f1;
                        const uint32_t hi = pack_f16x2(w0, w1);
                        if (BOTH) {
                            p[nt][b][h] = transpose8x8(pack_f16x2(fmaf(f16_low(hi), second, w0), fmaf(f16_high(hi), second, w1)));
                        } else {
                            p[nt][b][h] = transpose8x8(hi);
                            lo[nt][b][h] = transpose8x8(pack_f16x2(w0 - f16_low(hi), w1 - f16_high(hi)));
                        }
                    }
            }
        } else {
            bool moved = false;
            float keep[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = s[nt][0][e];
#pragma unroll
                    for (int b = 0; b < kBlk; ++b)
#pragma unroll
                        for (int h = 0; h < 2; ++h) x = fmaxf(x, s[nt][b][h * 2 + e]);
                    x = fmaxf(over_rows(x), m[nt][e]);
                    keep[nt][e] = 1.f;
                    if (x != m[nt][e]) {
                        keep[nt][e] = ex2(m[nt][e] - x);
                        m[nt][e] = x;
                        moved = true;
                    }
                }
            if (__any_sync(0xffffffffu, moved)) {
                rescale(keep);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    l[nt][0] *= keep[nt][0];
                    l[nt][1] *= keep[nt][1];
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float m0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], m1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
#pragma unroll
                for (int b = 0; b < kBlk; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float p0 = ex2(s[nt][b][h * 2] - m0), p1 = ex2(s[nt][b][h * 2 + 1] - m1);
                        l[nt][0] += p0;
                        l[nt][1] += p1;
                        const uint32_t hi = pack_bf16x2(p0, p1);
                        lo[nt][b][h] = transpose8x8(pack_bf16x2(p0 - __uint_as_float(hi << 16), p1 - __uint_as_float(hi & 0xFFFF0000u)));
                        p[nt][b][h] = transpose8x8(hi);
                    }
            }
        }
#pragma unroll
        for (int b = 0; b < kBlk; ++b) {
            if (I8) {
                uint4 vr[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) vr[n] = v_piece(stage, b * 4 + n, 0);
#pragma unroll
                for (int w = 0; w < HD / 32; ++w) {
                    uint32_t x[2], y[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t t0 = word_of(vr[h * 2], w) ^ 0x80808080u, t1 = word_of(vr[h * 2 + 1], w) ^ 0x80808080u;
                        x[h] = __byte_perm(t0, t1, 0x5140);
                        y[h] = __byte_perm(t0, t1, 0x7362);
                    }
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t z0 = half ? y[0] : x[0], z1 = half ? y[1] : x[1];
                        const uint32_t a0 = f16_of_bytes(z0, 0x4140), a1 = f16_of_bytes(z0, 0x4342), a2 = f16_of_bytes(z1, 0x4140), a3 = f16_of_bytes(z1, 0x4342);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma<I8>(acc[nt][w * 2 + half], a0, a1, a2, a3, p[nt][b][0], p[nt][b][1]);
                            if (!BOTH) mma<I8>(acc[nt][w * 2 + half], a0, a1, a2, a3, lo[nt][b][0], lo[nt][b][1]);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < VI; ++i) {
                    uint4 vr[4];
#pragma unroll
                    for (int n = 0; n < 4; ++n) vr[n] = v_piece(stage, b * 4 + n, i);
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t t0 = word_of(vr[0], w), t1 = word_of(vr[1], w), t2 = word_of(vr[2], w), t3 = word_of(vr[3], w);
                        const uint32_t a0 = __byte_perm(t0, t1, 0x5410), a1 = __byte_perm(t0, t1, 0x7632), a2 = __byte_perm(t2, t3, 0x5410), a3 = __byte_perm(t2, t3, 0x7632);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {          // a second part may be 0 or negative, and infinities have had their weight from the first
                            mma<I8>(acc[nt][i * 4 + w], a0, a1, a2, a3, p[nt][b][0], p[nt][b][1]);
                            mma<I8>(acc[nt][i * 4 + w], finite(a0), finite(a1), finite(a2), finite(a3), lo[nt][b][0], lo[nt][b][1]);
                        }
                    }
                }
            }
        }
    }
    // Channel of row g of tile t of O^T; row g + 8 is the next one.
    __device__ __forceinline__ int channel(int t) const { return I8 ? g * (HD / 8) + 2 * t : (t >> 2) * 64 + g * 8 + (t & 3) * 2; }

    // What the block has of a segment, to sh.ml and the warps' rings, one entry per warp that had rows; returns how many.  One tile is always on
    // its way while another is worked on, the next segment's first behind this one's last; where the rows of the tile to be
    // requested next lie is looked up a step ahead.
    int used;                   // half of the ring that is worked on
    bool pending;               // whether the other half's tile has been requested
    __device__ __forceinline__ int segment(const Segment& g0, const Segment& g1, bool more, int parity) {
        const int first = g0.t0 + warp * kTile, tiles = g0.tiles(first, kUnit), first1 = g1.t0 + warp * kTile;
        const bool next_has = more && first1 < g1.t1;
        const uint32_t ring = smem_u32(sh.ring[warp]);
        if (!pending && tiles > 0) request(ring + (used ^ 1) * kStage, row_of(g0.s, first, g0.t1), g0.kvh);
        pending = tiles > 0;
        Row next;               // of the tile behind the pending one
        if (tiles > 1) next = row_of(g0.s, first + kUnit, g0.t1);
        else if (next_has) next = row_of(g1.s, first1, g1.t1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                m[nt][e] = -INFINITY;
                l[nt][e] = 0.f;
                up[nt][e] = I8 ? kLowest : 0.f;
                times[nt][e] = ex2(15.f - kLowest);
                qf[nt][e] = sh.qf[parity][nt * 8 + 2 * j + e];
            }
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[nt][t][e] = 0.f;
        }
        if (more) request_q(g1);
        for (int i = 0; i < tiles; ++i) {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncwarp();       // also: all lanes are done with the half that is filled next
            used ^= 1;
            pending = i + 1 < tiles || next_has;
            if (pending) {
                request(ring + (used ^ 1) * kStage, next, i + 1 < tiles ? g0.kvh : g1.kvh);
                if (i + 2 < tiles) next = row_of(g0.s, first + (i + 2) * kUnit, g0.t1);
                else if (i + 2 == tiles && next_has) next = row_of(g1.s, first1, g1.t1);
            }
            step(ring + used * kStage, g0.t1 - (first + i * kUnit), parity, i == 0);
        }
        const int active = min(kWarps, (g0.t1 - g0.t0 + kTile - 1) / kTile);
        if (warp < active) {
            float* const o = reinterpret_cast<float*>(sh.ring[warp][used]);
            if (lane == 0) sh.o_at[warp] = used;
            __syncwarp();
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], d);
                if (g == 0) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) sh.part[warp][nt * 8 + 2 * j + e] = make_float4(m[nt][e], up[nt][e], l[nt][e], 0.f);
                }
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    *reinterpret_cast<float2*>(o + (nt * 8 + 2 * j) * kPad + channel(t)) = make_float2(acc[nt][t][0], acc[nt][t][2]);
                    *reinterpret_cast<float2*>(o + (nt * 8 + 2 * j + 1) * kPad + channel(t)) = make_float2(acc[nt][t][1], acc[nt][t][3]);
                }
            }
        }
        // the next segment's queries; a tile requested behind them may still be on its way
        if (pending) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        if (more && warp == kWarps - 1) make_q(parity ^ 1);
        return active;
    }

    // Parts joined so far: where their references lie and what they add up to.  Values of a part are in units of 2^(m + up).
    struct Sum {
        float m = -INFINITY, up = -INFINITY, l = 0.f;
        float4 x = make_float4(0, 0, 0, 0);
        // To the references of these parts too
        template <int N> __device__ __forceinline__ void raise(const Part (&p)[N], int n) {
            float to = m;
#pragma unroll
            for (int k = 0; k < N; ++k) if (k < n) to = fmaxf(to, p[k].x);
            const float zero = to == -INFINITY ? 0.f : to, by = ex2(m - zero);
            l *= by;
            if (I8) {
                const float from = up + (m - zero);
                float with = from;
#pragma unroll
                for (int k = 0; k < N; ++k) if (k < n) with = fmaxf(with, p[k].y + (p[k].x - zero));
                up = with;
                scale(ex2(from - (with == -INFINITY ? 0.f : with)));
            } else {
                scale(by);
            }
            m = to;
        }
        __device__ __forceinline__ void scale(float f) { x.x *= f; x.y *= f; x.z *= f; x.w *= f; }
        __device__ __forceinline__ void add(const Part& p, const float4& o) {
            const float by = p.x - (m == -INFINITY ? 0.f : m), f = ex2(by), fx = I8 ? ex2(p.y + by - (up == -INFINITY ? 0.f : up)) : f;
            l = fmaf(p.z, f, l);
            x.x = fmaf(o.x, fx, x.x); x.y = fmaf(o.y, fx, x.y); x.z = fmaf(o.z, fx, x.z); x.w = fmaf(o.w, fx, x.w);
        }
    };
    __device__ __forceinline__ void store_out(int s, int head, int ch, Sum& r, bool empty) {
        r.scale(1.f / r.l);
        if (I8) r.scale(ex2(r.up - 15.f));          // apart: the product may lie below fp32
        uint32_t* const o = reinterpret_cast<uint32_t*>(a.out + s * a.ldo + (size_t)head * HD + ch);
        o[0] = empty ? 0u : pack_bf16x2(r.x.x, r.x.y);
        o[1] = empty ? 0u : pack_bf16x2(r.x.z, r.x.w);
    }

    // The block's warps joined: to `slot`, or (slot < 0) to the output.
    __device__ __forceinline__ void join(int s, int head0, int heads, int active, const Slots& w, int slot) {
        for (int i = threadIdx.x; i < heads * (HD / 4); i += kThreads) {
            const int h = i / (HD / 4), ch = (i % (HD / 4)) * 4;
            Part p[kWarps];
#pragma unroll
            for (int k = 0; k < kWarps; ++k) p[k] = sh.part[k][h];      // of the active ones
            Sum r;
            r.raise(p, active);
#pragma unroll
            for (int k = 0; k < kWarps; ++k)
                if (k < active) {
                    const float* const o = reinterpret_cast<const float*>(sh.ring[k][sh.o_at[k]]) + h * kPad + ch;
                    float4 x = *reinterpret_cast<const float4*>(o);
                    if (BOTH) {
                        const float4 y = *reinterpret_cast<const float4*>(o + 4 * kPad);
                        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
                    }
                    r.add(p[k], x);
                }
            if (slot < 0) {
                store_out(s, head0 + h, ch, r, active == 0);
            } else {
                *reinterpret_cast<float4*>(w.o(slot) + h * HD + ch) = r.x;
                if (ch == 0) w.part_of(slot)[h] = make_float4(r.m, r.up, r.l, 0.f);
            }
        }
        __syncthreads();            // the rings are free
    }

    // The slot of part k of a head group whose first block is `first`.
    static __device__ __forceinline__ int slot_of(int first, int k) { return 2 * (first + k) + (k == 0 ? 1 : 0); }
    // Parts p0, p0 + step, ... (n of them) of a head group added in this order: to slot `to`, or (to < 0) to the output.  References, sums and values of
    // kAtOnce parts come in one trip.
    __device__ __forceinline__ void add_parts(const Segment& g0, int first, int p0, int step, int n, const Slots& w, int to) {
        constexpr int kAtOnce = 6;
        // A sum goes to the slot of its first part: a head's threads, which are of one warp, have all read that part's reference before one of them
        // writes the sum's.  So all lanes go through the loop together, those without a channel with another's.
        const int n_all = g0.heads * (HD / 4);
        for (int i0 = warp * 32; i0 < n_all; i0 += kThreads) {
            const bool mine = i0 + lane < n_all;
            const int i = mine ? i0 + lane : n_all - 1, h = i / (HD / 4), ch = (i % (HD / 4)) * 4;
            Sum r;
            for (int k0 = 0; k0 < n; k0 += kAtOnce) {
                Part p[kAtOnce];
                float4 o[kAtOnce];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const int slot = slot_of(first, p0 + min(k0 + k, n - 1) * step);
                    p[k] = __ldcg(w.part_of(slot) + h);
                    o[k] = __ldcg(reinterpret_cast<const float4*>(w.o(slot) + h * HD + ch));
                }
                r.raise(p, kAtOnce);    // those behind the last are the last again
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k)
                    if (k0 + k < n) r.add(p[k], o[k]);
            }
            __syncwarp();
            if (!mine) continue;
            if (to < 0) {
                store_out(g0.s, g0.head0 + h, ch, r, false);
            } else {
                *reinterpret_cast<float4*>(w.o(to) + h * HD + ch) = r.x;
                if (ch == 0) w.part_of(to)[h] = make_float4(r.m, r.up, r.l, 0.f);
            }
        }
    }
    // Whether this block is the last of n to come here; it then sees what the others wrote, and the counter is zero again.
    __device__ __forceinline__ bool arrive(int* counter, int n) {
        __syncthreads();
        if (threadIdx.x == 0) {
            int before;         // releases what the block has written (the barrier in front orders it) and acquires what the others have
            asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
            const bool last = before == n - 1;
            if (last) *counter = 0;
            sh.last = last;
        }
        __syncthreads();
        return sh.last != 0;
    }

    __device__ __forceinline__ int length(int s) const {
        const int asked = a.len[s];
        const long long most = min((long long)c.width * c.page_size, (long long)kMaxLen);
        if (asked > most) report(a.d_status, CATS_ERR_INVALID_ARG);
        return (int)min((long long)max(asked, 0), most);
    }
    static __device__ __forceinline__ long long quotient(long long a, long long b) {      // 64-bit division is a hundred instructions
        return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
    }
    static __device__ __forceinline__ long long share_of(long long block, long long units, long long blocks) { return quotient(block * units, blocks); }
    static __device__ __forceinline__ int units_of(int len) { return len > 0 ? (len - 1) / kUnit + 1 : 1; }

    // The sequence that unit `first(total)` lies in, to sh.seq; sh.before: units per head group of those in front of it, sh.total: of all.
    template <typename F> __device__ __forceinline__ void find(int groups, F first) {
        if (c.n_seqs <= 32) {               // a warp's lanes
            const int n = lane < c.n_seqs ? units_of(length(lane)) : 0;
            long long upto = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long t = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += t;
            }
            const long long total = __shfl_sync(0xffffffffu, upto, 31), want = first(total * groups);
            if (warp == 0) {
                if (want >= (upto - n) * groups && want < upto * groups) {
                    sh.seq = lane;
                    sh.before = upto - n;
                }
                if (lane == 0) sh.total = total * groups;
            }
            __syncthreads();
            return;
        }
        const int each = (c.n_seqs + kThreads - 1) / kThreads, s0 = min(c.n_seqs, (int)threadIdx.x * each), s1 = min(c.n_seqs, s0 + each);
        long long mine = 0;
        for (int s = s0; s < s1; ++s) mine += units_of(length(s));
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += t;
        }
        if (lane == 31) sh.warp_sum[warp] = upto;
        __syncthreads();
        long long total = 0;
        for (int k = 0; k < kWarps; ++k) {
            if (k < warp) upto += sh.warp_sum[k];
            total += sh.warp_sum[k];
        }
        long long before = upto - mine;
        const long long want = first(total * groups);
        if (want >= before * groups && want < upto * groups) {
            int s = s0;
            for (;; ++s) {
                const int n = units_of(length(s));
                if (want < (before + n) * groups) break;
                before += n;
            }
            sh.seq = s;
            sh.before = before;
        }
        if (threadIdx.x == 0) sh.total = total * groups;
        __syncthreads();
    }

    __device__ __forceinline__ void run() {
        const int per_kv = a.n_heads / c.n_kv, chunks = (per_kv + NT * 8 - 1) / (NT * 8), groups = c.n_kv * chunks;
        const int me = blockIdx.x;
        // block b of the first min(blocks, units) has units [b units / blocks, (b + 1) units / blocks)
        auto blocks_for = [&](long long units) { return (long long)min((long long)gridDim.x, units); };
        find(groups, [&](long long units) {
            const long long n = blocks_for(units);
            return me < n ? share_of(me, units, n) : -1;
        });
        const long long units = sh.total, n_blocks = blocks_for(units);
        if (me >= n_blocks) return;
        long long u = share_of(me, units, n_blocks);
        const long long u_end = share_of(me + 1, units, n_blocks);
        auto block_of = [&](long long unit) { return (int)quotient((unit + 1) * n_blocks - 1, units); };
        const Slots w = {(float*)a.ws, (int*)((float*)a.ws + 2 * kMaxBlocks * kSlotFloats)};
        // the sequence at hand, its length and the next one's, and how far the segments have come in it
        int s = sh.seq, len = length(s), len1 = s + 1 < c.n_seqs ? length(s + 1) : 0, n = units_of(len);
        const long long from = u - sh.before * groups;
        const int group0 = from >> 32 ? (int)(from / n) : (int)((uint32_t)from / (uint32_t)n);
        int kvh = group0 / chunks, chunk = group0 % chunks, unit = (int)(u - sh.before * groups - (long long)group0 * n);
        auto next_segment = [&] {                    // from unit u on
            if (unit == n) {
                unit = 0;
                if (++chunk == chunks) {
                    chunk = 0;
                    if (++kvh == c.n_kv) {
                        kvh = 0;
                        ++s;
                        len = len1;
                        len1 = s + 1 < c.n_seqs ? length(s + 1) : 0;
                        n = units_of(len);
                    }
                }
            }
            Segment g;
            g.s = s;
            g.kvh = kvh;
            g.head0 = kvh * per_kv + chunk * NT * 8;
            g.heads = min(NT * 8, per_kv - chunk * NT * 8);
            g.unit = unit;
            g.units = n;
            const int mine = (int)min((long long)(n - unit), u_end - u);
            g.t0 = unit * kUnit;
            g.t1 = (int)min((long long)len, (long long)(unit + mine) * kUnit);
            u += mine;
            unit += mine;
            return g;
        };
        Segment now = next_segment();
        long long at = share_of(me, units, n_blocks);        // its first unit
        used = 1;
        pending = false;
        request_q(now);
        const int first_row = now.t0 + warp * kTile;
        if (first_row < now.t1) {
            request(smem_u32(sh.ring[warp]), row_of(now.s, first_row, now.t1), now.kvh);
            pending = true;
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        __syncthreads();
        if (warp == kWarps - 1) make_q(0);
        __syncthreads();
        for (int parity = 0;; parity ^= 1) {
            const long long end = u;
            const bool more = end < u_end;
            Segment next = now;
            if (more) next = next_segment();
            const int active = segment(now, next, more, parity);
            if (end - at == now.units) {
                join(now.s, now.head0, now.heads, active, w, -1);
            } else {
                // blocks first .. last have rows of this head group; the first of them in its second slot
                const int first = block_of(at - now.unit), last = block_of(at - now.unit + now.units - 1), parts = last - first + 1;
                join(now.s, now.head0, now.heads, active, w, slot_of(first, me - first));
                // up to kGroup parts are added at once, more in groups of so many and then the groups
                const bool grouped = parts > kGroup;
                const int p0 = grouped ? (me - first) / kGroup * kGroup : 0;
                for (int level = 0; level < 2; ++level) {
                    const bool top = level == 1 || !grouped;
                    const int n = !grouped ? parts : (level == 0 ? min(kGroup, parts - p0) : (parts + kGroup - 1) / kGroup);
                    if (!arrive(level == 1 ? w.groups(first) : (p0 == 0 ? w.first(first) : w.later(first + p0)), n)) break;
                    add_parts(now, first, level == 0 ? p0 : 0, level == 0 ? 1 : kGroup, n, w, top ? -1 : slot_of(first, p0));
                    if (top) break;
                }
            }
            if (!more) break;
            now = next;
            at = end;
        }
    }
};

template <int HD, bool I8, int NT, bool BOTH> __global__ void __launch_bounds__(kThreads, NT == 1 ? kBlocksPerSm : 2) k_paged_attn(const __grid_constant__ PagedDev c, const __grid_constant__ PagedAttn a) {
    extern __shared__ __align__(16) uint8_t smem[];
    typename Attn<HD, I8, NT, BOTH>::Shared& sh = *reinterpret_cast<typename Attn<HD, I8, NT, BOTH>::Shared*>(smem);
    pdl_launch_dependents();
    pdl_wait();
    Attn<HD, I8, NT, BOTH>(c, a, sh).run();
}

template <int HD, bool I8, int NT, bool BOTH> cudaError_t launch_k(const PagedDev& c, const PagedAttn& a, cudaStream_t st) {
    typedef Attn<HD, I8, NT, BOTH> A;
    const long long per_kv = a.n_heads / c.n_kv, groups = c.n_kv * ((per_kv + NT * 8 - 1) / (NT * 8));
    const long long most = (long long)c.width * c.page_size, units = (most - 1) / A::kUnit + 1;
    const long long fit = NT == 1 ? kMaxBlocks : 148 * 2, blocks = units >= fit ? fit : min(fit, units * groups * c.n_seqs);
    constexpr size_t smem = sizeof(typename A::Shared);
    static_assert((smem + 1024) * (NT == 1 ? kBlocksPerSm : 2) <= 228 * 1024, "the blocks of an SM share its memory");
    static std::atomic<uint64_t> known{0};           // devices whose attribute is set
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!(known.load(std::memory_order_acquire) >> dev & 1)) {
        e = cudaFuncSetAttribute(k_paged_attn<HD, I8, NT, BOTH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        known.fetch_or((uint64_t)1 << dev, std::memory_order_release);
    }
    return launch_i8(k_paged_attn<HD, I8, NT, BOTH>, dim3((unsigned)blocks), dim3(kThreads), smem, st, c, a);
}

}  // namespace

size_t paged_attn_workspace(int, int, int, int) { return 2 * kMaxBlocks * kSlotFloats * 4 + 3 * kMaxBlocks * sizeof(int); }

template <int HD> cudaError_t launch_hd(const PagedDev& c, const PagedAttn& a, int i8, cudaStream_t st) {
    // eight heads at a time while the group has no more: the accumulators of sixteen leave registers for half the rows in flight
    const int group = a.n_heads / c.n_kv;
    if (i8) return group <= 4 ? launch_k<HD, true, 1, true>(c, a, st) : (group <= 8 ? launch_k<HD, true, 1, false>(c, a, st) : launch_k<HD, true, 2, false>(c, a, st));
    return group <= 8 ? launch_k<HD, false, 1, false>(c, a, st) : launch_k<HD, false, 2, false>(c, a, st);
}

cudaError_t launch_paged_attn(const PagedDev& c, const PagedAttn& a, int i8, int hd, cudaStream_t st) {
    return hd == 128 ? launch_hd<128>(c, a, i8, st) : launch_hd<64>(c, a, i8, st);
}

}  // namespace cats
