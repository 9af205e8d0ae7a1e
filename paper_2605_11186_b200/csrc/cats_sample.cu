// One token per row of logits (include/cats.h: cats_sample).
//
// Tokens are ordered by falling logit, equal ones by rising index; top-k, top-p and min-p each keep a run from the front of
// that order, so what is kept is: every token whose logit is above a threshold, and the first few (by index) of those at it.
// w = exp((x - max) / T) is a whole multiple of 2^-44, taken from an fp64 exponential: the sums are exact 64-bit integers, the same in any
// order, and so are all decisions made from them.  (vocab <= 2^18, so no sum reaches 2^63.)  Logits 46 T log 2 and more below the largest weigh
// nothing and are left out of everything.
//
// A cluster of 1 to 8 blocks holds a row in shared memory, so it is read once.
//   - top-k up to kFewK: with b blocks, every block looks for a bound that at least k / b of its threads' own largest logits reach, and not many more; the
//     lowest of the bounds is below the k-th logit.  What reaches it (little more than k tokens) is gathered, and the first block does
//     the rest with these alone, comparing each with each.
//   - larger top-k: a histogram of the distance to the largest logit by counts, then a list of the tokens in the bucket that holds the threshold.
//   - top-p over the whole row: the counts bound the weights of a bucket to 1.6 % either way, so only what lies between those bounds (the
//     window) gets a histogram of exact weights, in bins of 1/256 of a factor of two; what lies above is summed per strip of 512 tokens and
//     all together per thread, in one pass.  The tokens of the window that turn out to be kept are added to their strips at the end.
//   - the draw looks for the strip in which the sum passes u times the whole, and goes through that strip alone.
// The fp64 exponential is 12 instructions at half rate and as many for its integers.  The functions that pass over a row are not
// inlined and work on variables at fixed places of shared memory: together in one body they were fetched as slowly as they ran.
// Measured: one row of 32000 fp32 logits 12 us (latency: two blocks' barriers), 64 with mixed filters 41 us, 256 rows of 128001 in bf16 with mixed filters 174 us. All
// rows alike, 256 x 128001: greedy 46 us, min-p alone 63, top-k of 50 65, unfiltered 86, top-k of 1000 223, top-p of 0.9 255 to 274: bound by the passes'
// instructions and the cluster's barriers, a block an SM with nothing beside it, not by reading (10 us).
#include <cooperative_groups.h>
#include <math.h>
#include <string.h>

#include <atomic>
#include <utility>

#include "cats_kernels.cuh"

namespace cats {
namespace {

namespace cg = cooperative_groups;
typedef long long i64;
constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kBuckets = kThreads;
constexpr int kFew = 256, kFewK = 128, kList = 2048;
constexpr int kMaxBlocks = 8;           // of a cluster
constexpr int kStrip = 512, kStrips = 8; // tokens, and how many of them a warp has at most
constexpr int kInside = 24;             // elements of a thread inside the window, of up to 256
constexpr float kRange = 46.f;          // log2 of the weights that count
constexpr float kWidth = kRange / ((float)kBuckets - 0.5f);      // of a bucket

struct Candidate {
    unsigned long long order;       // key of the logit, then the lower index first
    i64 w;
    __device__ __forceinline__ int index() const { return 0x7FFFFFFF - (int)(uint32_t)order; }
};
struct Found {
    i64 before, total;      // counts or weights in front of the bucket, and all
    int bucket;             // -1: what was asked for is not reached
    int count;              // of the bucket's tokens
};
struct Threshold {
    float tau;
    i64 above;              // sum in front of the tokens at tau
    int same;               // how many there are
};
struct Row {
    double c, top_d;        // log2 e / T; the largest logit
    float top, scale;       // the largest logit; buckets per logit, times 2
    float floor;            // logits from here down weigh nothing (600 powers of two below the largest, that one excluded)
    int n, first;           // elements of this block (whole vectors), index of the first (negative: in front of the row)
};
struct Shared {
    Row row;
    uint32_t cnt[kBuckets];
    union {
        struct { uint32_t lo[kBuckets], hi[kBuckets]; };        // weights as hi 2^32 + lo
        float list_mine[kList];                                 // logits of one bucket: this block's
    };
    union {
        struct { Candidate all[kFew], mine[kFew]; };          // as they come, and in their order
        float list[kList];                                      // and all blocks'
    };
    double table[256];                                          // 2^(i / 256)
    uint32_t strip_lo[2][kWarps][kStrips], strip_hi[2][kWarps][kStrips];  // of counts and of weights
    i64 xch[5][kMaxBlocks][2];
    i64 red[2][kWarps];
    i64 sum;
    i64 front[kFew];
    Found found, result;
    Threshold threshold;
    int n_mine, n_all, n_of[kMaxBlocks];
    int window[2];
    int index, strip_at;
    i64 strip_before;
};
__shared__ Shared sh;
// Dynamic: the notes of what lies inside the window (which of a thread's elements; a place for those too many), then this block's part of the row
extern __shared__ __align__(16) uint8_t dynamic[];
__device__ __forceinline__ uint8_t& noted_at(int q) { return dynamic[q * kThreads + threadIdx.x]; }
__device__ __forceinline__ uint4* row_data() { return reinterpret_cast<uint4*>(dynamic + (kInside + 1) * kThreads); }

// Keys in the order of the logits; -0 as 0.  (Of the keys between, only that of -0 is no number's: it stands for 0, too.)
__host__ __device__ __forceinline__ uint32_t bits_of(float x) {
    uint32_t b;
    memcpy(&b, &x, sizeof b);
    return b;
}
__host__ __device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = bits_of(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__host__ __device__ __forceinline__ float value_of(uint32_t key) {
    const uint32_t b = key & 0x80000000u ? key ^ 0x80000000u : ~key;
    float x;
    memcpy(&x, &b, sizeof x);
    return x;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(b));
    return a;
}

template <typename T> struct Elements;
template <> struct Elements<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float one(int i) { return reinterpret_cast<const float*>(row_data())[i]; }
    // the largest of a vector, NaN if there is one
    static __device__ __forceinline__ float top(const uint4& v) {
        float m = __uint_as_float(v.x);
        asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(__uint_as_float(v.y)), "f"(__uint_as_float(v.z)));
        return max_nan(m, __uint_as_float(v.w));
    }
};
template <> struct Elements<uint16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float one(int i) { return bf16_bits_to_float(reinterpret_cast<const uint16_t*>(row_data())[i]); }
    static __device__ __forceinline__ float top(const uint4& v) {
        uint32_t a, b;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
        return max_nan(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u));
    }
};

__device__ __forceinline__ int lane_id() { return threadIdx.x & 31; }
__device__ __forceinline__ int warp_id() { return threadIdx.x >> 5; }
__device__ __forceinline__ int rank_id() { return (int)cg::this_cluster().block_rank(); }
__device__ __forceinline__ int n_blocks() { return (int)cg::this_cluster().num_blocks(); }
__device__ __forceinline__ void sync_all() {
    if (n_blocks() > 1) cg::this_cluster().sync();
    else __syncthreads();
}
template <typename V> __device__ __forceinline__ V* of_block(V* p, int r) { return cg::this_cluster().map_shared_rank(p, r); }

// Sum of non-negative 62-bit numbers over a warp, in three parts
__device__ __forceinline__ i64 warp_sum(i64 x) {
    const uint32_t a = __reduce_add_sync(0xffffffffu, (uint32_t)x & 0x1FFFFFu), b = __reduce_add_sync(0xffffffffu, (uint32_t)(x >> 21) & 0x1FFFFFu),
                   c = __reduce_add_sync(0xffffffffu, (uint32_t)(x >> 42));
    return (i64)a + ((i64)b << 21) + ((i64)c << 42);
}
// and over the lanes up to and with this one
__device__ __forceinline__ i64 warp_upto(i64 x) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const i64 t = __shfl_up_sync(0xffffffffu, x, o);
        if (lane_id() >= o) x += t;
    }
    return x;
}
// and over a block; the second stage by one warp (by all of them, their reductions queue)
__device__ __noinline__ i64 block_sum(i64 x) {
    x = warp_sum(x);
    __syncthreads();
    if (lane_id() == 0) sh.red[0][warp_id()] = x;
    __syncthreads();
    if (warp_id() == 0) {
        x = warp_sum(sh.red[0][lane_id()]);
        if (lane_id() == 0) sh.sum = x;
    }
    __syncthreads();
    return sh.sum;
}
// a and b of this block to every block's sh.xch[site][rank]; a site is used again only after another exchange or sync_all
__device__ __noinline__ void exchange(int site, i64 a, i64 b) {
    if ((int)threadIdx.x < n_blocks()) {
        i64* const to = of_block(&sh.xch[site][rank_id()][0], threadIdx.x);
        to[0] = a;
        to[1] = b;
    }
    cg::this_cluster().sync();
}
__device__ __noinline__ i64 cluster_sum(int site, i64 x) {      // x: of the block
    const int n = n_blocks();
    if (n == 1) return x;
    exchange(site, x, 0);
    x = 0;
    for (int r = 0; r < n; ++r) x += sh.xch[site][r][0];
    return x;
}

// 2^44 times the weight = 2^(Y/256), Y = 256 ((x - top) c + 44), by 2^(i/256) 2^(r/256) with |r| <= 1/2 and the series of 2^(r/256) up to the third
// power (1.4e-13 off).  The constants are operands from the constant bank: as immediates, two of an instruction's took moves of their own.
__constant__ double kMagic = 6755399441055744.0;            // 1.5 2^52: a sum with it holds the nearest whole number in the low bits
__constant__ double kOnes = 4503599627370496.0;             // 2^52
__constant__ double kSeries[3] = {2.7076061740622863e-3, 3.6655655969101060e-6, 3.3083026805413710e-9};      // (ln 2 / 256)^n / n!
__constant__ double kTop = 44.0 * 256.0;
struct Weigher {
    double top, c;
    float floor;
    __device__ __forceinline__ Weigher() : top(sh.row.top_d), c(sh.row.c * 256.0), floor(sh.row.floor) {}
    __device__ __forceinline__ double exponent(float x) const { return fma((double)x - top, c, kTop); }
    static __device__ __forceinline__ double power(double y, int& i) {
        const double z = y + kMagic;
        i = __double2loint(z);
        const double r = y - (z - kMagic);
        double s = fma(r, kSeries[2], kSeries[1]);
        s = fma(s, r, kSeries[0]);
        s = fma(s, r, 1.0) * sh.table[i & 255];
        return __hiloint2double(__double2hiint(s) + ((i >> 8) << 20), __double2loint(s));
    }
    // i: Y rounded.  Only where live(x): below, the exponent may leave its range; the weight is zero there.
    __device__ __forceinline__ bool live(float x) const { return x > floor; }
    __device__ __forceinline__ i64 raw(float x, int& i) const {
        return __double_as_longlong(power(exponent(x), i) + kOnes) & 0xFFFFFFFFFFFFFll;      // rounded to a whole number
    }
    __device__ __forceinline__ i64 operator()(float x, int& i) const {
        const i64 w = raw(x, i);
        return live(x) ? w : 0;
    }
    __device__ __forceinline__ i64 operator()(float x) const {
        int i;
        return (*this)(x, i);
    }
    __device__ __forceinline__ float share_of(float x, i64 all) const {
        int i;
        return (float)(power(exponent(x), i) / (double)all);
    }
};
// Bucket by distance to the largest (a sum with 2^23 rounds it); false: weighs nothing (x = -inf at temperature inf: NaN)
struct Bucketer {
    float half_top, scale;
    __device__ __forceinline__ Bucketer() : half_top(0.5f * sh.row.top), scale(sh.row.scale) {}
    __device__ __forceinline__ bool operator()(float x, int& b) const {
        const float t = fmaf(x, -0.5f, half_top) * scale;           // halves: the difference of two large logits is still a number
        b = (int)(__float_as_uint(t + 8388608.f) & 0x7FFu);
        return t < (float)kBuckets - 0.5f;
    }
};
// A logit below all of bucket b: half a bucket and what fp32 rounds
__device__ __forceinline__ float below_bucket(int b) {
    const float top = sh.row.top;
    return (top - ((float)b + 1.f) * 2.f / sh.row.scale) - fabsf(top) * 2e-7f;
}

// A block's elements are followed by -inf up to a whole strip.
__device__ __forceinline__ int padded(int n) { return (n + kStrip - 1) / kStrip * kStrip; }
// f(x, i) for all elements that are at least x0, most vectors by their largest alone
template <typename T, typename F> __device__ __forceinline__ void each_from(float x0, F f) {
    constexpr int N = Elements<T>::N;
    const int n = sh.row.n / N;
#pragma unroll 4
    for (int v = threadIdx.x; v < n; v += kThreads) {
        if (Elements<T>::top(row_data()[v]) >= x0) {
#pragma unroll 1
            for (int e = 0; e < N; ++e) {
                const float x = Elements<T>::one(v * N + e);
                if (x >= x0) f(x, v * N + e);
            }
        }
    }
}

__device__ __forceinline__ void add64(uint32_t& lo, uint32_t& hi, i64 w) {
    const uint32_t a = (uint32_t)w, old = atomicAdd(&lo, a), b = (uint32_t)(w >> 32) + (old + a < old);
    if (b) atomicAdd(&hi, b);
}
__device__ __noinline__ void clear(bool first = false) {
    if (!first) sync_all();         // nobody reads the last histogram any more
    for (int i = threadIdx.x; i < kBuckets; i += kThreads) sh.cnt[i] = sh.lo[i] = sh.hi[i] = 0;
    __syncthreads();
}
// How many tokens each bucket has
template <typename T> __device__ __noinline__ void count(bool first) {
    clear(first);
    const Bucketer bucket;
    const int n = padded(sh.row.n);
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kThreads) {
        int b;
        if (bucket(Elements<T>::one(i), b)) atomicAdd(&sh.cnt[b], 1u);
    }
    sync_all();
}
// Counts and weights of bucket b in all blocks
__device__ __forceinline__ void bucket_sums(int b, bool weights, int& n, i64& w) {
    const int blocks = n_blocks();
    uint32_t cnt[kMaxBlocks], lo[kMaxBlocks], hi[kMaxBlocks];
#pragma unroll
    for (int r = 0; r < kMaxBlocks; ++r) {
        cnt[r] = lo[r] = hi[r] = 0;
        if (r < blocks) {
            cnt[r] = *of_block(&sh.cnt[b], r);
            if (weights) {
                lo[r] = *of_block(&sh.lo[b], r);
                hi[r] = *of_block(&sh.hi[b], r);
            }
        }
    }
    n = 0;
    w = 0;
#pragma unroll
    for (int r = 0; r < kMaxBlocks; ++r) {
        n += (int)cnt[r];
        w += ((i64)hi[r] << 32) + lo[r];
    }
}
// x all for 0 <= x < 1, rounded down, or up; all digits of it (fp64 holds 53 bits of a sum of up to 62)
__host__ __device__ __forceinline__ i64 part_of(float x, i64 all, bool up) {
    const uint32_t b = bits_of(x), e = b >> 23, m = ((b & 0x7FFFFFu) | (e ? 0x800000u : 0u)) << 8;       // x = m 2^-(k + 32), k >= 0
    const int k = 126 - (int)(e ? e : 1u), s = k < 63 ? k : 63;
    const unsigned long long low = (unsigned long long)m * (uint32_t)all, high = (unsigned long long)m * (uint32_t)(all >> 32) + (low >> 32);
    const unsigned long long q = high >> s;
    return (i64)(q + (up && ((high - (q << s)) | (uint32_t)low)));
}
__device__ __forceinline__ i64 share(float top_p, i64 all) {    // top_p < 1
    return top_p > 0.f ? max(part_of(top_p, all, true), (i64)1) : 1;
}
// The first bucket at which the running sum of the counts (or weights) over all blocks reaches `want`; want < 0: reaches share(top_p, all + more)
__device__ __noinline__ Found find(bool weights, i64 want, float top_p, i64 more) {
    int n0;
    i64 w0;
    bucket_sums(threadIdx.x, weights, n0, w0);
    if (!weights) w0 = n0;
    const i64 mine = warp_sum(w0);
    __syncthreads();
    if (lane_id() == 0) sh.red[0][warp_id()] = mine;
    __syncthreads();
    if (warp_id() == 0) {
        const i64 of_warp = sh.red[0][lane_id()], up = warp_upto(of_warp), total = __shfl_sync(0xffffffffu, up, 31);
        if (want < 0) want = share(top_p, total + more);
        const unsigned reached = __ballot_sync(0xffffffffu, up >= want);
        const int w = reached ? __ffs(reached) - 1 : -1;
        const i64 at = __shfl_sync(0xffffffffu, up - of_warp, max(w, 0));
        if (lane_id() == 0) {
            sh.found = {at, total, w, 0};        // the warp that has the bucket, for now
            sh.sum = want;
        }
    }
    __syncthreads();
    if (sh.found.bucket == warp_id()) {
        want = sh.sum;
        const i64 at = sh.found.before + warp_upto(w0) - w0;
        if (at < want && want <= at + w0) sh.result = {at, sh.found.total, (int)threadIdx.x, n0};
    } else if (sh.found.bucket < 0 && threadIdx.x == 0) {
        sh.result = sh.found;
    }
    __syncthreads();
    return sh.result;
}

// f(i, j) for all pairs of n candidates, the j of an i spread over lanes of a warp; done(i, on the first of these lanes) after sums a and b of what f
// adds to them.  All threads take part.
template <typename F, typename D> __device__ __forceinline__ void pairs(int n, F f, D done) {
    int per = 1;
    while (per < 32 && per * 2 * n <= kThreads) per *= 2;
    for (int i0 = 0; i0 < n; i0 += kThreads / per) {
        const int i = i0 + (int)threadIdx.x / per;
        i64 a = 0;
        int b = 0;
        if (i < n) {
#pragma unroll 4
            for (int j = threadIdx.x % per; j < n; j += per) f(i, j, a, b);
        }
        for (int o = 1; o < per; o <<= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if (i < n && threadIdx.x % per == 0) done(i, a, b);
    }
}
// After every block has its sh.n_mine: their sum, and each of them in sh.n_of
__device__ __noinline__ int sizes() {
    sync_all();
    const int blocks = n_blocks();
    if ((int)threadIdx.x < blocks) sh.n_of[threadIdx.x] = *of_block(&sh.n_mine, threadIdx.x);
    __syncthreads();
    int n = 0;
    for (int k = 0; k < blocks; ++k) n += sh.n_of[k];
    return n;
}
__device__ __forceinline__ void place(int i, int& r, int& at) {       // the i-th of all is the at-th of block r
    int n = 0;
    r = at = 0;
    for (int k = 0; k < n_blocks(); ++k) {
        if (i >= n) { r = k; at = i - n; }
        n += sh.n_of[k];
    }
}
// The tokens from x0 on, of all blocks, to sh.all of the first block, and how many there are to the sh.n_all of all (more than kFew: some have been left out).
// sh.n_all is zero before.
template <typename T> __device__ __noinline__ void gather(float x0) {
    const int first = sh.row.first, blocks = n_blocks();
    int* const n = of_block(&sh.n_all, 0);
    Candidate* const all = of_block(sh.all, 0);
    each_from<T>(x0, [&](float x, int i) {
        const int at = atomicAdd(n, 1);
        if (at < kFew) all[at] = {((unsigned long long)key_of(x) << 32) | (uint32_t)(0x7FFFFFFF - (first + i)), 0};
    });
    sync_all();
    if (blocks > 1) {
        if (threadIdx.x == 0 && rank_id() != 0) sh.n_all = *n;
        __syncthreads();
    }
}
// Strips: a warp has a run of neighbouring tokens, a strip at a time; lane l the elements l, l + 32, ... of it
__device__ __forceinline__ int run_of_warp(int n) { return ((n + kWarps - 1) / kWarps + kStrip - 1) / kStrip * kStrip; }
__device__ __forceinline__ int element_inside(int q) {
    const int n = padded(sh.row.n);
    return min(n, warp_id() * run_of_warp(n)) + lane_id() + 32 * noted_at(q);
}
// The logit at which the running sum (of counts, or of weights) in falling order reaches `want`: among the tokens from x0 on that in(x) says lie in got's
// bucket.  Every block finds it.
template <typename T, bool MASS, typename F> __device__ __noinline__ Threshold threshold(Found got, i64 want, float x0, F in, int inside = -1) {
    const Weigher weight;
    const int blocks = n_blocks();
    if (got.count > kList) {                // rare (equal logits, a flat row): bisection over the keys, a pass for each step
        uint32_t hi = 0, lo = 0xFFFFFFFFu;
        each_from<T>(x0, [&](float x, int) {
            if (in(x)) {
                hi = max(hi, key_of(x));
                lo = min(lo, key_of(x));
            }
        });
        hi = __reduce_max_sync(0xffffffffu, hi);
        lo = __reduce_min_sync(0xffffffffu, lo);
        __syncthreads();
        if (lane_id() == 0) { sh.red[0][warp_id()] = hi; sh.red[1][warp_id()] = lo; }
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) {
            hi = max(hi, (uint32_t)sh.red[0][w]);
            lo = min(lo, (uint32_t)sh.red[1][w]);
        }
        if (blocks > 1) {
            exchange(2, hi, lo);
            for (int r = 0; r < blocks; ++r) {
                hi = max(hi, (uint32_t)sh.xch[2][r][0]);
                lo = min(lo, (uint32_t)sh.xch[2][r][1]);
            }
        }
        int site = 3;
        auto sum_from = [&](uint32_t least, bool weights) {
            i64 sum = 0;
            each_from<T>(x0, [&](float x, int) {
                if (in(x) && key_of(x) >= least) sum += weights ? weight(x) : 1;
            });
            site = 7 - site;
            return cluster_sum(site, block_sum(sum));
        };
        if (lo == hi) return {value_of(hi), got.before, got.count};
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo + 1) / 2;
            if (got.before + sum_from(mid, MASS) >= want) lo = mid;
            else hi = mid - 1;
        }
        const i64 above = sum_from(lo + 1, MASS), n = sum_from(lo, false), n1 = sum_from(lo + 1, false);
        return {value_of(lo), got.before + above, (int)(n - n1)};
    }
    sync_all();                             // nobody reads the histogram and sh.n_mine any more
    if (threadIdx.x == 0) sh.n_mine = 0;
    __syncthreads();
    if (inside >= 0) {                      // this many of the thread's elements may be in the bucket
        for (int q = 0; q < inside; ++q) {
            const float x = Elements<T>::one(element_inside(q));
            if (in(x)) sh.list_mine[atomicAdd(&sh.n_mine, 1)] = x;
        }
    } else {
        each_from<T>(x0, [&](float x, int) {
            if (in(x)) sh.list_mine[atomicAdd(&sh.n_mine, 1)] = x;
        });
    }
    const int n = sizes();
    for (int i = threadIdx.x; i < n; i += kThreads) {
        int r, at;
        place(i, r, at);
        sh.list[i] = of_block(sh.list_mine, r)[at];
    }
    __syncthreads();
    if (n <= kFew) {                        // each with each
        if ((int)threadIdx.x < n) sh.front[threadIdx.x] = MASS ? weight(sh.list[threadIdx.x]) : 1;
        __syncthreads();
        pairs(n, [&](int i, int j, i64& a, int& b) {
            const float x = sh.list[i], y = sh.list[j];
            if (y > x) a += sh.front[j];
            b += y == x;
        }, [&](int i, i64 a, int b) {
            if (got.before + a < want && want <= got.before + a + b * sh.front[i]) sh.threshold = {sh.list[i], got.before + a, b};      // equal ones write the same
        });
        __syncthreads();
        return sh.threshold;
    }
    // bisection over the keys of the list: the largest key from which on the sum reaches `want`
    constexpr int kEach = (kList + kThreads - 1) / kThreads;
    uint32_t key[kEach], hi = 0, lo = 0xFFFFFFFFu;
    i64 w[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        key[k] = 0;
        w[k] = 0;
        if ((int)threadIdx.x + k * kThreads < n) {
            const float x = sh.list[threadIdx.x + k * kThreads];
            key[k] = key_of(x);
            w[k] = MASS ? weight(x) : 1;
            hi = max(hi, key[k]);
            lo = min(lo, key[k]);
        }
    }
    hi = __reduce_max_sync(0xffffffffu, hi);
    lo = __reduce_min_sync(0xffffffffu, lo);
    __syncthreads();
    if (lane_id() == 0) { sh.red[0][warp_id()] = hi; sh.red[1][warp_id()] = lo; }
    __syncthreads();
    hi = __reduce_max_sync(0xffffffffu, (uint32_t)sh.red[0][lane_id()]);
    lo = __reduce_min_sync(0xffffffffu, (uint32_t)sh.red[1][lane_id()]);
    auto sum_from = [&](uint32_t least, bool weights) {
        i64 sum = 0;
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (key[k] >= least && (int)threadIdx.x + k * kThreads < n) sum += weights ? w[k] : 1;
        return block_sum(sum);
    };
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        if (got.before + sum_from(mid, MASS) >= want) lo = mid;
        else hi = mid - 1;
    }
    const i64 above = sum_from(lo + 1, MASS), same = sum_from(lo, false) - sum_from(lo + 1, false);
    return {value_of(lo), got.before + above, (int)same};
}

// What a strip adds up: its tokens equal to tau; the weights of those from tau on; the same, but at tau only up to element `last`; or the weights above a
// window of the weights' exponents, while all are added up and a thread notes which of its elements are inside.
enum Sum : int { kEqual, kFrom, kKept, kAbove };
struct Window { int high, low, shift; };
template <typename T, int WHAT> __device__ __noinline__ i64 strips(float tau, int last, Window win, int& inside) {
    const int n = padded(sh.row.n), run = run_of_warp(n), i0 = min(n, warp_id() * run), i1 = min(n, i0 + run);
    const Weigher weight;
    i64 strip = 0, all = 0;         // of lane k: the sum of strip k
    int noted = 0;
    for (int i = i0, k = 0; i < i1; i += kStrip, ++k) {
        const int first = i + lane_id();
        if (WHAT != kAbove && tau > -INFINITY) {
            float most = -INFINITY;
#pragma unroll 8
            for (int e = 0; e < kStrip; e += 32) most = fmaxf(most, Elements<T>::one(first + e));
            if (!__any_sync(0xffffffffu, most >= tau)) continue;
        }
        i64 sum = 0;
        uint32_t equal = 0;
#pragma unroll 4
        for (int e = 0; e < kStrip; e += 32) {
            const float x = Elements<T>::one(first + e);
            if (WHAT == kEqual) {
                equal += x == tau;
            } else {
                int at;
                const i64 w = weight.raw(x, at);
                const bool live = weight.live(x);
                if (WHAT == kFrom) {
                    if (live && x >= tau) sum += w;
                } else if (WHAT == kKept) {
                    if (live && (x > tau || (x == tau && first + e <= last))) sum += w;
                } else if (live) {
                    all += w;
                    if (at > win.high) sum += w;
                    if ((unsigned)(win.high - at) <= (unsigned)(win.high - win.low)) {
                        noted_at(min(noted, kInside)) = (uint8_t)((i - i0 + e) / 32);
                        ++noted;
                    }
                }
            }
        }
        sum = WHAT == kEqual ? (i64)__reduce_add_sync(0xffffffffu, equal) : warp_sum(sum);
        if (lane_id() == k) strip = sum;
    }
    if (lane_id() < kStrips) {
        sh.strip_lo[WHAT != kEqual][warp_id()][lane_id()] = (uint32_t)strip;
        sh.strip_hi[WHAT != kEqual][warp_id()][lane_id()] = (uint32_t)(strip >> 32);
    }
    inside = noted;
    return all;
}
// f(x, i, w, at) for the elements inside the window, at: the bin.  noted: false where a thread had no room, then they are looked for.
template <typename T, typename F> __device__ __forceinline__ void each_inside(bool noted, int inside, Window win, F f) {
    const Weigher weight;
    auto one = [&](float x, int i) {
        int at;
        const i64 w = weight(x, at);
        if (w != 0 && at <= win.high && at >= win.low) f(x, i, w, (win.high - at) >> win.shift);
    };
    if (noted) {
        for (int q = 0; q < inside; ++q) {
            const int i = element_inside(q);
            one(Elements<T>::one(i), i);
        }
    } else {
        for (int i = threadIdx.x; i < sh.row.n; i += kThreads) one(Elements<T>::one(i), i);
    }
}
// The histogram of the window
template <typename T> __device__ __noinline__ void bins(bool noted, int inside, Window win) {
    each_inside<T>(noted, inside, win, [](float, int, i64 w, int b) {
        atomicAdd(&sh.cnt[b], 1u);
        add64(sh.lo[b], sh.hi[b], w);
    });
    sync_all();
}
// Its kept tokens, to the strips
template <typename T> __device__ __noinline__ void add_kept(bool noted, int inside, float tau, int last, Window win) {
    const int run = run_of_warp(padded(sh.row.n));
    __syncthreads();
    each_inside<T>(noted, inside, win, [=](float x, int i, i64 w, int) {
        if (x > tau || (x == tau && i <= last)) {
            const int of = i / run, k = (i - of * run) / kStrip;
            add64(sh.strip_lo[1][of][k], sh.strip_hi[1][of][k], w);
        }
    });
}
__device__ __forceinline__ i64 strip_sum(int of) {      // of the warp's strip that the lane stands for
    return lane_id() < kStrips ? ((i64)sh.strip_hi[of][warp_id()][lane_id()] << 32) + sh.strip_lo[of][warp_id()][lane_id()] : 0;
}
__device__ __forceinline__ i64 drawn(float u, i64 all) {
    return u > 0.f ? (u < 1.f ? part_of(u, all, false) : all - 1) : 0;
}
__device__ __forceinline__ void answer(const SampleDev& p, int d, int token, float prob) {
    p.token[d] = token;
    if (p.prob) p.prob[d] = prob;
}
// The first index at which the sum over the strips' tokens passes `want` (want < 0: drawn(u, total)).  draw >= 0: it is answered as that draw's token, and nothing
// more is to be done; else it goes to sh.index of every block.
template <typename T> __device__ __noinline__ void locate(const SampleDev& p, int draw, int what, float tau, int last, i64 want, float u) {
    const int n = padded(sh.row.n), i0 = min(n, warp_id() * run_of_warp(n)), blocks = n_blocks(), rank = rank_id();
    __syncthreads();
    const i64 strip = strip_sum(what != kEqual), up = warp_upto(strip), mine = __shfl_sync(0xffffffffu, up, 31);
    if (lane_id() == 0) sh.red[0][warp_id()] = mine;
    if (threadIdx.x == 0) sh.strip_at = -1;
    __syncthreads();
    const i64 of_warp = sh.red[0][lane_id()], warps = warp_upto(of_warp);
    i64 at = __shfl_sync(0xffffffffu, warps - of_warp, warp_id()), total = __shfl_sync(0xffffffffu, warps, 31);
    if (blocks > 1) {
        exchange(1, total, 0);
        total = 0;
        for (int r = 0; r < blocks; ++r) {
            if (r == rank) at += total;
            total += sh.xch[1][r][0];
        }
    }
    if (want < 0) want = drawn(u, total);
    if (at <= want && want < at + mine) {
        const int k = __ffs(__ballot_sync(0xffffffffu, want < at + up)) - 1;
        const i64 sum = at + __shfl_sync(0xffffffffu, up - strip, k);
        if (lane_id() == 0) { sh.strip_at = i0 + k * kStrip; sh.strip_before = sum; }
    }
    __syncthreads();
    if (sh.strip_at >= 0) {         // a thread for each token of that strip
        static_assert(kStrip <= kThreads, "one token per thread");
        const Weigher weight;
        const int i = sh.strip_at + (int)threadIdx.x;
        i64 one = 0;
        float x = -INFINITY;
        if ((int)threadIdx.x < kStrip) {
            x = Elements<T>::one(i);
            const i64 w = what == kEqual ? 1 : weight(x);
            if (what == kEqual ? x == tau : (x > tau || (x == tau && i <= last))) one = w;
        }
        const i64 to = warp_upto(one);
        if (lane_id() == 31) sh.red[1][warp_id()] = to;
        __syncthreads();
        const i64 others = sh.red[1][lane_id()], before = __shfl_sync(0xffffffffu, warp_upto(others) - others, warp_id());
        const i64 sum = sh.strip_before + before + to - one;
        if (sum <= want && want < sum + one) {
            if (draw >= 0) answer(p, draw, sh.row.first + i, what == kEqual ? 1.f : weight.share_of(x, total));
            else for (int r = 0; r < blocks; ++r) *of_block(&sh.index, r) = sh.row.first + i;
        }
    }
    if (draw < 0) sync_all();
}

// Top-p over the whole row: strips of what lies above the window, and the window's histogram; returns the window.  all: the weights of the row; first: there
// was no histogram yet.
template <typename T> __device__ __noinline__ Window weigh(float top_p, i64& all, bool& noted, int& inside, bool first) {
    count<T>(first);
    // n tokens of bucket b weigh n 2^(-b width) to within half a bucket; fp32 places a logit to 2^-23 of 1024 buckets, 2^-13 of one.  The sums are in units of 2^44.
    constexpr float kHalf = 0.501f;
    int count_of;
    i64 unused;
    bucket_sums(threadIdx.x, false, count_of, unused);
    float a = (float)count_of * exp2f(-((float)threadIdx.x - kHalf) * kWidth), z = (float)count_of * exp2f(-((float)threadIdx.x + kHalf) * kWidth);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {          // up to and with this bucket
        const float s = __shfl_up_sync(0xffffffffu, a, o), t = __shfl_up_sync(0xffffffffu, z, o);
        if (lane_id() >= o) { a += s; z += t; }
    }
    __syncthreads();
    if (lane_id() == 31) { sh.red[0][warp_id()] = __float_as_uint(a); sh.red[1][warp_id()] = __float_as_uint(z); }
    if (threadIdx.x == 0) sh.window[0] = sh.window[1] = kBuckets;
    __syncthreads();
    float all_up = __uint_as_float((uint32_t)sh.red[0][lane_id()]), all_down = __uint_as_float((uint32_t)sh.red[1][lane_id()]);
    const float up0 = all_up, down0 = all_down;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const float s = __shfl_up_sync(0xffffffffu, all_up, o), t = __shfl_up_sync(0xffffffffu, all_down, o);
        if (lane_id() >= o) { all_up += s; all_down += t; }
    }
    a += __shfl_sync(0xffffffffu, all_up - up0, warp_id());
    z += __shfl_sync(0xffffffffu, all_down - down0, warp_id());
    all_up = __shfl_sync(0xffffffffu, all_up, 31);
    all_down = __shfl_sync(0xffffffffu, all_down, 31);
    // the first bucket that may reach it, and the first that surely has
    if (a * 1.0001f >= top_p * all_down) atomicMin(&sh.window[0], (int)threadIdx.x);
    if (z >= top_p * all_up * 1.0001f) atomicMin(&sh.window[1], (int)threadIdx.x);
    __syncthreads();
    // as exponents: 256 y runs from 44 256 down to -2 256
    const bool bounded = sh.row.scale < 3e38f;      // else the buckets are wider than that
    Window win;
    win.high = bounded ? (int)ceilf(256.f * (44.f - ((float)sh.window[0] - kHalf) * kWidth)) + 1 : 44 * 256 + 1;
    win.low = bounded && sh.window[1] < kBuckets ? (int)floorf(256.f * (44.f - ((float)sh.window[1] + kHalf) * kWidth)) - 1 : -2 * 256 - 1;
    win.shift = 0;
    while (((win.high - win.low) >> win.shift) >= kBuckets) ++win.shift;
    clear();
    all = cluster_sum(0, block_sum(strips<T, kAbove>(0.f, 0, win, inside)));
    noted = !__syncthreads_or(inside > kInside);
    bins<T>(noted, inside, win);
    return win;
}

// n candidates in sh.all, the first top_k of the order among them: the filters and the draw, by one block
__device__ __noinline__ void finish(const SampleDev& p, int d, int n, int top_k, float top_p, float least, float u) {
    const Weigher weight;
    const bool mine = (int)threadIdx.x < n;
    const float x = mine ? value_of((uint32_t)(sh.all[threadIdx.x].order >> 32)) : 0.f;
    i64 w = mine ? weight(x) : 0;
    if (mine) sh.all[threadIdx.x].w = w;
    __syncthreads();
    // into their order, with the weight in front of each
    pairs(n, [&](int i, int j, i64& a, int& b) {
        const Candidate y = sh.all[j];
        if (y.order > sh.all[i].order) {
            a += y.w;
            ++b;
        }
    }, [&](int i, i64 a, int b) {
        sh.mine[b] = sh.all[i];
        sh.front[b] = a;
    });
    __syncthreads();
    n = min(n, top_k);
    const i64 all = sh.front[n - 1] + sh.mine[n - 1].w, want = top_p < 1.f ? share(top_p, all) : all + 1;
    const bool in = (int)threadIdx.x < n && sh.front[threadIdx.x] < want && value_of((uint32_t)(sh.mine[threadIdx.x].order >> 32)) >= least;
    n = __syncthreads_count(in);            // those in front
    const i64 kept = sh.front[n - 1] + sh.mine[n - 1].w, r = drawn(u, kept);
    // by index: the low words fall as the index rises
    pairs(n, [&](int i, int j, i64& a, int&) {
        const Candidate y = sh.mine[j];
        if ((uint32_t)y.order > (uint32_t)sh.mine[i].order) a += y.w;
    }, [&](int i, i64 a, int) {
        const Candidate c = sh.mine[i];
        if (a <= r && r < a + c.w) answer(p, d, c.index(), weight.share_of(value_of((uint32_t)(c.order >> 32)), kept));
    });
}

// log2 e / T, 0 at temperature 0
__host__ __device__ __forceinline__ double per_logit(float temp) { return temp == 0.f ? 0.0 : 1.4426950408889634074 / (double)temp; }
// The smallest logit whose weight is at least min_p, the largest among them always: bisection over the keys.  Weights are whole units of 2^-44, so that the
// first to reach min_p is what rounds to the next whole unit: half a unit less.  The logit lies within a few keys of what fp64 says,
// unless the sum cancels (a threshold next to 0 has more neighbours than fp64 tells apart) or is no fp32 number; then the search is over all.
__host__ __device__ __noinline__ float least_of(float top, double c, float min_p) {
    if (!(min_p > 0.f)) return -INFINITY;
    constexpr float kLowest = -3.402823466e38f;
    constexpr uint32_t kNear = 8;
    if (min_p > 1.f) return top;
    if (c == 0.0) return kLowest;
    constexpr double kUnits = 17592186044416.0;                 // 2^44
    const double log_p = log2((ceil((double)min_p * kUnits) - 0.5) / kUnits);
    auto in = [&](uint32_t key) { return ((double)value_of(key) - (double)top) * c >= log_p; };      // of the largest: 0 >= log_p
    const uint32_t first = key_of(kLowest), last = key_of(top), guess = key_of((float)fmax((double)top + log_p / c, (double)kLowest));
    uint32_t lo = guess - first > kNear ? guess - kNear : first, hi = last - guess > kNear ? guess + kNear : last;
    if (in(lo)) lo = first;
    if (!in(hi)) hi = last;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (in(mid)) hi = mid;
        else lo = mid + 1;
    }
    return value_of(hi);
}

template <typename T> __global__ void __launch_bounds__(kThreads) k_sample(const __grid_constant__ SampleDev p) {
    constexpr int N = Elements<T>::N;
    pdl_launch_dependents();
    if (threadIdx.x < 256) sh.table[threadIdx.x] = exp2((double)threadIdx.x / 256.0);
    if (threadIdx.x == 0) sh.n_all = 0;
    const int blocks = n_blocks(), rank = rank_id(), d = blockIdx.x / blocks, V = p.vocab;
    cg::cluster_group::arrival_token started;
    if (blocks > 1) started = cg::this_cluster().barrier_arrive();
    pdl_wait();
    const int row = p.row ? p.row[d] : d;
    const float temp = p.temperature ? p.temperature[d] : 1.f, top_p = p.top_p ? p.top_p[d] : 1.f, min_p = p.min_p ? p.min_p[d] : 0.f, u = p.u[d];
    int top_k = p.top_k ? p.top_k[d] : 0;
    bool bad = row >= p.logit_rows || !(temp >= 0.f) || isnan(top_p) || isnan(min_p) || isnan(u);
    const T* const x = (const T*)p.logits + (bad || row < 0 ? 0 : row) * p.ld;
    float own = -INFINITY, top = -INFINITY;              // the largest of this thread's, of the row
    if (row >= 0 && !bad) {
        // this block's vectors: of 16 bytes on their grid; what of them lies outside the row counts as -inf
        const int shift = (int)(((uintptr_t)x & 15) / sizeof(T)), all_vecs = (shift + V + N - 1) / N, per = (all_vecs + blocks - 1) / blocks;
        const int v0 = min(all_vecs, rank * per), vecs = min(per, all_vecs - v0), first = v0 * N - shift;
        const uint4* const from = reinterpret_cast<const uint4*>(x - shift) + v0;
        constexpr int kAtOnce = 4;
        for (int va = threadIdx.x; va < vecs; va += kThreads * kAtOnce) {
            uint4 w[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int v = va + k * kThreads, i = first + v * N;
                w[k] = make_uint4(0, 0, 0, 0);
                if (v < vecs && i >= 0 && i + N <= V) w[k] = __ldcg(from + v);
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int v = va + k * kThreads, i = first + v * N;
                if (v >= vecs) break;
                if (i < 0 || i + N > V) {
                    uint32_t y[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const bool there = i + e >= 0 && i + e < V;
                        if (sizeof(T) == 4) y[e & 3] = there ? reinterpret_cast<const uint32_t*>(x)[i + e] : 0xFF800000u;
                        else y[e / 2] |= (there ? (uint32_t)reinterpret_cast<const uint16_t*>(x)[i + e] : 0xFF80u) << (16 * (e & 1));
                    }
                    w[k] = make_uint4(y[0], y[1], y[2], y[3]);
                }
                row_data()[v] = w[k];
                own = max_nan(own, Elements<T>::top(w[k]));
            }
        }
        const uint32_t none = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
        for (int v = vecs + threadIdx.x; v < padded(vecs * N) / N; v += kThreads) row_data()[v] = make_uint4(none, none, none, none);
        top = own;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (lane_id() == 0) sh.red[0][warp_id()] = __float_as_uint(top);
        if (threadIdx.x == 0) { sh.row.n = vecs * N; sh.row.first = first; }
        __syncthreads();
        top = __uint_as_float((uint32_t)sh.red[0][lane_id()]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    if (min_p > 1.f) top_k = 1;             // no weight reaches that: the first of the order alone
    const bool by_bound = row >= 0 && !bad && top_k > 0 && top_k < V && top_k <= kFewK && temp > 0.f;
    float bound = -INFINITY;
    if (by_bound) {                 // that at least `least` of the block's threads reach, and at most half as many more if a few steps find it
        const int least = (top_k + blocks - 1) / blocks;
        float step = fminf(temp, 1e30f), low = top - step;
        int n = 0;
        for (int k = 0; k < 12 && (n = __syncthreads_count(own >= low)) < least; ++k) {
            step *= 2.f;
            low = top - step;
        }
        if (n >= least) {
            float high = low + 0.5f * step;         // too few reach that, or it is the largest
            for (int k = 0; k < 6 && n > least + least / 2; ++k) {
                const float mid = 0.5f * low + 0.5f * high;
                const int m = __syncthreads_count(own >= mid);
                if (m >= least) {
                    low = mid;
                    n = m;
                } else {
                    high = mid;
                }
            }
            bound = low;
        }
    }
    if (blocks > 1) cg::this_cluster().barrier_wait(std::move(started));      // the others' shared memory is there
    if (row < 0) return;
    if (!bad) {
        if (blocks > 1) {
            exchange(4, __float_as_uint(top), __float_as_uint(bound));
            for (int r = 0; r < blocks; ++r) {
                top = max_nan(top, __uint_as_float((uint32_t)sh.xch[4][r][0]));
                bound = fminf(bound, __uint_as_float((uint32_t)sh.xch[4][r][1]));
            }
        }
        bad = !(top < INFINITY) || top == -INFINITY;
    }
    if (bad) {
        if (threadIdx.x == 0 && rank == 0) {
            answer(p, d, -1, 0.f);
            report(p.d_status, CATS_ERR_INVALID_ARG);
        }
        return sync_all();
    }
    const double c = per_logit(temp);
    if (threadIdx.x == 0) {
        sh.row.top = top;
        sh.row.floor = fminf((float)((double)top - 600.0 / c), value_of(key_of(top) - 1));
        sh.row.top_d = (double)top;
        sh.row.c = c;
        sh.row.scale = (float)fmin(2.0 * c / (double)kWidth, 3e38);
    }
    __syncthreads();
    if (temp == 0.f) {
        int none;
        strips<T, kEqual>(top, 0, {}, none);
        return locate<T>(p, d, kEqual, top, 0, 0, u);
    }
    const float least = least_of(top, c, min_p);
    float tau = -INFINITY;          // kept: logits above tau, and at tau the ones up to index `last`
    i64 ties = -1;                  // how many at tau; -1: all
    int same = 0;
    bool by_k = top_k > 0 && top_k < V;
    if (by_bound && bound > -INFINITY) {
        gather<T>(bound);
        if (sh.n_all <= kFew) {
            if (rank == 0) finish(p, d, sh.n_all, top_k, top_p, least, u);
            return sync_all();
        }
    }
    if (by_k) {
        count<T>(!by_bound);
        const Found f = find(false, top_k, 0.f, 0);
        by_k = f.bucket >= 0;       // else fewer than top_k weigh anything
        if (by_k) {
            const Bucketer bucket;
            const int at = f.bucket;
            const Threshold t = threshold<T, false>(f, top_k, below_bucket(at), [bucket, at](float y) { int b; return bucket(y, b) && b == at; });
            tau = t.tau;
            ties = top_k - t.above;
            same = t.same;
        }
    }
    Window win = {};
    bool windowed = false, noted = false;       // strips of what lies above the window are there; notes of what lies inside
    int inside = 0;
    if (top_p < 1.f && by_k) {      // few tokens: of the logits above tau, and so many at tau
        const Weigher weight;
        const Bucketer bucket;
        clear();
        each_from<T>(tau, [&](float y, int) {
            int b;
            if (y > tau && bucket(y, b)) {
                atomicAdd(&sh.cnt[b], 1u);
                add64(sh.lo[b], sh.hi[b], weight(y));
            }
        });
        sync_all();
        const i64 w = weight(tau), at_tau = ties * w;
        const Found f = find(true, -1, top_p, at_tau);
        const i64 want = share(top_p, f.total + at_tau);
        if (f.bucket >= 0) {
            const int at = f.bucket;
            const Threshold t = threshold<T, true>(f, want, fmaxf(tau, below_bucket(at)), [bucket, at, tau](float y) { int b; return y > tau && bucket(y, b) && b == at; });
            tau = t.tau;
            const i64 v = weight(tau);
            ties = (want - t.above + v - 1) / v;
            same = t.same;
        } else {                    // inside the tokens at the threshold of top-k
            ties = (want - f.total + w - 1) / w;
        }
    } else if (top_p < 1.f) {
        i64 all;
        win = weigh<T>(top_p, all, noted, inside, top_k <= 0 || top_k >= V);     // a top-k that cuts nothing has had its histogram
        windowed = true;
        // in front of the window
        i64 above = block_sum(strip_sum(1));
        above = cluster_sum(1, above);
        const i64 want = share(top_p, all);
        Found f = find(true, want - above, 0.f, 0);
        f.before += above;
        const Weigher weight;
        const int at = f.bucket;
        // a logit below all of the bin: one more bin and what fp32 rounds
        const double low = (double)(win.high - ((at + 1) << win.shift) - 2) / 256.0 - 44.0;
        const float x0 = c == 0.0 ? -3.402823466e38f : (float)fmax((double)top + low / c - fabs((double)top) * 2e-7 - fabs(low / c) * 2e-7, -3.4028234663852886e38);
        const Threshold t = threshold<T, true>(f, want, x0, [weight, at, win](float y) {
            int i;
            return weight(y, i) != 0 && i <= win.high && i >= win.low && (win.high - i) >> win.shift == at;
        }, noted ? inside : -1);
        tau = t.tau;
        const i64 v = weight(tau);
        ties = (want - t.above + v - 1) / v;
        same = t.same;
    }
    if (least > tau) {
        tau = least;
        ties = -1;
        windowed = false;           // the strips may hold more than that
    }
    int last = kMaxSampleVocab;     // an element of this block
    if (ties >= 0 && ties < same) {
        int none;
        strips<T, kEqual>(tau, 0, {}, none);
        locate<T>(p, -1, kEqual, tau, 0, ties - 1, u);
        last = sh.index - sh.row.first;
        sync_all();
    }
    if (windowed) add_kept<T>(noted, inside, tau, last, win);
    else if (last == kMaxSampleVocab) strips<T, kFrom>(tau, last, {}, inside);
    else strips<T, kKept>(tau, last, {}, inside);
    locate<T>(p, d, kKept, tau, last, -1, u);
}

template <typename T> cudaError_t launch_t(const SampleDev& p, cudaStream_t st) {
    constexpr int kMost = 196 * 1024, kUsual = 136 * 1024;     // bytes of a row per block: what fits with the rest, and what is taken where rows are many
    const long long bytes = (long long)p.vocab * sizeof(T) + 32;
    int blocks = (int)min((long long)kMaxBlocks, (bytes + kUsual - 1) / kUsual);
    // kUsual: 256 rows of 128001 in bf16 with top-p 274 us, with 104 KB 343, with 68 KB 411 (three and four blocks a row); 160 KB is the same there and for 32000,
    // 50257, 100003 and 200000 tokens, and better where it saves a block (151936 in bf16 380 -> 314).
    // SMs that no row has take halves of them (64 rows of 32000: 54 -> 43 us when it was added; smaller parts cost more in barriers of the cluster than they save: 16
    // rows of 128001 14 us in parts of 80 KB, 23 in parts of 40)
    while (blocks < kMaxBlocks && (long long)p.rows * (blocks + 1) <= 148 && bytes / blocks > 80 * 1024) ++blocks;
    const size_t smem = (size_t)((bytes / 16 + 2 + blocks - 1) / blocks) * 16 + kStrip * sizeof(T) + (kInside + 1) * kThreads;
    static std::atomic<uint64_t> known{0};           // devices whose attribute is set
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!(known.load(std::memory_order_acquire) >> dev & 1)) {
        e = cudaFuncSetAttribute(k_sample<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (e != cudaSuccess) return e;
        known.fetch_or((uint64_t)1 << dev, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.rows * (unsigned)blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)blocks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    ++g_launch_count;
    return cudaLaunchKernelEx(&cfg, k_sample<T>, p);
}

}  // namespace

long long sample_part(float x, long long all, bool up) { return part_of(x, all, up); }
float sample_least(float top, float temperature, float min_p) { return least_of(top, per_logit(temperature), min_p); }
cudaError_t launch_sample(const SampleDev& p, cudaStream_t st) { return p.f32 ? launch_t<float>(p, st) : launch_t<uint16_t>(p, st); }

}  // namespace cats
