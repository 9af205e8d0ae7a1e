// One token per row of logits (include/cats.h: cats_sample).
//
// Tokens are ordered by falling logit, equal ones by rising index; top-k, top-p and min-p each keep a run from the front of
// that order, so what is kept is: every token whose logit is above a threshold, and the first few (by index) of those at it.
// w = exp((x - max) / T) is a whole multiple of 2^-44, taken from an fp64 exponential: the sums are exact 64-bit integers, the same in any
// order, and so are all decisions made from them.  (vocab <= 2^18, so no sum reaches 2^63.)  Logits 46 T log 2 and more below the largest weigh
// nothing and are left out of everything.
//
// A cluster of 1 to 8 blocks holds a row in shared memory, so it is read once.
//   - top-k up to kFewK: the k-th largest of the threads' own maxima bounds the k-th logit from below; what reaches that bound (little more
//     than k tokens) is gathered, and the first block does the rest with these alone, comparing each with each.
//   - else thresholds come from a histogram of the distance to the largest logit, then of the keys within the bucket that holds the
//     threshold, until at most kFew tokens are left.  For top-p the counts bound the weights of a bucket to 1.6 % either way, so
//     only the buckets between those bounds get exact sums by atomics; everything above and all together are sums in registers.
//     Where at most kFew tokens lie in the buckets up to the threshold's, these are gathered and finished as above.
// The fp64 exponential, 12 instructions at half rate, is what rows without top-k spend their time on.
#include <cooperative_groups.h>

#include <atomic>
#include <utility>

#include "cats_kernels.cuh"

namespace cats {
namespace {

namespace cg = cooperative_groups;
typedef long long i64;
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBuckets = 1024;
constexpr int kFew = 256, kFewK = 128;
constexpr int kMaxBlocks = 8;           // of a cluster
constexpr float kRange = 46.f;          // log2 of the weights that count

// Keys in the order of the logits; -0 as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

template <typename T> struct Elements;
template <> struct Elements<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float get(const uint4& v, int e) { return __uint_as_float(e == 0 ? v.x : (e == 1 ? v.y : (e == 2 ? v.z : v.w))); }
    // the largest of a vector, NaN if there is one
    static __device__ __forceinline__ float top(const uint4& v) {
        float m = __uint_as_float(v.x);
        asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(__uint_as_float(v.y)), "f"(__uint_as_float(v.z)));
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(__uint_as_float(v.w)));
        return m;
    }
};
template <> struct Elements<uint16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float get(const uint4& v, int e) {
        const uint32_t w = e < 2 ? v.x : (e < 4 ? v.y : (e < 6 ? v.z : v.w));
        return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
    }
    static __device__ __forceinline__ float top(const uint4& v) {
        uint32_t a, b;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
        float m = __uint_as_float(a << 16);
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(__uint_as_float(a & 0xFFFF0000u)));
        return m;
    }
};
__device__ __forceinline__ float max_nan(float a, float b) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(b));
    return a;
}

struct Candidate {
    float x;
    int index;
    i64 w;
};
struct Found {
    int bucket;             // -1: the target is not reached
    int count_before, count;
    i64 before;             // of what was asked for: counts or weights
};

template <typename T> struct Row {
    static constexpr int N = Elements<T>::N;
    struct Shared {
        uint32_t cnt[kBuckets], lo[kBuckets], hi[kBuckets];     // counts, and weights as hi 2^32 + lo
        Candidate all[kFew], mine[kFew];
        double table[64];                                       // 2^(i / 64)
        i64 xch[2][kMaxBlocks][2];
        i64 red[2][kWarps];
        Found found;
        int n_mine, n_of[kMaxBlocks + 1];
        int window[2];
        uint32_t tau;
        i64 above;
        int same, index;
    };
    const SampleDev& p;
    Shared& sh;
    const uint4* data;              // this block's vectors
    cg::cluster_group cluster;
    const int rank, blocks, lane, warp;
    int vecs, first;                // vectors of this block, index of its first element (negative: in front of the row)
    int parity;
    float top, bucket_scale;
    double c;

    __device__ __forceinline__ Row(const SampleDev& p_, Shared& s_, const uint4* d_)
        : p(p_), sh(s_), data(d_), cluster(cg::this_cluster()), rank((int)cluster.block_rank()), blocks((int)cluster.num_blocks()), lane(threadIdx.x & 31),
          warp(threadIdx.x >> 5), parity(0) {}

    __device__ __forceinline__ void sync() {
        if (blocks > 1) cluster.sync();
        else __syncthreads();
    }
    template <typename F> __device__ __forceinline__ void each(F f) const {
        for (int v = threadIdx.x; v < vecs; v += kThreads) {
            const uint4 x = data[v];
#pragma unroll
            for (int e = 0; e < N; ++e) f(Elements<T>::get(x, e), first + v * N + e);
        }
    }
    // 2^44 times the weight = 2^y, by 2^(i/64) 2^r with |r| <= 1/128 and the series of 2^r up to the fourth power (4e-14 off)
    __device__ __forceinline__ double power(double y) const {
        const double z = fma(y, 64.0, 6755399441055744.0);          // 1.5 2^52: 64 y as a whole number in the low bits
        const int i = __double2loint(z);
        const double r = fma(z - 6755399441055744.0, -0.015625, y);
        double s = fma(r, 9.6181291076284772e-3, 5.5504108664821580e-2);        // (ln 2)^n / n!
        s = fma(s, r, 2.4022650695910071e-1);
        s = fma(s, r, 6.9314718055994531e-1);
        s = fma(s, r, 1.0) * sh.table[i & 63];
        return __hiloint2double(__double2hiint(s) + ((i >> 6) << 20), __double2loint(s));
    }
    __device__ __forceinline__ double power_of(float x) const { return fma((double)x - (double)top, c, 44.0); }
    __device__ __forceinline__ i64 weight(float x) const {
        const double y = power_of(x);
        const i64 w = __double_as_longlong(power(y) + 4503599627370496.0) & 0xFFFFFFFFFFFFFll;      // + 2^52: rounded to a whole number
        return y > -2.0 ? w : 0;                                    // -inf too
    }
    // Bucket by distance to the largest (a sum with 2^23 rounds it); false: weighs nothing (x = -inf at temperature inf: NaN)
    __device__ __forceinline__ bool bucket_of(float x, int& b) const {
        const float t = (0.5f * top - 0.5f * x) * bucket_scale;       // halves: the difference of two large logits is still a number
        b = (int)(__float_as_uint(t + 8388608.f) & 0x7FFu);
        return t < (float)kBuckets - 0.5f;
    }
    // a and b of this block to every block's sh.xch[parity ^ 1][rank]
    __device__ __forceinline__ void exchange(i64 a, i64 b) {
        if ((int)threadIdx.x < blocks) {
            i64* const to = cluster.map_shared_rank(&sh.xch[parity][rank][0], threadIdx.x);
            to[0] = a;
            to[1] = b;
        }
        cluster.sync();
        parity ^= 1;
    }
    // Sums of (a, b) over the threads of this block in front of this one; totals in all_a, all_b
    __device__ __forceinline__ void before(i64& a, i64& b, i64& all_a, i64& all_b) {
        i64 x = a, y = b;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const i64 s = __shfl_up_sync(0xffffffffu, x, o), t = __shfl_up_sync(0xffffffffu, y, o);
            if (lane >= o) { x += s; y += t; }
        }
        __syncthreads();
        if (lane == 31) { sh.red[0][warp] = x; sh.red[1][warp] = y; }
        __syncthreads();
        a = x - a;
        b = y - b;
        all_a = all_b = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) { a += all_a; b += all_b; }
            all_a += sh.red[0][w];
            all_b += sh.red[1][w];
        }
    }

    // f(x, ...) for all elements that are at least x0, most vectors by their largest alone
    template <typename F> __device__ __forceinline__ void each_from(float x0, F f) const {
        for (int v = threadIdx.x; v < vecs; v += kThreads) {
            const uint4 x = data[v];
            if (Elements<T>::top(x) >= x0) {
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (Elements<T>::get(x, e) >= x0) f(Elements<T>::get(x, e), first + v * N + e);
            }
        }
    }
    __device__ __forceinline__ void add_weight(int b, i64 w) {
        const uint32_t lo = (uint32_t)w, old = atomicAdd(&sh.lo[b], lo), hi = (uint32_t)(w >> 32) + (old + lo < old);
        if (hi) atomicAdd(&sh.hi[b], hi);
    }
    __device__ __forceinline__ void clear() {
        sync();                     // nobody reads the last one any more
        for (int i = threadIdx.x; i < kBuckets; i += kThreads) sh.cnt[i] = sh.lo[i] = sh.hi[i] = 0;
        __syncthreads();
    }
    // Histogram of what f puts into a bucket (f(x, b): whether it does) among the logits from x0 on, by counts alone or with the weights
    template <bool MASS, typename F> __device__ __forceinline__ void histogram(float x0, F f) {
        clear();
        auto one = [&](float x, int) {
            int b;
            if (!f(x, b)) return;
            // all lanes at one bucket (equal logits): one of them adds for all
            const unsigned at = __activemask();
            const int b0 = __shfl_sync(at, b, __ffs(at) - 1);
            i64 w = MASS ? weight(x) : 0;
            if (at == 0xffffffffu && __all_sync(at, b == b0)) {
                if (MASS) {
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
                }
                if (lane == 0) {
                    atomicAdd(&sh.cnt[b], 32u);
                    if (MASS && w) add_weight(b, w);
                }
            } else {
                atomicAdd(&sh.cnt[b], 1u);
                if (MASS && w) add_weight(b, w);
            }
        };
        if (x0 > -INFINITY) each_from(x0, one);
        else each(one);
        sync();
    }
    // Counts and weights of bucket b in all blocks
    template <bool MASS> __device__ __forceinline__ void bucket_sums(int b, i64& n, i64& w) {
        uint32_t cnt[kMaxBlocks], lo[kMaxBlocks], hi[kMaxBlocks];
#pragma unroll
        for (int r = 0; r < kMaxBlocks; ++r) {
            cnt[r] = lo[r] = hi[r] = 0;
            if (r < blocks) {
                cnt[r] = blocks > 1 ? cluster.map_shared_rank(sh.cnt, r)[b] : sh.cnt[b];
                if (MASS) {
                    lo[r] = blocks > 1 ? cluster.map_shared_rank(sh.lo, r)[b] : sh.lo[b];
                    hi[r] = blocks > 1 ? cluster.map_shared_rank(sh.hi, r)[b] : sh.hi[b];
                }
            }
        }
        n = w = 0;
#pragma unroll
        for (int r = 0; r < kMaxBlocks; ++r) {
            n += cnt[r];
            if (MASS) w += ((i64)hi[r] << 32) + lo[r];
        }
    }
    // The first bucket at which the running sum of the counts (or weights) over all blocks reaches what target(total) says
    template <bool MASS, typename F> __device__ __forceinline__ Found find(F target, i64& total) {
        constexpr int each_has = kBuckets / kThreads;
        i64 val[each_has], cnt[each_has], a = 0, n = 0;
#pragma unroll
        for (int i = 0; i < each_has; ++i) {
            bucket_sums<MASS>(threadIdx.x * each_has + i, cnt[i], val[i]);
            if (!MASS) val[i] = cnt[i];
            a += val[i];
            n += cnt[i];
        }
        i64 all_n;
        if (threadIdx.x == 0) sh.found.bucket = -1;
        before(a, n, total, all_n);
        const i64 want = target(total);
#pragma unroll
        for (int i = 0; i < each_has; ++i) {
            if (a < want && want <= a + val[i]) sh.found = {(int)threadIdx.x * each_has + i, (int)n, (int)cnt[i], a};
            a += val[i];
            n += cnt[i];
        }
        __syncthreads();
        const Found f = sh.found;
        __syncthreads();
        return f;
    }

    // Tokens from x0 on that f takes, of all blocks, to sh.all of this block (every block, or the first alone).  Returns how many there are: if more than kFew, none
    // have been taken.
    template <typename F> __device__ __forceinline__ int gather(bool first_only, float x0, F f) {
        if (threadIdx.x == 0) sh.n_mine = 0;
        sync();                     // and nobody reads sh.mine any more
        auto one = [&](float x, int index) {
            if (f(x)) {
                const int at = atomicAdd(&sh.n_mine, 1);
                if (at < kFew) sh.mine[at] = {x, index, 0};
            }
        };
        if (x0 > -INFINITY) each_from(x0, one);
        else each(one);
        sync();
        if ((int)threadIdx.x < blocks) sh.n_of[threadIdx.x + 1] = blocks > 1 ? *cluster.map_shared_rank(&sh.n_mine, threadIdx.x) : sh.n_mine;
        __syncthreads();
        int n = 0, r = 0, at = 0;   // this thread's candidate: the at-th of block r
        for (int k = 0; k < blocks; ++k) {
            if ((int)threadIdx.x >= n) { r = k; at = threadIdx.x - n; }
            n += sh.n_of[k + 1];
        }
        if (n <= kFew && (int)threadIdx.x < n && (!first_only || rank == 0)) sh.all[threadIdx.x] = (blocks > 1 ? cluster.map_shared_rank(sh.mine, r) : sh.mine)[at];
        return n;
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
            if (i < n)
                for (int j = threadIdx.x % per; j < n; j += per) f(i, j, a, b);
            for (int o = 1; o < per; o <<= 1) {
                a += __shfl_xor_sync(0xffffffffu, a, o);
                b += __shfl_xor_sync(0xffffffffu, b, o);
            }
            if (i < n && threadIdx.x % per == 0) done(i, a, b);
        }
    }
    static __device__ __forceinline__ bool in_front(const Candidate& a, const Candidate& b) { return a.x > b.x || (a.x == b.x && a.index < b.index); }

    // The logit at which the running sum (of counts, or of weights) in falling order reaches `want`, among the tokens that f takes (f(x, b): whether, and its bucket), after
    // their histogram: to sh.tau its key, to sh.above the sum in front of it and to sh.same how many tokens have it.
    template <bool MASS, typename F> __device__ __forceinline__ void threshold(Found got, i64 want, F f) {
        i64 skipped = got.before;
        uint32_t k0 = 0, k1 = 0xFFFFFFFFu;      // keys that are left
        int shift = 32;                         // 32: by f; else buckets of 2^shift keys from k1 down
        auto in = [&](float x) {
            const uint32_t k = key_of(x);
            int b;
            if (k < k0 || k > k1) return false;
            if (shift == 32) return f(x, b) && b == got.bucket;
            return (int)((k1 - k) >> shift) == got.bucket;
        };
        while (got.count > kFew) {
            // range of the keys in this bucket
            uint32_t most = 0, least = 0xFFFFFFFFu;
            each([&](float x, int) {
                if (in(x)) {
                    const uint32_t k = key_of(x);
                    most = max(most, k);
                    least = min(least, k);
                }
            });
            most = __reduce_max_sync(0xffffffffu, most);
            least = __reduce_min_sync(0xffffffffu, least);
            __syncthreads();
            if (lane == 0) { sh.red[0][warp] = most; sh.red[1][warp] = least; }
            __syncthreads();
            for (int w = 0; w < kWarps; ++w) {
                most = max(most, (uint32_t)sh.red[0][w]);
                least = min(least, (uint32_t)sh.red[1][w]);
            }
            if (blocks > 1) {
                exchange(most, least);
                for (int r = 0; r < blocks; ++r) {
                    most = max(most, (uint32_t)sh.xch[parity ^ 1][r][0]);
                    least = min(least, (uint32_t)sh.xch[parity ^ 1][r][1]);
                }
            }
            if (most == least) {
                __syncthreads();
                if (threadIdx.x == 0) { sh.tau = most; sh.above = skipped; sh.same = got.count; }
                __syncthreads();
                return;
            }
            const uint32_t n0 = least, n1 = most;
            int s = 0;
            while (((n1 - n0) >> s) >= (uint32_t)kBuckets) ++s;
            // keys between the least and the most of a bucket are all in it
            histogram<MASS>(value_of(n0), [&](float x, int& b) {
                const uint32_t k = key_of(x);
                b = (int)((n1 - k) >> s);
                return k >= n0 && k <= n1 && weighs(x, f);
            });
            k0 = n0;
            k1 = n1;
            shift = s;
            i64 total;
            got = find<MASS>([&](i64) { return want - skipped; }, total);
            skipped += got.before;
        }
        const int n = gather(false, -INFINITY, [&](float x) { return in(x) && (shift == 32 || weighs(x, f)); });
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) sh.all[i].w = MASS ? weight(sh.all[i].x) : 1;
        __syncthreads();
        pairs(n, [&](int i, int j, i64& a, int& b) {
            if (sh.all[j].x > sh.all[i].x) a += sh.all[j].w;
            b += sh.all[j].x == sh.all[i].x;
        }, [&](int i, i64 a, int b) {
            if (skipped + a < want && want <= skipped + a + b * sh.all[i].w) {
                sh.tau = key_of(sh.all[i].x);
                sh.above = skipped + a;
                sh.same = b;
            }
        });
        __syncthreads();
    }
    template <typename F> static __device__ __forceinline__ bool weighs(float x, F f) {
        int b;
        return f(x, b);
    }

    // The first index at which the running sum of f over the row exceeds `target`, to sh.index of every block that asks; total: the whole sum.  A warp takes
    // a run of neighbouring vectors.
    template <typename F, typename G> __device__ __forceinline__ void walk(F f, G target, i64& total) {
        const int run = ((vecs + kWarps - 1) / kWarps + 31) / 32 * 32, v0 = min(vecs, warp * run), v1 = min(vecs, v0 + run);      // at most 32 strips of 32 vectors
        auto of_vec = [&](int v) {
            i64 s = 0;
            if (v < v1) {
                const uint4 x = data[v];
#pragma unroll
                for (int e = 0; e < N; ++e) s += f(Elements<T>::get(x, e), first + v * N + e);
            }
            return s;
        };
        i64 strip = 0;              // of lane i: the sum of strip i
        for (int v = v0, i = 0; v < v1; v += 32, ++i) {
            i64 one = of_vec(v + lane);
            if (__any_sync(0xffffffffu, one != 0)) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) one += __shfl_xor_sync(0xffffffffu, one, o);
                if (lane == i) strip = one;
            }
        }
        i64 mine = strip;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const i64 t = __shfl_up_sync(0xffffffffu, mine, o);
            if (lane >= o) mine += t;
        }
        const i64 strips = mine;    // up to and with strip i
        mine = __shfl_sync(0xffffffffu, mine, 31);
        __syncthreads();
        if (lane == 0) sh.red[0][warp] = mine;
        __syncthreads();
        i64 at = 0, block = 0;
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) at = block;
            block += sh.red[0][w];
        }
        total = block;
        if (blocks > 1) {
            exchange(block, 0);
            total = 0;
            for (int r = 0; r < blocks; ++r) {
                if (r == rank) at += total;
                total += sh.xch[parity ^ 1][r][0];
            }
        }
        const i64 want = target(total);
        if (at <= want && want < at + mine) {
            const int i = __ffs(__ballot_sync(0xffffffffu, want < at + strips)) - 1, v = v0 + i * 32 + lane;
            const i64 s = of_vec(v);
            i64 upto = s;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const i64 t = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += t;
            }
            i64 sum = at + __shfl_sync(0xffffffffu, strips - strip, i) + upto - s;
            if (sum <= want && want < sum + s) {
                const uint4 x = data[v];
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const int index = first + v * N + e;
                    const i64 one = f(Elements<T>::get(x, e), index);
                    if (sum <= want && want < sum + one) {
                        for (int r = 0; r < blocks; ++r) *(blocks > 1 ? cluster.map_shared_rank(&sh.index, r) : &sh.index) = index;
                    }
                    sum += one;
                }
            }
        }
        sync();
    }

    __device__ __forceinline__ void answer(int d, int token, float prob) const {
        p.token[d] = token;
        if (p.prob) p.prob[d] = prob;
    }
    static __device__ __forceinline__ i64 drawn(float u, i64 all) {
        const double x = u < 0.f ? 0.0 : (double)u;
        return x >= 1.0 ? all - 1 : min(all - 1, (i64)(x * (double)all));
    }
    static __device__ __forceinline__ i64 share(float top_p, i64 all) {
        const i64 want = (i64)ceil((double)top_p * (double)all);
        return want < 1 ? 1 : want;
    }

    // Few candidates, those in front of the order among them: the rest of the filters and the draw, by the first block.  all: the weight that top-p is a share of, or
    // (negative) that of the first top_k.
    __device__ __forceinline__ void finish(int d, int n, int top_k, float top_p, float least, float u, i64 all) {
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) sh.all[i].w = weight(sh.all[i].x);
        __syncthreads();
        // rank and weight in front, kept in sh.mine
        pairs(n, [&](int i, int j, i64& a, int& b) {
            if (in_front(sh.all[j], sh.all[i])) {
                a += sh.all[j].w;
                ++b;
            }
        }, [&](int i, i64 a, int b) { sh.mine[i] = {0.f, b, a}; });
        __syncthreads();
        if (all < 0) {
            i64 a = 0, b = 0;
            for (int i = threadIdx.x; i < n; i += kThreads)
                if (sh.mine[i].index < top_k) a += sh.all[i].w;
            block_sum(a);
            all = a;
        }
        const i64 want = top_p < 1.f ? share(top_p, all) : all + 1;
        i64 kept = 0;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            if (sh.mine[i].index >= top_k || sh.mine[i].w >= want || !(sh.all[i].x >= least)) sh.all[i].w = 0;
            kept += sh.all[i].w;
        }
        block_sum(kept);
        const i64 r = drawn(u, kept);
        pairs(n, [&](int i, int j, i64& a, int&) {
            if (sh.all[j].index < sh.all[i].index) a += sh.all[j].w;
        }, [&](int i, i64 a, int) {
            if (a <= r && r < a + sh.all[i].w) answer(d, sh.all[i].index, (float)(power(power_of(sh.all[i].x)) / (double)kept));
        });
    }
    __device__ __forceinline__ void block_sum(i64& a) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        __syncthreads();
        if (lane == 0) sh.red[0][warp] = a;
        __syncthreads();
        a = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) a += sh.red[0][w];
    }

    // Top-p over the whole row: the bucket in which the weights reach `want` = top_p of all of them (`total`).
    __device__ __forceinline__ Found by_weight(float top_p, i64& want, i64& total) {
        histogram<false>(-INFINITY, [&](float x, int& b) { return bucket_of(x, b); });
        // Between b - 1/2 and b + 1/2 buckets from the largest, n tokens weigh n 2^(-b width) to within half a bucket; the sums below are in units of 2^44 and
        // rounded by far less than the rest of a bucket that is added.
        constexpr int each_has = kBuckets / kThreads;
        constexpr float width = kRange / ((float)kBuckets - 0.5f);
        float most = 0.f, least = 0.f, up[each_has], down[each_has];
#pragma unroll
        for (int i = 0; i < each_has; ++i) {
            const int b = threadIdx.x * each_has + i;
            i64 n, w;
            bucket_sums<false>(b, n, w);
            up[i] = (float)n * exp2f(-((float)b - 0.75f) * width);
            down[i] = (float)n * exp2f(-((float)b + 0.75f) * width);
            most += up[i];
            least += down[i];
        }
        float a = most, z = least;          // up to and with this thread
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const float s = __shfl_up_sync(0xffffffffu, a, o), t = __shfl_up_sync(0xffffffffu, z, o);
            if (lane >= o) { a += s; z += t; }
        }
        __syncthreads();
        if (lane == 31) { sh.red[0][warp] = __float_as_uint(a); sh.red[1][warp] = __float_as_uint(z); }
        if (threadIdx.x == 0) { sh.window[0] = kBuckets; sh.window[1] = kBuckets; }
        __syncthreads();
        float all_most = 0.f, all_least = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) { a += all_most; z += all_least; }
            all_most += __uint_as_float((uint32_t)sh.red[0][w]);
            all_least += __uint_as_float((uint32_t)sh.red[1][w]);
        }
        a -= most;
        z -= least;
#pragma unroll
        for (int i = 0; i < each_has; ++i) {        // the first bucket that may reach it, and the first that surely has
            a += up[i];
            z += down[i];
            if (a * 1.0001f >= top_p * all_least) atomicMin(&sh.window[0], (int)threadIdx.x * each_has + i);
            if (z >= top_p * all_most * 1.0001f) atomicMin(&sh.window[1], (int)threadIdx.x * each_has + i);
        }
        __syncthreads();
        const bool bounded = bucket_scale < 3e38f;      // else the buckets are wider than that
        const int b0 = bounded ? sh.window[0] : 0, b1 = bounded ? sh.window[1] : kBuckets;
        i64 above = 0, all = 0;
        each([&](float x, int) {
            int b;
            if (bucket_of(x, b)) {
                const i64 w = weight(x);
                all += w;
                if (b < b0) above += w;
                else if (b <= b1 && w) add_weight(b, w);
            }
        });
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            all += __shfl_xor_sync(0xffffffffu, all, o);
            above += __shfl_xor_sync(0xffffffffu, above, o);
        }
        __syncthreads();
        if (lane == 0) { sh.red[0][warp] = all; sh.red[1][warp] = above; }
        __syncthreads();
        all = above = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) { all += sh.red[0][w]; above += sh.red[1][w]; }
        if (blocks > 1) {
            exchange(all, above);
            all = above = 0;
            for (int r = 0; r < blocks; ++r) { all += sh.xch[parity ^ 1][r][0]; above += sh.xch[parity ^ 1][r][1]; }
        }
        total = all;
        want = share(top_p, all);
        i64 in_window;
        Found f = find<true>([&](i64) { return want - above; }, in_window);
        f.before += above;
        return f;
    }

    // The smallest logit whose weight is at least min_p, the largest among them always
    __device__ __forceinline__ float least_of(float min_p) const {
        if (!(min_p > 0.f)) return -INFINITY;
        const double log_p = log2((double)min_p);
        if (log_p >= 0.0) return top;
        if (c == 0.0) return -3.402823466e38f;
        auto in = [&](float x) { return ((double)x - (double)top) * c >= log_p; };
        float x = (float)fmax((double)top + log_p / c, -3.4028234663852886e38);
        while (in(x) && x > -3.402823466e38f) x = value_of(key_of(x) - 1);
        while (!in(x)) x = value_of(key_of(x) + 1);
        return fminf(x, top);
    }

    __device__ __forceinline__ void run(uint4* store) {
        const int d = blockIdx.x / blocks, row = p.row ? p.row[d] : d, V = p.vocab;
        if (row < 0) return;
        const float temp = p.temperature ? p.temperature[d] : 1.f, top_p = p.top_p ? p.top_p[d] : 1.f, min_p = p.min_p ? p.min_p[d] : 0.f, u = p.u[d];
        int top_k = p.top_k ? p.top_k[d] : 0;
        bool bad = row >= p.logit_rows || !(temp >= 0.f) || isnan(top_p) || isnan(min_p) || isnan(u);
        cg::cluster_group::arrival_token started;
        if (blocks > 1) started = cluster.barrier_arrive();
        if (threadIdx.x < 64) sh.table[threadIdx.x] = exp2((double)threadIdx.x / 64.0);
        // this block's vectors: of 16 bytes on their grid; what of them lies outside the row counts as -inf
        const bool unseen = bad;
        float own = -INFINITY;              // this thread's largest
        if (!bad) {
            const T* const x = (const T*)p.logits + row * p.ld;
            const int shift = (int)(((uintptr_t)x & 15) / sizeof(T)), all_vecs = (shift + V + N - 1) / N, per = (all_vecs + blocks - 1) / blocks;
            const int v0 = min(all_vecs, rank * per);
            vecs = min(per, all_vecs - v0);
            first = v0 * N - shift;
            const uint4* const from = reinterpret_cast<const uint4*>(x - shift) + v0;
            constexpr int kAtOnce = 8;
            for (int va = threadIdx.x; va < vecs; va += kThreads * kAtOnce) {
                uint4 w[kAtOnce];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const int v = va + k * kThreads, i = first + v * N;
                    if (v < vecs) {
                        if (i >= 0 && i + N <= V) {
                            w[k] = __ldcg(from + v);
                        } else {
                            uint32_t y[4] = {0, 0, 0, 0};
#pragma unroll
                            for (int e = 0; e < N; ++e) {
                                const bool there = i + e >= 0 && i + e < V;
                                if (sizeof(T) == 4) y[e] = there ? reinterpret_cast<const uint32_t*>(x)[i + e] : 0xFF800000u;
                                else y[e / 2] |= (there ? (uint32_t)reinterpret_cast<const uint16_t*>(x)[i + e] : 0xFF80u) << (16 * (e & 1));
                            }
                            w[k] = make_uint4(y[0], y[1], y[2], y[3]);
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const int v = va + k * kThreads;
                    if (v < vecs) {
                        store[v] = w[k];
                        own = max_nan(own, Elements<T>::top(w[k]));
                    }
                }
            }
            top = own;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (lane == 0) sh.red[0][warp] = __float_as_uint(top);
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = max_nan(top, __uint_as_float((uint32_t)sh.red[0][w]));
            if (blocks > 1) {
                cluster.barrier_wait(std::move(started));       // the others' shared memory is there
                exchange(__float_as_uint(top), 0);
                for (int r = 0; r < blocks; ++r) top = max_nan(top, __uint_as_float((uint32_t)sh.xch[parity ^ 1][r][0]));
            }
            bad = !(top < INFINITY) || top == -INFINITY;
        }
        if (bad) {
            if (threadIdx.x == 0 && rank == 0) {
                answer(d, -1, 0.f);
                report(p.d_status, CATS_ERR_INVALID_ARG);
            }
            if (blocks > 1 && unseen) cluster.barrier_wait(std::move(started));
            return;
        }
        i64 total;
        if (temp == 0.f) {
            walk([&](float x, int) { return (i64)(x == top); }, [](i64) { return (i64)0; }, total);
            if (threadIdx.x == 0 && rank == 0) answer(d, sh.index, 1.f);
            return;
        }
        c = 1.4426950408889634074 / (double)temp;
        bucket_scale = (float)fmin(2.0 * c * ((double)kBuckets - 0.5) / (double)kRange, 3e38);
        const float least = least_of(min_p);
        auto weighed = [&](float x, int& b) { return bucket_of(x, b); };
        uint32_t tau = 0;               // kept: keys above tau, and at tau the ones up to index `last`
        i64 ties = -1;                  // how many at tau; -1: all
        int same = 0;
        bool by_k = top_k > 0 && top_k < V;
        if (by_k && top_k <= kFewK) {
            int b;
            clear();
            if (bucket_of(own, b)) atomicAdd(&sh.cnt[b], 1u);
            sync();
            const Found f = find<false>([&](i64) { return (i64)top_k; }, total);
            if (f.bucket >= 0) {        // half a bucket and what fp32 rounds below its end
                const float x0 = (top - ((float)f.bucket + 1.f) * 2.f / bucket_scale) - fabsf(top) * 2e-7f;
                const int n = gather(true, x0, [](float) { return true; });
                if (n <= kFew) {
                    if (rank == 0) finish(d, n, top_k, top_p, least, u, -1);
                    return sync();
                }
            }
        }
        if (by_k) {
            histogram<false>(-INFINITY, [&](float x, int& b) { return bucket_of(x, b); });
            const Found f = find<false>([&](i64) { return (i64)top_k; }, total);
            by_k = f.bucket >= 0;       // else fewer than top_k weigh anything
            if (by_k && f.count_before + f.count <= kFew) {
                const int n = gather(true, -INFINITY, [&](float x) { int b; return bucket_of(x, b) && b <= f.bucket; });
                if (rank == 0) finish(d, n, top_k, top_p, least, u, -1);
                return sync();
            }
            if (by_k) {
                threshold<false>(f, top_k, weighed);
                tau = sh.tau;
                ties = top_k - sh.above;
                same = sh.same;
            }
        }
        if (top_p < 1.f) {
            const i64 at_tau = by_k ? ties * weight(value_of(tau)) : 0;
            i64 want = 0;
            Found f;
            if (by_k) {                 // few tokens
                histogram<true>(value_of(tau), [&](float x, int& b) { return bucket_of(x, b) && key_of(x) > tau; });
                f = find<true>([&](i64 above) { return want = share(top_p, above + at_tau); }, total);
            } else {
                f = by_weight(top_p, want, total);
            }
            if (f.bucket >= 0 && f.count_before + f.count <= kFew) {
                const int n = gather(true, -INFINITY, [&](float x) { int b; return bucket_of(x, b) && key_of(x) > tau && b <= f.bucket; });
                if (rank == 0) finish(d, n, INT_MAX, top_p, least, u, total + at_tau);
                return sync();
            }
            if (f.bucket >= 0) {
                threshold<true>(f, want, [&](float x, int& b) { return bucket_of(x, b) && key_of(x) > tau; });
                tau = sh.tau;
                const i64 w = weight(value_of(tau));
                ties = (want - sh.above + w - 1) / w;
                same = sh.same;
            } else {                    // inside the tokens at the threshold of top-k
                const i64 w = weight(value_of(tau));
                ties = (want - total + w - 1) / w;
            }
        }
        if (least > -INFINITY && key_of(least) > tau) {
            tau = key_of(least);
            ties = -1;
        }
        int last = INT_MAX;
        if (ties >= 0 && ties < same) {
            walk([&](float x, int) { return (i64)(key_of(x) == tau); }, [&](i64) { return ties - 1; }, total);
            last = sh.index;
            sync();
        }
        walk([&](float x, int index) {
            const uint32_t k = key_of(x);
            return k > tau || (k == tau && index <= last) ? weight(x) : (i64)0;
        }, [&](i64 all) { return drawn(u, all); }, total);
        if (threadIdx.x == 0 && rank == 0) {
            const int i = sh.index;
            const T v = ((const T*)p.logits + row * p.ld)[i];
            const float x = sizeof(T) == 4 ? *reinterpret_cast<const float*>(&v) : __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(&v) << 16);
            answer(d, i, (float)(power(power_of(x)) / (double)total));
        }
    }
};

template <typename T> __global__ void __launch_bounds__(kThreads, 2) k_sample(const __grid_constant__ SampleDev p) {
    __shared__ __align__(16) typename Row<T>::Shared sh;
    extern __shared__ __align__(16) uint4 data[];
    pdl_launch_dependents();
    pdl_wait();
    Row<T>(p, sh, data).run(data);
}

template <typename T> cudaError_t launch_t(const SampleDev& p, cudaStream_t st) {
    constexpr int kMost = 200 * 1024, kUsual = 88 * 1024;      // bytes of a row per block: what fits, and with what two share an SM
    const long long bytes = (long long)p.vocab * sizeof(T) + 32;
    int blocks = (int)min((long long)kMaxBlocks, (bytes + kUsual - 1) / kUsual);
    while (blocks < kMaxBlocks && (long long)p.rows * (blocks + 1) <= 148 && bytes / blocks > 16 * 1024) ++blocks;      // SMs that no row has
    const size_t smem = (size_t)((bytes / 16 + 2 + blocks - 1) / blocks) * 16;
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

cudaError_t launch_sample(const SampleDev& p, cudaStream_t st) { return p.f32 ? launch_t<float>(p, st) : launch_t<uint16_t>(p, st); }

}  // namespace cats
