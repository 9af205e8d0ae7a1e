// One token per row of logits (include/cats.h: cats_sample).
//
// Tokens are ordered by falling logit, equal ones by rising index; top-k, top-p and min-p each keep a run from the front of
// that order, so what is kept is: every token whose key is above a threshold, and the first few (by index) of those at it.
// w = exp((x - max) / T) is a whole multiple of 2^-44, taken from an fp64 exponential: the sums are exact 64-bit integers, the same in any
// order, and so are all decisions made from them.  (vocab <= 2^18, so no sum reaches 2^63.)
// A block per row; thresholds by bisection over the keys, every step a pass over the row.
#include "cats_kernels.cuh"

namespace cats {
namespace {

typedef long long i64;
constexpr int kThreads = 1024;

// Keys in the order of the logits; -0 as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

__device__ __forceinline__ i64 weight(float x, float top, double c) {
    if (x == -INFINITY) return 0;
    const double t = ((double)x - (double)top) * c;
    return t < -46.0 ? 0 : __double2ll_rn(exp2(t + 44.0));
}

template <typename F> __device__ __forceinline__ i64 block_sum(F f, int n, i64* red) {
    i64 s = 0;
    for (int i = threadIdx.x; i < n; i += kThreads) s += f(i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    s = red[threadIdx.x & 31];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

// Sum of v over the threads before this one
__device__ __forceinline__ i64 block_before(i64 v, i64* red) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    i64 s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const i64 t = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += t;
    }
    __syncthreads();
    if (lane == 31) red[warp] = s;
    __syncthreads();
    i64 before = 0;
    for (int w = 0; w < warp; ++w) before += red[w];
    return before + s - v;
}

template <typename T> __global__ void __launch_bounds__(kThreads) k_sample(const SampleDev p) {
    __shared__ i64 red[32];
    pdl_launch_dependents();
    pdl_wait();
    const int d = blockIdx.x, row = p.row ? p.row[d] : d, V = p.vocab;
    if (row < 0) return;
    auto refuse = [&] {
        if (threadIdx.x == 0) {
            p.token[d] = -1;
            if (p.prob) p.prob[d] = 0.f;
            report(p.d_status, CATS_ERR_INVALID_ARG);
        }
    };
    const float temp = p.temperature ? p.temperature[d] : 1.f, top_p = p.top_p ? p.top_p[d] : 1.f, min_p = p.min_p ? p.min_p[d] : 0.f, u = p.u[d];
    const int top_k = p.top_k ? p.top_k[d] : 0;
    if (row >= p.logit_rows || !(temp >= 0.f) || isnan(top_p) || isnan(min_p) || isnan(u)) return refuse();
    const T* const x = (const T*)p.logits + row * p.ld;
    auto value = [&](int i) { return sizeof(T) == 4 ? (float)x[i] : __uint_as_float((uint32_t)x[i] << 16); };
    // key and lowest index of the largest, and whether anything is NaN or +inf
    i64 best = 0;
    int bad = 0;
    for (int i = threadIdx.x; i < V; i += kThreads) {
        const float v = value(i);
        bad |= !(v < INFINITY);
        best = max(best, ((i64)key_of(v) << 20) | (i64)(0xFFFFF - i));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = best;
    if (__syncthreads_or(bad)) return refuse();
    best = red[threadIdx.x & 31];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    const uint32_t top_key = (uint32_t)(best >> 20);
    const float top = value_of(top_key);
    if (top == -INFINITY) return refuse();
    if (temp == 0.f) {
        if (threadIdx.x == 0) {
            p.token[d] = 0xFFFFF - (int)(best & 0xFFFFF);
            if (p.prob) p.prob[d] = 1.f;
        }
        return;
    }
    const double c = 1.4426950408889634074 / (double)temp;
    uint32_t at = 0;                // kept: keys above `at`, and the first `ties` tokens of key `at`
    i64 ties = V;
    if (top_k > 0 && top_k < V) {
        uint32_t lo = 0, hi = top_key;      // the largest key that top_k tokens reach
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo + 1) / 2;
            if (block_sum([&](int i) { return (i64)(key_of(value(i)) >= mid); }, V, red) >= top_k) lo = mid;
            else hi = mid - 1;
        }
        at = lo;
        ties = top_k - block_sum([&](int i) { return (i64)(key_of(value(i)) > lo); }, V, red);
    }
    const i64 above_k = block_sum([&](int i) { return key_of(value(i)) > at ? weight(value(i), top, c) : 0; }, V, red);
    i64 same_k = block_sum([&](int i) { return (i64)(key_of(value(i)) == at); }, V, red);
    ties = min(ties, same_k);
    if (top_p < 1.f) {
        const i64 all = above_k + ties * weight(value_of(at), top, c);
        i64 want = (i64)ceil((double)top_p * (double)all);
        want = want < 1 ? 1 : want;
        uint32_t lo = at, hi = top_key;     // the largest key from which on the weights reach `want`
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo + 1) / 2;
            if (block_sum([&](int i) { return key_of(value(i)) >= mid ? weight(value(i), top, c) : 0; }, V, red) >= want) lo = mid;
            else hi = mid - 1;
        }
        const i64 above = block_sum([&](int i) { return key_of(value(i)) > lo ? weight(value(i), top, c) : 0; }, V, red);
        const i64 w = weight(value_of(lo), top, c);
        const i64 n = w > 0 ? (want - above + w - 1) / w : ties;
        if (lo > at) ties = n;
        else ties = min(ties, n);
        at = lo;
    }
    if (min_p > 0.f) {
        const double least = log2((double)min_p);
        auto in = [&](uint32_t key) { return ((double)value_of(key) - (double)top) * c >= least || key == top_key; };
        uint32_t lo = at, hi = top_key;     // the smallest key that is in
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (in(mid)) hi = mid;
            else lo = mid + 1;
        }
        if (lo > at) { at = lo; ties = V; }
    }
    // in index order: each thread a run of tokens
    const int run = (V + kThreads - 1) / kThreads, i0 = min(V, (int)threadIdx.x * run), i1 = min(V, i0 + run);
    i64 same = 0;
    for (int i = i0; i < i1; ++i) same += key_of(value(i)) == at;
    i64 left = ties - block_before(same, red);
    auto kept = [&](int i, i64& rest) -> i64 {
        const uint32_t k = key_of(value(i));
        if (k < at || (k == at && rest-- <= 0)) return 0;
        return weight(value(i), top, c);
    };
    i64 mine = 0, rest = left;
    for (int i = i0; i < i1; ++i) mine += kept(i, rest);
    const i64 before = block_before(mine, red);
    __syncthreads();
    if (threadIdx.x == kThreads - 1) red[0] = before + mine;
    __syncthreads();
    const i64 all = red[0];
    const double uu = u < 0.f ? 0.0 : (double)u;
    const i64 r = uu >= 1.0 ? all - 1 : min(all - 1, (i64)(uu * (double)all));
    if (before <= r && r < before + mine) {
        i64 sum = before;
        rest = left;
        for (int i = i0; i < i1; ++i) {
            sum += kept(i, rest);
            if (sum > r) {
                p.token[d] = i;
                if (p.prob) p.prob[d] = (float)(exp2(((double)value(i) - (double)top) * c + 44.0) / (double)all);
                break;
            }
        }
    }
}

}  // namespace

cudaError_t launch_sample(const SampleDev& p, cudaStream_t st) {
    const dim3 grid((unsigned)p.rows);
    return p.f32 ? launch_i8(k_sample<float>, grid, dim3(kThreads), 0, st, p) : launch_i8(k_sample<uint16_t>, grid, dim3(kThreads), 0, st, p);
}

}  // namespace cats
