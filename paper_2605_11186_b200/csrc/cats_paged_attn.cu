// Attention of one new token per sequence over the paged cache (include/cats.h: cats_paged_attention):
//   out[s][h] = sum_t softmax_t(q[s][h] . k[t][g] scale) v[t][g],   g = h / (n_heads / n_kv_heads)
// A block per (sequence, query head); its warps take the rows in turn, one pass with a running maximum and sum each, and join at the end.
#include "cats_paged.cuh"

namespace cats {
namespace {

template <int HD, bool I8> __device__ __forceinline__ void row_values(const uint8_t* p, int lane, float* v) {
    constexpr int N = HD / 32;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = I8 ? (float)reinterpret_cast<const int8_t*>(p)[lane * N + i] : bf16_bits_to_float(reinterpret_cast<const uint16_t*>(p)[lane * N + i]);
}

template <int HD, bool I8> __global__ void __launch_bounds__(128) k_paged_attn(const PagedDev c, const PagedAttn a) {
    constexpr int N = HD / 32;
    __shared__ float m_s[4], l_s[4], o_s[4][HD];
    pdl_launch_dependents();
    pdl_wait();
    const int s = blockIdx.x, h = blockIdx.y, g = h / (a.n_heads / c.n_kv), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float scale = a.scale * 1.4426950408889634f;
    const long long most = (long long)c.width * c.page_size;
    const int asked = a.len[s], len = (int)min((long long)max(asked, 0), most);
    if (asked > most && threadIdx.x == 0 && h == 0) report(a.d_status, CATS_ERR_INVALID_ARG);
    float q[N], o[N], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        q[i] = bf16_bits_to_float(a.q[s * a.ldq + h * HD + lane * N + i]) * scale;
        o[i] = 0.f;
    }
    for (int t = warp; t < len; t += 4) {
        PagedDev::Row at;
        if (!c.locate(s, t, at)) {
            if (lane == 0) report(a.d_status, CATS_ERR_INVALID_ARG);
            continue;
        }
        const size_t off = ((size_t)at.at + (size_t)g * c.head16) * 16, so = (size_t)at.s + (size_t)g * c.s_head;
        float k[N], v[N], x = 0.f;
        row_values<HD, I8>(c.k + off, lane, k);
        row_values<HD, I8>(c.v + off, lane, v);
#pragma unroll
        for (int i = 0; i < N; ++i) x = fmaf(q[i], k[i], x);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        if (I8) x *= c.ks[so];
        const float m1 = fmaxf(m, x), base = m1 == -INFINITY ? 0.f : m1, keep = exp2f(m - base), p = exp2f(x - base);
        const float w = I8 ? p * c.vs[so] : p;
        l = l * keep + p;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = fmaf(w, v[i], o[i] * keep);
        m = m1;
    }
    if (lane == 0) { m_s[warp] = m; l_s[warp] = l; }
#pragma unroll
    for (int i = 0; i < N; ++i) o_s[warp][lane * N + i] = o[i];
    __syncthreads();
    if ((int)threadIdx.x < HD) {
        const float top = fmaxf(fmaxf(m_s[0], m_s[1]), fmaxf(m_s[2], m_s[3])), base = top == -INFINITY ? 0.f : top;
        float sum = 0.f, acc = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = exp2f(m_s[w] - base);
            sum += l_s[w] * f;
            acc += o_s[w][threadIdx.x] * f;
        }
        a.out[s * a.ldo + h * HD + threadIdx.x] = float_to_bf16_bits(len > 0 ? acc / sum : 0.f);
    }
}

}  // namespace

size_t paged_attn_workspace(int n_seqs, int n_heads, int n_kv, int hd) { return 1024; }

cudaError_t launch_paged_attn(const PagedDev& c, const PagedAttn& a, int i8, int hd, cudaStream_t st) {
    const dim3 grid((unsigned)c.n_seqs, (unsigned)a.n_heads);
    if (hd == 128) return i8 ? launch_i8(k_paged_attn<128, true>, grid, dim3(128), 0, st, c, a) : launch_i8(k_paged_attn<128, false>, grid, dim3(128), 0, st, c, a);
    return i8 ? launch_i8(k_paged_attn<64, true>, grid, dim3(128), 0, st, c, a) : launch_i8(k_paged_attn<64, false>, grid, dim3(128), 0, st, c, a);
}

}  // namespace cats
