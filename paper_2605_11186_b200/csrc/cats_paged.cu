// Rows into and out of the paged cache (include/cats.h: cats_paged_append, cats_paged_read).
//
// Append, per row and head: y = R(pos) k (rotate-half pairs (i, i + hd / 2), angle pos base^(-2i/hd)), rounded to bf16, or held as
//   a = max(max|y|, 2^-100),   q = rint(127 y / a),   scale = a / 127,
// a head that holds an infinity or a NaN as zeros with a NaN scale.  Queries are rotated and rounded to bf16 in the same pass.
// Read: the same rows back, q scale.  Both move every byte once: bound by HBM for a prompt, by latency for a token.
#include <math.h>

#include "cats_i8.cuh"
#include "cats_paged.cuh"

namespace cats {
namespace {

struct Frequencies { double turns[64]; };       // turns per position of each pair: base^(-2i/hd) / 2 pi

// Eight values from p on, as fp32.  VEC: p on the 16-byte grid.
template <bool VEC> __device__ __forceinline__ void load8(const float* p, float* v) {
    if (VEC) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p[i];
    }
}
template <bool VEC> __device__ __forceinline__ void load8(const uint16_t* p, float* v) {
    if (VEC) {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = bf16_bits_to_float(p[i]);
    }
}
template <bool VEC> __device__ __forceinline__ void store8(float* p, const float* v) {
    if (VEC) {
        reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = v[i];
    }
}
template <bool VEC> __device__ __forceinline__ void store8(uint16_t* p, const float* v) {
    if (VEC) {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = float_to_bf16_bits(v[i]);
    }
}

// cos and sin of `turns` whole turns.  Reduced to an eighth of a turn to either side of a multiple of a quarter in fp64, so that what
// fp32 rounds is small: off by less than 2^-22 at any position.
__device__ __forceinline__ float2 cos_sin_turns(double turns) {
    const double quarters = 4.0 * (turns - rint(turns));
    const double n = rint(quarters);
    float s, c;
    sincospif(0.5f * (float)(quarters - n), &s, &c);
    const int k = (int)n & 3;
    if (k & 1) { const float t = c; c = -s; s = t; }
    return k & 2 ? make_float2(-c, -s) : make_float2(c, s);
}

constexpr int kThreads = 256;

// Blocks of a row (blockIdx.y).  HD / 16 threads hold a head, each 8 elements of its first half and the 8 that they are rotated with; heads in
// the order K, V, queries.  A thread's input is requested before the position is known: position, page and angles are three more trips
// one behind the other (8191 rows of 96 heads with the reading back: 230 us when a block held a row and asked for them first).
template <typename T, bool VEC, int HD, bool I8>
__global__ void __launch_bounds__(kThreads) k_paged_append(const __grid_constant__ PagedDev c, const __grid_constant__ PagedRows r, const __grid_constant__ Frequencies f, int rotate) {
    constexpr int HALF = HD / 2, TH = HD / 16;
    __shared__ __align__(16) float cos_s[HALF], sin_s[HALF];
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x, units = (r.n_heads + 2 * c.n_kv) * TH, u = blockIdx.y * kThreads + threadIdx.x, unit = min(u, units - 1);
    const int head = unit / TH, e = (unit % TH) * 8;
    const int which = head < c.n_kv ? 0 : (head < 2 * c.n_kv ? 1 : 2), h = which == 2 ? head - 2 * c.n_kv : head - which * c.n_kv;
    const T* const x = (which == 0 ? (const T*)r.k + row * r.ldk : (which == 1 ? (const T*)r.v + row * r.ldv : (const T*)r.q + row * r.ldq)) + (size_t)h * HD + e;
    float lo[8], hi[8];
    load8<VEC>(x, lo);
    load8<VEC>(x + HALF, hi);
    const int pos = r.pos[row];
    if (pos < 0) return;
    PagedDev::Row at;
    if (!c.locate(r.seq ? r.seq[row] : row, pos, at)) {
        if (threadIdx.x == 0) report(r.d_status, CATS_ERR_INVALID_ARG);
        return;
    }
    if (rotate) {
        if ((int)threadIdx.x < HALF) {
            const float2 cs = cos_sin_turns((double)pos * f.turns[threadIdx.x]);
            cos_s[threadIdx.x] = cs.x;
            sin_s[threadIdx.x] = cs.y;
        }
        __syncthreads();
        if (which != 1) {
            float cs[8], sn[8];
            load8<true>(cos_s + e, cs);
            load8<true>(sin_s + e, sn);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float a = lo[i], b = hi[i];
                lo[i] = a * cs[i] - b * sn[i];
                hi[i] = b * cs[i] + a * sn[i];
            }
        }
    }
    if (which == 2) {
        if (u < units) {
            uint16_t* const o = r.q_out + row * r.ldqo + (size_t)h * HD + e;
            store8<VEC>(o, lo);
            store8<VEC>(o + HALF, hi);
        }
    } else if (!I8) {
        uint16_t* const o = reinterpret_cast<uint16_t*>((which ? c.v : c.k) + ((size_t)at.at + (size_t)h * c.head16) * 16) + e;
        if (u < units) {
            store8<true>(o, lo);
            store8<true>(o + HALF, hi);
        }
    }
    if (I8) {
        uint32_t mx = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) mx = max(mx, max(abs_bits(lo[i]), abs_bits(hi[i])));
#pragma unroll
        for (int o = TH / 2; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        if (which != 2 && u < units) {
            const bool finite = mx < 0x7F800000u;
            const float a = fmaxf(__uint_as_float(mx), kTinyMax);
            const Factor by = factor_127_over(finite ? a : 1.f);
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float v = !finite ? 0.f : (i < 2 ? lo[4 * i + j] : hi[4 * (i - 2) + j]);
                    b[j] = __float_as_uint(__fadd_rn(fmaf(v, by.hi, __fmul_rn(v, by.lo)), kRintMagic));
                }
                w[i] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
            }
            uint8_t* const o = (which ? c.v : c.k) + ((size_t)at.at + (size_t)h * c.head16) * 16 + e;
            *reinterpret_cast<uint2*>(o) = make_uint2(w[0], w[1]);
            *reinterpret_cast<uint2*>(o + HALF) = make_uint2(w[2], w[3]);
            if (e == 0) (which ? c.vs : c.ks)[(size_t)at.s + (size_t)h * c.s_head] = finite ? a / 127.f : __int_as_float(0x7FC00000);
        }
    }
}

// A block per row; a thread takes 16 bytes of kEach heads of the cache at a time, all requested before the first is used.  (One or two at a time: 82 us for
// 16384 rows of 32 int8 heads; position, page and rows are three trips one behind the other, so much has to be on its way at once.)
template <typename T, bool VEC, int HD, bool I8>
__global__ void __launch_bounds__(kThreads) k_paged_read(const __grid_constant__ PagedDev c, const __grid_constant__ PagedRows r) {
    constexpr int N = I8 ? 16 : 8, TH = HD / N, kEach = 4;
    pdl_launch_dependents();
    pdl_wait();
    const int row = blockIdx.x, pos = r.pos[row];
    if (pos < 0) return;
    PagedDev::Row at;
    if (!c.locate(r.seq ? r.seq[row] : row, pos, at)) {
        if (threadIdx.x == 0) report(r.d_status, CATS_ERR_INVALID_ARG);
        return;
    }
    const int units = 2 * c.n_kv * TH;
    for (int u0 = threadIdx.x; u0 < units; u0 += blockDim.x * kEach) {
        uint4 w[kEach];
        float s[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int u = u0 + k * blockDim.x;
            if (u < units) {
                const int head = u / TH, which = head >= c.n_kv, h = head - which * c.n_kv;
                w[k] = __ldcg(reinterpret_cast<const uint4*>(which ? c.v : c.k) + (size_t)at.at + (size_t)h * c.head16 + u % TH);
                if (I8) s[k] = __ldcg((which ? c.vs : c.ks) + (size_t)at.s + (size_t)h * c.s_head);
            }
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int u = u0 + k * blockDim.x;
            if (u >= units) break;
            const int head = u / TH, which = head >= c.n_kv, h = head - which * c.n_kv;
            T* const o = (which ? (T*)r.v_out + row * r.ldv : (T*)r.k_out + row * r.ldk) + (size_t)h * HD + u % TH * N;
            const uint32_t x[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
            float v[N];
            if (I8) {
#pragma unroll
                for (int i = 0; i < N; ++i)      // a byte b as the float 2^23 + (b + 128), then minus 2^23 + 128: exact
                    v[i] = (__uint_as_float(__byte_perm(x[i >> 2] ^ 0x80808080u, 0x4B000000u, 0x7440u + (i & 3))) - 8388736.f) * s[k];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[2 * i] = __uint_as_float(x[i] << 16);
                    v[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
                }
            }
#pragma unroll
            for (int i = 0; i < N; i += 8) store8<VEC>(o + i, v + i);
        }
    }
}

// Whether rows of `p` start on 16 bytes, every one.
bool on_grid(const void* p, long long ld, int size) { return (uintptr_t)p % 16 == 0 && (ld * size) % 16 == 0; }

// The frequencies of the thread's last call: 64 calls of pow() take longer than the kernel.
const Frequencies& frequencies(float base, int hd) {
    thread_local float last_base = 0.f;
    thread_local int last_hd = 0;
    thread_local Frequencies f;
    if (base != last_base || hd != last_hd) {
        for (int i = 0; i < hd / 2; ++i) f.turns[i] = pow((double)base, -2.0 * i / hd) / 6.283185307179586476925;
        last_base = base;
        last_hd = hd;
    }
    return f;
}

template <typename T, bool VEC, int HD, bool I8>
cudaError_t append_k(const PagedDev& c, const PagedRows& r, cudaStream_t st) {
    const int units = (r.n_heads + 2 * c.n_kv) * (HD / 16);
    static const Frequencies none = {};
    return launch_i8(k_paged_append<T, VEC, HD, I8>, dim3((unsigned)r.rows, (unsigned)((units + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, c, r, r.rope_base > 0.f ? frequencies(r.rope_base, HD) : none,
                     r.rope_base > 0.f ? 1 : 0);
}
template <typename T, bool VEC> cudaError_t append_t(const PagedDev& c, const PagedRows& r, int i8, int hd, cudaStream_t st) {
    if (hd == 128) return i8 ? append_k<T, VEC, 128, true>(c, r, st) : append_k<T, VEC, 128, false>(c, r, st);
    return i8 ? append_k<T, VEC, 64, true>(c, r, st) : append_k<T, VEC, 64, false>(c, r, st);
}
template <typename T, bool VEC, int HD, bool I8> cudaError_t read_k(const PagedDev& c, const PagedRows& r, cudaStream_t st) {
    const int units = 2 * c.n_kv * (HD / (I8 ? 16 : 8));
    return launch_i8(k_paged_read<T, VEC, HD, I8>, dim3((unsigned)r.rows), dim3(min(kThreads, (units + 127) / 128 * 32)), 0, st, c, r);
}
template <typename T, bool VEC> cudaError_t read_t(const PagedDev& c, const PagedRows& r, int i8, int hd, cudaStream_t st) {
    if (hd == 128) return i8 ? read_k<T, VEC, 128, true>(c, r, st) : read_k<T, VEC, 128, false>(c, r, st);
    return i8 ? read_k<T, VEC, 64, true>(c, r, st) : read_k<T, VEC, 64, false>(c, r, st);
}

}  // namespace

cudaError_t launch_paged_append(const PagedDev& c, const PagedRows& r, int i8, int hd, cudaStream_t st) {
    const int size = r.f32 ? 4 : 2;
    const bool vec = on_grid(r.k, r.ldk, size) && on_grid(r.v, r.ldv, size) && (r.n_heads == 0 || (on_grid(r.q, r.ldq, size) && on_grid(r.q_out, r.ldqo, 2)));
    if (r.f32) return vec ? append_t<float, true>(c, r, i8, hd, st) : append_t<float, false>(c, r, i8, hd, st);
    return vec ? append_t<uint16_t, true>(c, r, i8, hd, st) : append_t<uint16_t, false>(c, r, i8, hd, st);
}
cudaError_t launch_paged_read(const PagedDev& c, const PagedRows& r, int i8, int hd, cudaStream_t st) {
    const int size = r.f32 ? 4 : 2;
    const bool vec = on_grid(r.k_out, r.ldk, size) && on_grid(r.v_out, r.ldv, size);
    if (r.f32) return vec ? read_t<float, true>(c, r, i8, hd, st) : read_t<float, false>(c, r, i8, hd, st);
    return vec ? read_t<uint16_t, true>(c, r, i8, hd, st) : read_t<uint16_t, false>(c, r, i8, hd, st);
}

}  // namespace cats
