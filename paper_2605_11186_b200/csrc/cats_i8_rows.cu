// Row kernels of the 8-bit integer path: every kernel makes rows y of fp32 values and leaves them as int8 with one scale
// per row,
//   a = max(max|y|, 2^-100),   q = rint(127 y / a),   scale = a / 127        (y ~ q * scale)
// where y is a bf16 or fp32 row itself (attention output, a weight matrix), silu(gate) * up, or the RMSNorm of the
// residual stream after the preceding projection's output has been added to it.  A row that holds an infinity or a NaN
// gets a NaN scale and zeros, so that whatever is computed from it is NaN too.
//
// Bound by HBM for many rows and by latency (one trip to memory, one block-wide reduction) for the few rows of a tree.
// A row is read once and stays in registers; the norm needs sum x^2 and max|x g|, which are independent of each other, so
// both go through ONE reduction: y = (x g) r with r > 0 has its maximum where |x g| has.  Maxima are taken on the bit
// patterns of |y| as unsigned integers: the order of finite values, with infinities and NaNs above them all.
#include "cats_kernels.cuh"

namespace cats {
namespace {

constexpr float kTinyMax = 7.888609052210118e-31f;    // 2^-100: the smallest maximum a scale is made from

template <typename T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float get(const float* p) { return __ldg(p); }
    static __device__ __forceinline__ void get8(const float* p, float* v) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};
template <> struct Elem<uint16_t> {     // bf16 bits
    static __device__ __forceinline__ float get(const uint16_t* p) { return bf16_bits_to_float(__ldg(p)); }
    static __device__ __forceinline__ void get8(const uint16_t* p, float* v) {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
};
template <typename T, int V> __device__ __forceinline__ void load_v(const T* p, float* v) {
    if (V == 8) Elem<T>::get8(p, v);
    else v[0] = Elem<T>::get(p);
}
// a residual or delta element that another thread of this launch never writes, but that may be overwritten in place by
// the same thread afterwards: plain loads, not the read-only path
template <int V> __device__ __forceinline__ void load_rw(const void* base, long long off, bool f32, float* v) {
    if (f32) {
        const float* p = (const float*)base + off;
        if (V == 8) {
            const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            v[0] = p[0];
        }
    } else {
        const uint16_t* p = (const uint16_t*)base + off;
        if (V == 8) {
            const uint4 a = *reinterpret_cast<const uint4*>(p);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        } else {
            v[0] = bf16_bits_to_float(p[0]);
        }
    }
}
template <int V> __device__ __forceinline__ void store_rw(void* base, long long off, bool f32, const float* v) {
    if (f32) {
        float* p = (float*)base + off;
        if (V == 8) {
            reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            p[0] = v[0];
        }
    } else {
        uint16_t* p = (uint16_t*)base + off;
        if (V == 8)
            *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
        else
            p[0] = float_to_bf16_bits(v[0]);
    }
}
// (y rs) inv and not y (rs inv): |y rs| <= a, so the result is finite and within 127 (1 + 2^-22) whatever rs and a are
template <int V> __device__ __forceinline__ void store_q(int8_t* p, const float* y, float rs, float inv) {
    if (V == 8) {
        uint32_t w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            w[h] = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[h] |= ((uint32_t)__float2int_rn(y[h * 4 + i] * rs * inv) & 0xFFu) << (8 * i);
        }
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
        p[0] = (int8_t)__float2int_rn(y[0] * rs * inv);
    }
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
// silu(g) u = g u / (1 + e^-g): for g -> -inf the quotient goes to -0 (e^-g reaches infinity), for g -> inf to g.
__device__ __forceinline__ float silu_mul(float g, float u) { return __fdividef(g, 1.f + __expf(-g)) * u; }

// One vector of the row at column c: the values y (before the norm's row factor) of this operator.
template <int OP, typename TX, int V>
__device__ __forceinline__ void row_values(const I8RowsDev& p, long long row, int c, float* y, float& ss, bool write_resid) {
    if (OP == I8_NORM) {
        float r[V], g[V];
        load_rw<V>(p.x, row * p.ldx + c, p.x_f32, r);
        load_v<uint16_t, V>((const uint16_t*)p.gain + c, g);
        if (p.delta != nullptr) {
            float d[V];
            load_rw<V>(p.delta, row * p.ldd + c, p.d_f32, d);
#pragma unroll
            for (int i = 0; i < V; ++i) r[i] += d[i];
        }
        if (write_resid && p.resid_out != nullptr) store_rw<V>(p.resid_out, row * p.ldo + c, p.x_f32, r);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            ss = fmaf(r[i], r[i], ss);
            y[i] = r[i] * g[i];
        }
    } else if (OP == I8_SWIGLU) {
        float g[V], u[V];
        load_v<TX, V>((const TX*)p.x + row * p.ldx + c, g);
        load_v<TX, V>((const TX*)p.x + row * p.ldx + p.cols + c, u);
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = silu_mul(g[i], u[i]);
    } else {
        load_v<TX, V>((const TX*)p.x + row * p.ldx + c, y);
    }
}

// NT threads per row.  NV > 0: the row fits NV vectors of V elements per thread and stays in registers.  NV == 0: any
// length; the row is read twice.  NT == 32: a block of 128 threads holds four rows, one per warp, and needs no barrier.
template <int OP, typename TX, int V, int NV, int NT>
__global__ void __launch_bounds__(NT == 32 ? 128 : NT) k_i8_rows(const I8RowsDev p) {
    __shared__ float red_s[32];
    __shared__ uint32_t red_m[32];
    pdl_launch_dependents();
    const long long row = NT == 32 ? (long long)blockIdx.x * 4 + (threadIdx.x >> 5) : (long long)blockIdx.x;
    const int tid = NT == 32 ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
    pdl_wait();
    if (NT == 32 && row >= p.rows) return;
    constexpr int NR = NV > 0 ? NV : 1;
    float y[NR][V];
    float ss = 0.f;
    uint32_t mx = 0;
    if (NV > 0) {
#pragma unroll
        for (int k = 0; k < NR; ++k) {
            const int c = (k * NT + tid) * V;
            if (c < p.cols) {
                row_values<OP, TX, V>(p, row, c, y[k], ss, true);
#pragma unroll
                for (int i = 0; i < V; ++i) mx = max(mx, abs_bits(y[k][i]));
            }
        }
    } else {
        for (int c = tid * V; c < p.cols; c += NT * V) {
            row_values<OP, TX, V>(p, row, c, y[0], ss, false);
#pragma unroll
            for (int i = 0; i < V; ++i) mx = max(mx, abs_bits(y[0][i]));
        }
    }
    mx = __reduce_max_sync(0xffffffffu, mx);
    if (OP == I8_NORM) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    }
    if (NT > 32) {
        if ((tid & 31) == 0) {
            red_m[tid >> 5] = mx;
            red_s[tid >> 5] = ss;
        }
        __syncthreads();
        const int nw = NT / 32, l = tid & 31;
        mx = l < nw ? red_m[l] : 0u;
        mx = __reduce_max_sync(0xffffffffu, mx);
        if (OP == I8_NORM) {
            ss = l < nw ? red_s[l] : 0.f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        }
    }
    float rs = 1.f;
    if (OP == I8_NORM) rs = rsqrtf(ss / (float)p.cols + p.eps);
    float a = __uint_as_float(mx) * rs;
    const bool finite = abs_bits(a) < 0x7F800000u;
    a = fmaxf(a, kTinyMax);
    const float inv = 127.f / a;
    if (!finite) rs = 0.f;
    if (tid == 0) p.scale[row] = finite ? a / 127.f : __int_as_float(0x7FC00000);
    int8_t* const q = p.q + row * p.ldq;
    if (NV > 0) {
#pragma unroll
        for (int k = 0; k < NR; ++k) {
            const int c = (k * NT + tid) * V;
            if (c < p.cols) {
                if (!finite)
#pragma unroll
                    for (int i = 0; i < V; ++i) y[k][i] = 0.f;
                store_q<V>(q + c, y[k], rs, inv);
            }
        }
    } else {
        for (int c = tid * V; c < p.cols; c += NT * V) {
            row_values<OP, TX, V>(p, row, c, y[0], ss, true);
            if (!finite)
#pragma unroll
                for (int i = 0; i < V; ++i) y[0][i] = 0.f;
            store_q<V>(q + c, y[0], rs, inv);
        }
    }
}

// q * scale, rounded to bf16 or as fp32.  One block per (row, 4096 columns); V elements per thread and step.
template <int V>
__global__ void __launch_bounds__(256) k_i8_dequantize(const int8_t* __restrict__ q, long long ldq, const float* __restrict__ scale,
                                                       int cols, void* __restrict__ out, int out_f32, long long ldo) {
    pdl_launch_dependents();
    pdl_wait();
    const long long row = blockIdx.x;
    const float s = __ldg(scale + row);
    const int c_end = min(cols, ((int)blockIdx.y + 1) * 4096);
#pragma unroll 2
    for (int c = blockIdx.y * 4096 + threadIdx.x * V; c < c_end; c += 256 * V) {
        float v[V];
        if (V == 8) {
            const uint2 w = __ldg(reinterpret_cast<const uint2*>(q + row * ldq + c));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i % V] = (float)(int8_t)(((i < 4 ? w.x : w.y) >> (8 * (i & 3))) & 0xFFu) * s;
        } else {
            v[0] = (float)q[row * ldq + c] * s;
        }
        store_rw<V>(out, row * ldo + c, out_f32 != 0, v);
    }
}

// The QKV projection's rows [3 * D] fp32 to what the tree attention reads: q rotated, bf16; k rotated and v appended to cache
// rows prefix_len + t (rotate-half pairs (i, i + hd / 2), angle pos[t] * base^(-2i/hd) in fp64 so that far positions lose
// nothing; every value is rounded once, from the unrounded sums).  One block per (node, eighth of the heads).
__global__ void __launch_bounds__(256) k_i8_qkv(const float* __restrict__ qkv, const int32_t* __restrict__ pos, int nh, int hd,
                                                float rope_base, int prefix_len, uint16_t* __restrict__ q, uint16_t* __restrict__ kc,
                                                uint16_t* __restrict__ vc) {
    __shared__ float2 cs[64];
    pdl_launch_dependents();
    pdl_wait();
    const int t = blockIdx.x, half = hd / 2, D = nh * hd;
    if ((int)threadIdx.x < half) {
        const double inv_freq = pow((double)rope_base, -2.0 * (double)threadIdx.x / (double)hd);
        double s, c;
        sincos((double)pos[t] * inv_freq, &s, &c);
        cs[threadIdx.x] = make_float2((float)c, (float)s);
    }
    __syncthreads();
    const float* const row = qkv + (size_t)t * 3 * D;
    const size_t cache_row = (size_t)(prefix_len + t) * D;
    const int pairs = nh * half;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < pairs; i += gridDim.y * 256) {
        const int h = i / half, r = i - h * half, lo = h * hd + r, hi = lo + half;
        const float2 f = cs[r];
        const float q0 = row[lo], q1 = row[hi], k0 = row[D + lo], k1 = row[D + hi];
        q[(size_t)t * D + lo] = float_to_bf16_bits(q0 * f.x - q1 * f.y);
        q[(size_t)t * D + hi] = float_to_bf16_bits(q1 * f.x + q0 * f.y);
        kc[cache_row + lo] = float_to_bf16_bits(k0 * f.x - k1 * f.y);
        kc[cache_row + hi] = float_to_bf16_bits(k1 * f.x + k0 * f.y);
        vc[cache_row + lo] = float_to_bf16_bits(row[2 * D + lo]);
        vc[cache_row + hi] = float_to_bf16_bits(row[2 * D + hi]);
    }
}

template <int OP, typename TX, int V>
cudaError_t launch_rows_v(const I8RowsDev& p, cudaStream_t st) {
    const dim3 per_row((unsigned)p.rows);
    const int vecs = (p.cols + V - 1) / V;          // vectors of a row
    if (vecs <= 32 * 4) return launch_pdl(k_i8_rows<OP, TX, V, 4, 32>, dim3((unsigned)((p.rows + 3) / 4)), dim3(128), 0, st, p);
    if (vecs <= 512) return launch_pdl(k_i8_rows<OP, TX, V, 1, 512>, per_row, dim3(512), 0, st, p);
    if (vecs <= 1024) return launch_pdl(k_i8_rows<OP, TX, V, 2, 512>, per_row, dim3(512), 0, st, p);
    if (vecs <= 2048) return launch_pdl(k_i8_rows<OP, TX, V, 4, 512>, per_row, dim3(512), 0, st, p);
    return launch_pdl(k_i8_rows<OP, TX, V, 0, 512>, per_row, dim3(512), 0, st, p);
}

}  // namespace

cudaError_t launch_i8_rows(int op, const I8RowsDev& p, cudaStream_t st) {
    // vectors of 8 elements where every row of every operand starts on a vector
    auto vec = [&](const void* q, long long ld, int size) { return q == nullptr || (((uintptr_t)q % 16) == 0 && (ld * size) % 16 == 0); };
    const int xs = p.x_f32 ? 4 : 2;
    const bool v8 = p.cols % 8 == 0 && vec(p.x, p.ldx, xs) && vec(p.delta, p.ldd, p.d_f32 ? 4 : 2) && vec(p.resid_out, p.ldo, xs) &&
                    ((uintptr_t)p.gain % 16) == 0 && ((uintptr_t)p.q % 8) == 0 && p.ldq % 8 == 0;
#define CATS_I8_ROWS(OP) \
    (op == OP) return p.x_f32 ? (v8 ? launch_rows_v<OP, float, 8>(p, st) : launch_rows_v<OP, float, 1>(p, st)) \
                              : (v8 ? launch_rows_v<OP, uint16_t, 8>(p, st) : launch_rows_v<OP, uint16_t, 1>(p, st))
    if CATS_I8_ROWS(I8_SWIGLU);
    if CATS_I8_ROWS(I8_QUANTIZE);
#undef CATS_I8_ROWS
    // the norm takes its operand types at run time
    return v8 ? launch_rows_v<I8_NORM, float, 8>(p, st) : launch_rows_v<I8_NORM, float, 1>(p, st);
}

cudaError_t launch_i8_qkv(const float* qkv, const int32_t* pos, int T, int nh, int hd, float rope_base, int prefix_len, void* q, void* kc,
                          void* vc, cudaStream_t st) {
    return launch_pdl(k_i8_qkv, dim3(T, 8), dim3(256), 0, st, qkv, pos, nh, hd, rope_base, prefix_len, (uint16_t*)q, (uint16_t*)kc,
                      (uint16_t*)vc);
}

cudaError_t launch_i8_dequantize(const int8_t* q, long long ldq, const float* scale, int rows, int cols, void* out, int out_f32,
                                 long long ldo, cudaStream_t st) {
    const bool v8 = cols % 8 == 0 && ((uintptr_t)q % 8) == 0 && ldq % 8 == 0 && ((uintptr_t)out % 16) == 0 &&
                    (ldo * (out_f32 ? 4 : 2)) % 16 == 0;
    const dim3 grid((unsigned)rows, (unsigned)((cols + 4095) / 4096));
    return v8 ? launch_pdl(k_i8_dequantize<8>, grid, dim3(256), 0, st, q, ldq, scale, cols, out, out_f32, ldo)
              : launch_pdl(k_i8_dequantize<1>, grid, dim3(256), 0, st, q, ldq, scale, cols, out, out_f32, ldo);
}

}  // namespace cats
