// Rows into and out of the paged cache (include/cats.h: cats_paged_append, cats_paged_read).
//
// Append, per row and head: y = R(pos) k (rotate-half pairs (i, i + hd / 2), angle pos base^(-2i/hd)), rounded to bf16, or held as
//   a = max(max|y|, 2^-100),   q = rint(127 y / a),   scale = a / 127,
// a head that holds an infinity or a NaN as zeros with a NaN scale.  Queries are rotated and rounded to bf16 in the same pass.
// Read: the same rows back, q scale.  Both move every byte once: bound by HBM for a prompt, by latency for a token.
// Measured: 8191 rows of 32 int8 heads of 128 with 32 query heads appended in 70 us (338 MB at 4.8 TB/s: threads wait at the two barriers in front of the
// angles, and instructions take 55 % of the issue slots), 16384 such rows read as bf16 in 70 us (5.8 TB/s, two thirds of it writes), one row or 64 in 2.5 us.
#include <math.h>
#include <string.h>

#include "cats_i8.cuh"
#include "cats_paged.cuh"

namespace cats {
namespace {

struct Frequencies { double turns[64]; };       // turns per position of each pair: base^(-2i/hd) / 2 pi

// Eight values from p on, on the 16-byte grid.
__device__ __forceinline__ void load8(const float* p, float* v) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
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

// Sixteen values: in stores of 32 bytes where the row lies on that grid (wide), which leave no sector half written.  (As two stores of 16 bytes per
// thread reading 16384 rows of 32 int8 heads back took 82 us, with threads' 16 bytes side by side 89, so 70.)
template <bool VEC> __device__ __forceinline__ void store16(uint16_t* p, const float* v, bool wide) {
    if (VEC && wide) {
        uint32_t y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(p), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]), "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7]) : "memory");
    } else {
        store8<VEC>(p, v);
        store8<VEC>(p + 8, v + 8);
    }
}
template <bool VEC> __device__ __forceinline__ void store16(float* p, const float* v, bool wide) {
#pragma unroll
    for (int h = 0; h < 16; h += 8) {
        if (VEC && wide)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                         ::"l"(p + h), "r"(__float_as_uint(v[h])), "r"(__float_as_uint(v[h + 1])), "r"(__float_as_uint(v[h + 2])), "r"(__float_as_uint(v[h + 3])),
                           "r"(__float_as_uint(v[h + 4])), "r"(__float_as_uint(v[h + 5])), "r"(__float_as_uint(v[h + 6])), "r"(__float_as_uint(v[h + 7])) : "memory");
        else store8<VEC>(p + h, v + h);
    }
}

// cos and sin of `turns` whole turns.  Reduced to an eighth of a turn to either side of a multiple of a quarter in fp64, so that what
// fp32 rounds is small: off by less than 2^-22, and by what fp64 loses of that many turns, 2^-51 a position (2^-20 at the last one, 2^31).
__device__ __forceinline__ float2 cos_sin_turns(double turns) {
    const double quarters = 4.0 * (turns - rint(turns));
    const double n = rint(quarters);
    float s, c;
    sincospif(0.5f * (float)(quarters - n), &s, &c);
    const int k = (int)n & 3;
    if (k & 1) { const float t = c; c = -s; s = t; }
    return k & 2 ? make_float2(-c, -s) : make_float2(c, s);
}

constexpr int kThreads = 256, kAppendThreads = 128;

// Sixteen values as they lie in memory
template <typename T, bool VEC> struct Raw16 {
    uint4 w[sizeof(T)];
    __device__ __forceinline__ void load(const T* p) {
        if (VEC) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T); ++i) w[i] = __ldcg(reinterpret_cast<const uint4*>(p) + i);
        } else {
            T v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = p[i];
            memcpy(w, v, sizeof v);
        }
    }
    __device__ __forceinline__ void get(float* v) const {
        if (sizeof(T) == 4) {
            memcpy(v, w, 64);
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t x[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[8 * j + 2 * i] = __uint_as_float(x[i] << 16);
                    v[8 * j + 2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
                }
            }
        }
    }
};

// A block takes R rows and (blockIdx.y) 128 of the pieces of their heads: HD / 32 threads hold a head, each 16 elements of its first half and the 16 that they are
// rotated with; heads in the order K, V, queries.  The inputs of all R rows are requested first: positions, pages and angles are three
// more trips one behind the other, during which nothing else would be on its way (8191 rows of 96 heads and reading them back: 230 us with a row
// per block that asked for its inputs last, 135 with 256 threads of one row that asked first; then 114, and 106 with registers for 7
// blocks on an SM: 6 of them 108, 8 107, 9 115.  One row a block: 8191 rows of fp32 144 us with 7, 140 with 8, 137 with 9; 500 rows of bf16 9.4, 8.4, 9.3.)
template <typename T, bool VEC, int HD, bool I8, int R>
__global__ void __launch_bounds__(kAppendThreads, R == 2 ? 7 : 8) k_paged_append(const __grid_constant__ PagedDev c, const __grid_constant__ PagedRows r, const __grid_constant__ Frequencies f, int rotate, int wide) {
    constexpr int HALF = HD / 2, TH = HD / 32;
    static_assert(R * HALF <= kAppendThreads, "one thread per angle");
    __shared__ __align__(16) float cos_s[R][HALF], sin_s[R][HALF];
    __shared__ PagedDev::Row at_s[R];
    __shared__ int pos_s[R];
    pdl_launch_dependents();
    pdl_wait();
    const int row0 = blockIdx.x * R, units = (r.n_heads + 2 * c.n_kv) * TH, u = blockIdx.y * kAppendThreads + threadIdx.x, unit = min(u, units - 1);
    const int head = unit / TH, e = (unit % TH) * 16;
    const int which = head < c.n_kv ? 0 : (head < 2 * c.n_kv ? 1 : 2), h = which == 2 ? head - 2 * c.n_kv : head - which * c.n_kv;
    const T* const x = (which == 0 ? (const T*)r.k : (which == 1 ? (const T*)r.v : (const T*)r.q)) + (size_t)h * HD + e;
    const long long ld = which == 0 ? r.ldk : (which == 1 ? r.ldv : r.ldq);
    Raw16<T, VEC> in[R][2];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const long long row = min(row0 + i, r.rows - 1);
        in[i][0].load(x + row * ld);
        in[i][1].load(x + row * ld + HALF);
    }
    if ((int)threadIdx.x < R) {
        const int row = row0 + (int)threadIdx.x;
        int pos = row < r.rows ? r.pos[row] : -1;
        PagedDev::Row at = {0, 0};
        if (pos >= 0 && !c.locate(r.seq ? r.seq[row] : row, pos, at)) {
            pos = -1;
            report(r.d_status, CATS_ERR_INVALID_ARG);
        }
        pos_s[threadIdx.x] = pos;
        at_s[threadIdx.x] = at;
    }
    __syncthreads();
    if (rotate) {
        const int i = (int)threadIdx.x / HALF, k = (int)threadIdx.x % HALF;
        if (i < R) {
            const float2 cs = cos_sin_turns((double)pos_s[i] * f.turns[k]);
            cos_s[i][k] = cs.x;
            sin_s[i][k] = cs.y;
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (pos_s[i] < 0) continue;             // the same for all threads
        const long long row = row0 + i;
        const PagedDev::Row at = at_s[i];
        float lo[16], hi[16];
        in[i][0].get(lo);
        in[i][1].get(hi);
        if (rotate && which != 1) {
#pragma unroll
            for (int j = 0; j < 16; j += 8) {
                float cs[8], sn[8];
                load8(&cos_s[i][e + j], cs);
                load8(&sin_s[i][e + j], sn);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float p = lo[j + k], q = hi[j + k];
                    lo[j + k] = p * cs[k] - q * sn[k];
                    hi[j + k] = q * cs[k] + p * sn[k];
                }
            }
        }
        if (which == 2) {
            if (u < units) {
                uint16_t* const o = r.q_out + row * r.ldqo + (size_t)h * HD + e;
                store16<VEC>(o, lo, wide & 1);
                store16<VEC>(o + HALF, hi, wide & 1);
            }
        } else if (!I8) {
            uint16_t* const o = reinterpret_cast<uint16_t*>((which ? c.v : c.k) + ((size_t)at.at + (size_t)h * c.head16) * 16) + e;
            if (u < units) {
                store16<true>(o, lo, wide & 2);
                store16<true>(o + HALF, hi, wide & 2);
            }
        }
        if (I8 && __any_sync(0xffffffffu, which != 2)) {
            uint32_t mx = 0;
#pragma unroll
            for (int k = 0; k < 16; ++k) mx = max(mx, max(abs_bits(lo[k]), abs_bits(hi[k])));
#pragma unroll
            for (int o = TH / 2; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            if (which != 2 && u < units) {
                const bool finite = mx < 0x7F800000u;
                const float a = fmaxf(__uint_as_float(mx), kTinyMax);
                const Factor by = factor_127_over(finite ? a : 1.f);
                uint32_t w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    uint32_t b[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float v = !finite ? 0.f : (k < 4 ? lo[4 * k + j] : hi[4 * (k - 4) + j]);
                        b[j] = __float_as_uint(__fadd_rn(fmaf(v, by.hi, __fmul_rn(v, by.lo)), kRintMagic));
                    }
                    w[k] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
                }
                uint8_t* const o = (which ? c.v : c.k) + ((size_t)at.at + (size_t)h * c.head16) * 16 + e;
                *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4*>(o + HALF) = make_uint4(w[4], w[5], w[6], w[7]);
                if (e == 0) (which ? c.vs : c.ks)[(size_t)at.s + (size_t)h * c.s_head] = finite ? a / 127.f : __int_as_float(0x7FC00000);
            }
        }
    }
}

// A block per row; a thread takes 16 elements of two pieces of it, both requested before the first is used.
template <typename T, bool VEC, bool WIDE, int HD, bool I8>
__global__ void __launch_bounds__(kThreads) k_paged_read(const __grid_constant__ PagedDev c, const __grid_constant__ PagedRows r) {
    constexpr int TH = HD / 16, kEach = 2;
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
        uint4 w[kEach][I8 ? 1 : 2];
        float s[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int u = u0 + k * blockDim.x, head = u / TH, which = head >= c.n_kv, h = head - which * c.n_kv;
            if (u < units) {
                const uint4* const p = reinterpret_cast<const uint4*>(which ? c.v : c.k) + (size_t)at.at + (size_t)h * c.head16 + u % TH * (I8 ? 1 : 2);
#pragma unroll
                for (int i = 0; i < (I8 ? 1 : 2); ++i) w[k][i] = __ldcg(p + i);
                if (I8) s[k] = __ldcg((which ? c.vs : c.ks) + (size_t)at.s + (size_t)h * c.s_head);
            }
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int u = u0 + k * blockDim.x, head = u / TH, which = head >= c.n_kv, h = head - which * c.n_kv;
            if (u >= units) break;
            T* const o = (which ? (T*)r.v_out + row * r.ldv : (T*)r.k_out + row * r.ldk) + (size_t)h * HD + u % TH * 16;
            float v[16];
            if (I8) {
                const uint32_t x[4] = {w[k][0].x, w[k][0].y, w[k][0].z, w[k][0].w};
#pragma unroll
                for (int i = 0; i < 16; ++i)      // a byte b as the float 2^23 + (b + 128), then minus 2^23 + 128: exact
                    v[i] = (__uint_as_float(__byte_perm(x[i >> 2] ^ 0x80808080u, 0x4B000000u, 0x7440u + (i & 3))) - 8388736.f) * s[k];
            } else {
#pragma unroll
                for (int j = 0; j < (I8 ? 1 : 2); ++j) {
                    const uint32_t x[4] = {w[k][j].x, w[k][j].y, w[k][j].z, w[k][j].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[8 * j + 2 * i] = __uint_as_float(x[i] << 16);
                        v[8 * j + 2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
                    }
                }
            }
            store16<VEC>(o, v, WIDE);
        }
    }
}

// Whether rows of `p` start on so many bytes, every one.
bool on_grid(const void* p, long long ld, int size, int bytes = 16) { return (uintptr_t)p % bytes == 0 && (ld * size) % bytes == 0; }

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

template <typename T, bool VEC, int HD, bool I8, int R>
cudaError_t append_rows(const PagedDev& c, const PagedRows& r, cudaStream_t st) {
    const int units = (r.n_heads + 2 * c.n_kv) * (HD / 32);
    static const Frequencies none = {};
    // stores of 32 bytes: of the queries, of a bf16 cache
    const bool cache = !I8 && (uintptr_t)c.k % 32 == 0 && (uintptr_t)c.v % 32 == 0 && c.page16 % 2 == 0 && c.row16 % 2 == 0 && c.head16 % 2 == 0;
    const int wide = (r.n_heads && on_grid(r.q_out, r.ldqo, 2, 32) ? 1 : 0) | (cache ? 2 : 0);
    return launch_i8(k_paged_append<T, VEC, HD, I8, R>, dim3((unsigned)(((long long)r.rows + R - 1) / R), (unsigned)((units + kAppendThreads - 1) / kAppendThreads)), dim3(kAppendThreads), 0,
                     st, c, r, r.rope_base > 0.f ? frequencies(r.rope_base, HD) : none, r.rope_base > 0.f ? 1 : 0, wide);
}
template <typename T, bool VEC, int HD, bool I8>
cudaError_t append_k(const PagedDev& c, const PagedRows& r, cudaStream_t st) {
    // two rows a block where that leaves every SM with blocks enough; fp32 inputs fill the registers with one
    constexpr int R = VEC && sizeof(T) == 2 ? 2 : 1;
    if (R > 1 && (long long)r.rows * (r.n_heads + 2 * c.n_kv) * (HD / 32) >= 148ll * 8 * kAppendThreads * R) return append_rows<T, VEC, HD, I8, R>(c, r, st);
    return append_rows<T, VEC, HD, I8, 1>(c, r, st);
}
template <typename T, bool VEC> cudaError_t append_t(const PagedDev& c, const PagedRows& r, int i8, int hd, cudaStream_t st) {
    if (hd == 128) return i8 ? append_k<T, VEC, 128, true>(c, r, st) : append_k<T, VEC, 128, false>(c, r, st);
    return i8 ? append_k<T, VEC, 64, true>(c, r, st) : append_k<T, VEC, 64, false>(c, r, st);
}
template <typename T, bool VEC, int HD, bool I8> cudaError_t read_k(const PagedDev& c, const PagedRows& r, cudaStream_t st) {
    const int units = 2 * c.n_kv * (HD / 16), size = (int)sizeof(T);
    const dim3 grid((unsigned)r.rows), block(min(kThreads, (units + 63) / 64 * 32));
    if (VEC && on_grid(r.k_out, r.ldk, size, 32) && on_grid(r.v_out, r.ldv, size, 32)) return launch_i8(k_paged_read<T, VEC, true, HD, I8>, grid, block, 0, st, c, r);
    return launch_i8(k_paged_read<T, VEC, false, HD, I8>, grid, block, 0, st, c, r);
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
