// Row kernels of the 8-bit integer path: every kernel makes rows y of fp32 values and leaves them as int8 with one scale
// per row,
//   a = max(max|y|, 2^-100),   q = rint(127 y / a),   scale = a / 127        (y ~ q * scale)
// where y is a bf16 or fp32 row itself (attention output, a weight matrix), silu(gate) * up, or the RMSNorm of the
// residual stream after the preceding projection's output has been added to it.  A row that holds an infinity or a NaN
// gets a NaN scale and zeros, so that whatever is computed from it is NaN too.
//
// Bound by HBM for many rows and by latency (one trip to memory, one block-wide reduction) for the few rows of a tree.
// A row is read once and stays in registers; the norm needs sum x^2 and max|x g|, which are independent of each other, so
// both go through ONE reduction: y = (x g) r with r > 0 has its maximum where |x g| has.  The maxima keep NaNs.
#include "cats_i8.cuh"
#include "cats_kernels.cuh"

namespace cats {
namespace {

// Eight elements of a row as they lie in memory, 16 bytes each.  Loads and conversion are apart so that a thread can have all
// its loads in flight before it uses the first.  Rows are read once and marked so: left to age among them, the int8 rows
// were written back to HBM and fetched again by the kernel that reads them (SwiGLU of 4096 x 11008 and its values: 71 -> 56 us).
//
// load_any: for rows that start off the 16-byte grid or end inside a vector.  The 16-byte words around a vector are shifted into
// place; those of the row's first and last vector would hold bytes outside the row, which are not read: there the elements
// are loaded one by one, zeros behind the last column.
__device__ __forceinline__ uint32_t word_of(const uint4& a, int i) { return i == 0 ? a.x : (i == 1 ? a.y : (i == 2 ? a.z : a.w)); }
// words [m / 4 ...] of the NW words w, shifted right by m % 4 bytes (0 or 2); m the same for all lanes
template <int NW> __device__ __forceinline__ void shift_words(uint32_t* w, int m) {
    if (m & 8) {
#pragma unroll
        for (int i = 0; i + 2 < NW; ++i) w[i] = w[i + 2];
    }
    if (m & 4) {
#pragma unroll
        for (int i = 0; i + 1 < NW; ++i) w[i] = w[i + 1];
    }
    if (m & 2) {
#pragma unroll
        for (int i = 0; i + 1 < NW; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
}
template <typename T> struct Raw;
template <> struct Raw<float> {
    uint32_t w[8];
    __device__ __forceinline__ void load(const float* p) {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p)), b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) { w[i] = word_of(a, i); w[4 + i] = word_of(b, i); }
    }
    __device__ __forceinline__ void load_any(const float* row, int c, int cols) {
        const int m = (int)((uintptr_t)row & 15);
        if (m == 0 && c + 8 <= cols) return load(row + c);
        if (c > 0 && c + 12 - m / 4 <= cols) {
            const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(row + c) - m);
            const uint4 a = q[0], b = q[1], d = q[2];
            uint32_t v[12];
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = word_of(a, i); v[4 + i] = word_of(b, i); v[8 + i] = word_of(d, i); }
            shift_words<12>(v, m);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = c + i < cols ? __float_as_uint(row[c + i]) : 0u;
        }
    }
    __device__ __forceinline__ void get(float* v) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    }
};
template <> struct Raw<uint16_t> {     // bf16 bits
    uint32_t w[4];
    __device__ __forceinline__ void put(const uint4& a) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = word_of(a, i);
    }
    __device__ __forceinline__ void load(const uint16_t* p) { put(__ldcs(reinterpret_cast<const uint4*>(p))); }
    __device__ __forceinline__ void load_shared(const uint16_t* p) { put(*reinterpret_cast<const uint4*>(p)); }      // by all rows
    __device__ __forceinline__ void load_any(const uint16_t* row, int c, int cols) {
        const int m = (int)((uintptr_t)row & 15);
        if (m == 0 && c + 8 <= cols) return load(row + c);
        if (c > 0 && c + 16 - m / 2 <= cols) {
            const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(row + c) - m);
            const uint4 a = q[0], b = q[1];
            uint32_t v[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = word_of(a, i); v[4 + i] = word_of(b, i); }
            shift_words<8>(v, m);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = (c + 2 * i < cols ? (uint32_t)row[c + 2 * i] : 0u) | (c + 2 * i + 1 < cols ? (uint32_t)row[c + 2 * i + 1] << 16 : 0u);
        }
    }
    __device__ __forceinline__ void get(float* v) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
};
__device__ __forceinline__ void store_vec(float* p, const float* v) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store_vec(uint16_t* p, const float* v) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
// The same for rows off the grid: the 256 elements from column c0 on that a warp holds, eight per lane, go through its staging
// tile so that every store instruction covers a contiguous run (a lane storing its own eight elements one by one leaves a
// sector of its own each time).  bf16 in pairs from the first 4-byte boundary on.  All lanes take part.
__device__ __forceinline__ void stage_vec(float* stage, int lane, const float* v) {
    store_vec(stage + lane * 8, v);
    __syncwarp();
}
__device__ __forceinline__ void warp_store(float* row, int c0, int cols, float* stage, int lane, const float* v) {
    stage_vec(stage, lane, v);
    const int n = min(256, cols - c0);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i * 32 + lane < n) row[c0 + i * 32 + lane] = stage[i * 32 + lane];
    __syncwarp();
}
__device__ __forceinline__ void warp_store(uint16_t* row, int c0, int cols, float* stage, int lane, const float* v) {
    stage_vec(stage, lane, v);
    const int n = min(256, cols - c0), head = (int)(((uintptr_t)(row + c0) >> 1) & 1);
    if (head && lane == 0) row[c0] = float_to_bf16_bits(stage[0]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = head + 2 * (i * 32 + lane);
        if (e + 1 < n) *reinterpret_cast<uint32_t*>(row + c0 + e) = pack_bf16x2(stage[e], stage[e + 1]);
        else if (e < n) row[c0 + e] = float_to_bf16_bits(stage[e]);
    }
    __syncwarp();
}

template <int OP, bool GRID> __device__ __forceinline__ void store_q(int8_t* row, int c, int cols, bool vec, const float* y, float rs, const Factor& f) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = OP == I8_NORM ? __fmul_rn(y[i], rs) : y[i];
        w[i] = __float_as_uint(OP == I8_SWIGLU ? fmaf(v, f.hi, kRintMagic) : __fadd_rn(fmaf(v, f.hi, __fmul_rn(v, f.lo)), kRintMagic));
    }
    if (GRID || (vec && c + 8 <= cols)) {
        uint32_t o[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
            o[h] = __byte_perm(__byte_perm(w[h * 4], w[h * 4 + 1], 0x0040), __byte_perm(w[h * 4 + 2], w[h * 4 + 3], 0x0040), 0x5410);
        *reinterpret_cast<uint2*>(row + c) = make_uint2(o[0], o[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = (int8_t)(w[i] & 0xFFu);
    }
}

// max(m, |a|, |b|), NaN if any of them is
__device__ __forceinline__ float max_abs(float m, float a, float b) {
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(m), "f"(fabsf(a)), "f"(fabsf(b)));
    return m;
}
__device__ __forceinline__ float max_abs(float m, const float* y) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) m = max_abs(m, y[i], y[i + 1]);
    return m;
}
// silu(g) u = g u / (1 + e^-g): for g -> -inf the quotient goes to -0 (e^-g reaches infinity), for g -> inf to g.  Flushing forms of
// 2^x and 1/x, which need half the instructions: for gates from kFarGate up every intermediate is a normal number.
constexpr float kFarGate = -80.f, kFarExp = 4.1538374868278621e34f;      // 2^115: just below e^80, so that no gate below kFarGate is missed
constexpr uint32_t kFarMark = 0x80000000u;
__device__ __forceinline__ float silu_mul(float g, float u, float& e) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return g * r * u;
}
// The same below kFarGate, where 1 + e^-g is e^-g and its reciprocal leaves the fp32 range (at -87) before the product with a large up
// value does: e^g as the square of h = e^(g/2), one factor for g and one for u.  h is zero below -175, where no up value
// brings the product to the 2^-108 that half a step of the smallest scale is.
__device__ __forceinline__ float silu_mul_far(float g, float u) {
    float h;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(h) : "f"(g * 0.72134752044448170f));
    return (g * h) * (h * u);
}
// The largest of the row's threads' values, to all of them; for a block's row the barrier in front of the first write to red_m is here
template <bool WARP> __device__ __forceinline__ uint32_t row_max(uint32_t m, int tid, int NT, uint32_t* red_m) {
    m = __reduce_max_sync(0xffffffffu, m);
    if (WARP) return m;
    __syncthreads();
    if ((tid & 31) == 0) red_m[tid >> 5] = m;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, (tid & 31) < (NT >> 5) ? red_m[tid & 31] : 0u);
}

struct NoDelta {};        // the norm without a delta
template <typename T> struct MaybeRaw : Raw<T> { static constexpr bool has = true; };
template <> struct MaybeRaw<NoDelta> {
    static constexpr bool has = false;
    __device__ __forceinline__ void load(const void*) {}
    __device__ __forceinline__ void load_any(const void*, int, int) {}
    __device__ __forceinline__ void get(float*) const {}
};

// Eight elements of a row at column c, and from them the values y (before the norm's row factor).
// TD: SWIGLU's up values (TX), the norm's delta, or NoDelta.  GRID: every vector is whole and on the 16-byte grid.
template <int OP, typename TX, typename TD, bool GRID> struct RowVec {
    Raw<TX> x;
    MaybeRaw<TD> d;
    Raw<uint16_t> g;
    __device__ __forceinline__ void load(const I8RowsDev& p, long long row, int c) {
        const TX* const xr = (const TX*)p.x + row * p.ldx;
        const TD* const dr = OP == I8_SWIGLU ? (const TD*)p.x + row * p.ldx + p.cols : (const TD*)p.delta + row * p.ldd;
        if (GRID) {
            x.load(xr + c);
            if (OP != I8_QUANTIZE) d.load(dr + c);
            if (OP == I8_NORM) g.load_shared((const uint16_t*)p.gain + c);
        } else {
            x.load_any(xr, c, p.cols);
            if (OP != I8_QUANTIZE) d.load_any(dr, c, p.cols);
            if (OP == I8_NORM) g.load_any((const uint16_t*)p.gain, c, p.cols);
        }
    }
    __device__ __forceinline__ void sum(float* y) const {        // the norm: residual + delta; else the input
        x.get(y);
        if (OP == I8_NORM && MaybeRaw<TD>::has) {
            float t[8];
            d.get(t);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] += t[i];
        }
    }
    // acc: SWIGLU: the largest e^-gate so far (or NaN); the norm: the sum of squares so far
    __device__ __forceinline__ void values(float* y, float& acc) const {
        if (OP == I8_NORM) {
            float t[8];
            g.get(t);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                acc = fmaf(y[i], y[i], acc);
                y[i] *= t[i];
            }
        } else if (OP == I8_SWIGLU) {
            float u[8];
            d.get(u);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                float e0, e1;
                y[i] = silu_mul(y[i], u[i], e0);
                y[i + 1] = silu_mul(y[i + 1], u[i + 1], e1);
                acc = max_abs(acc, e0, e1);
            }
        }
    }
    // SWIGLU's values in a vector that has, or may have, gates below kFarGate; y: as sum() leaves it
    __device__ __forceinline__ void far_values(float* y) const {
        float u[8], e;
        d.get(u);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = y[i] < kFarGate ? silu_mul_far(y[i], u[i]) : silu_mul(y[i], u[i], e);
    }
};
// The norm's sums to the residual stream: in place and without a delta they are there already.
template <typename TX, typename TD, bool GRID>
__device__ __forceinline__ void store_resid(const I8RowsDev& p, long long row, int c, int c0, float* stage, int lane, const float* y) {
    if (p.resid_out == nullptr || (!MaybeRaw<TD>::has && p.resid_out == p.x)) return;
    TX* const out = (TX*)p.resid_out + row * p.ldo;
    if (!GRID) warp_store(out, c0, p.cols, stage, lane, y);
    else if (c < p.cols) store_vec(out + c, y);
}
__device__ __forceinline__ void zero(float* y, float& rs) {      // a row that is not finite is stored as zeros
    rs = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = 0.f;
}

// A row of SwiGLU with gates below kFarGate, by all threads that hold it.  They are rare: the row is read again, twice, a vector at a
// time, in a function of its own.  The pass over 4096 x 11008 and its values went from 56 to 60.5 us with this, to 64 with the choice
// per element inside values(), and to 70 with a second try over the vectors in registers, which leaves two blocks per SM of three.
template <typename TX, bool GRID, bool WARP>
__device__ __noinline__ void far_row(const I8RowsDev& p, long long row, int tid, int NT, uint32_t* red_m) {
    RowVec<I8_SWIGLU, TX, TX, GRID> in;
    float y[8], am = 0.f;
    for (int c = tid * 8; c < p.cols; c += NT * 8) {
        in.load(p, row, c);
        in.sum(y);
        in.far_values(y);
        am = max_abs(am, y);
    }
    const uint32_t mx = row_max<WARP>(abs_bits(am), tid, NT, red_m);
    const float a = fmaxf(__uint_as_float(mx), kTinyMax);
    const bool finite = mx < 0x7F800000u;
    const Factor factor = factor_127_over(finite ? a : 1.f);
    if (tid == 0) p.scale[row] = finite ? a / 127.f : __int_as_float(0x7FC00000);
    for (int c = tid * 8; c < p.cols; c += NT * 8) {
        in.load(p, row, c);
        in.sum(y);
        in.far_values(y);
        float rs;
        if (!finite) zero(y, rs);
        store_q<I8_SWIGLU, GRID>(p.q + row * p.ldq, c, p.cols, p.q_vec, y, 1.f, factor);
    }
}

// Largest block: what fits the 64 registers of 1024 threads is one vector, or two of a single input (the norm has three).
template <int OP, int NV> __host__ __device__ constexpr int row_threads() { return NV == 1 || (NV == 2 && OP != I8_NORM) ? 1024 : 512; }

// A block per row, NV vectors of 8 elements per thread (NV * 8 * blockDim.x >= cols): the row is read once and stays in
// registers.  LONG: any length, the row is read twice.  WARP: blocks of 128 threads hold four rows, one per warp, and need
// no barrier.
template <int OP, typename TX, typename TD, bool GRID, int NV, bool WARP, bool LONG>
__device__ __forceinline__ void i8_rows(const I8RowsDev& p) {
    __shared__ float red_s[32];
    __shared__ uint32_t red_m[32];
    __shared__ __align__(16) float stage_s[OP == I8_NORM && !GRID ? (WARP ? 4 : row_threads<OP, NV>() / 32) * 256 : 4];      // a staging tile per warp
    const int lane = threadIdx.x & 31;
    float* const stage = stage_s + (OP == I8_NORM && !GRID ? (threadIdx.x >> 5) * 256 : 0);
    pdl_launch_dependents();
    const long long row = WARP ? (long long)blockIdx.x * 4 + (threadIdx.x >> 5) : (long long)blockIdx.x;
    const int tid = WARP ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
    const int NT = WARP ? 32 : (int)blockDim.x;
    pdl_wait();
    if (WARP && row >= p.rows) return;
    float y[NV][8];
    float ss = 0.f;                 // the norm: sum of squares; SwiGLU: the largest e^-gate
    float am = 0.f;                 // max |y| of this thread, NaN if any is
    if (!LONG) {
        RowVec<OP, TX, TD, GRID> in[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * NT + tid) * 8;
            if (c < p.cols) in[k].load(p, row, c);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * NT + tid) * 8, c0 = c - lane * 8;
            if (c < p.cols) in[k].sum(y[k]);
            if (OP == I8_NORM && c0 < p.cols) store_resid<TX, TD, GRID>(p, row, c, c0, stage, lane, y[k]);
            if (c < p.cols) {
                in[k].values(y[k], ss);
                am = max_abs(am, y[k]);
            }
        }
    } else {
        for (int c = tid * 8; c < p.cols; c += NT * 8) {
            RowVec<OP, TX, TD, GRID> in;
            in.load(p, row, c);
            in.sum(y[0]);
            if (OP == I8_SWIGLU) in.far_values(y[0]);
            else in.values(y[0], ss);
            am = max_abs(am, y[0]);
        }
    }
    // the bits of non-negative values are in their order, NaN on top, and above them the mark of a row with gates below kFarGate
    uint32_t mx = abs_bits(am);
    if (OP == I8_SWIGLU && !LONG && !(ss < kFarExp)) mx = kFarMark;
    mx = __reduce_max_sync(0xffffffffu, mx);
    if (OP == I8_NORM) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    }
    if (!WARP) {
        if ((tid & 31) == 0) {
            red_m[tid >> 5] = mx;
            red_s[tid >> 5] = ss;
        }
        __syncthreads();
        const int nw = NT >> 5, l = tid & 31;
        mx = l < nw ? red_m[l] : 0u;
        mx = __reduce_max_sync(0xffffffffu, mx);
        if (OP == I8_NORM) {
            ss = l < nw ? red_s[l] : 0.f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        }
    }
    if (OP == I8_SWIGLU && !LONG && mx == kFarMark) return far_row<TX, GRID, WARP>(p, row, tid, NT, red_m);
    float rs = 1.f;
    if (OP == I8_NORM) rs = __frsqrt_rn(ss / (float)p.cols + p.eps);
    float a = __uint_as_float(mx) * rs;
    const bool finite = abs_bits(a) < 0x7F800000u;
    // 127 y / a: the norm's row factor is in both, so where a is the row's own maximum the quotient is taken without it, two
    // roundings fewer.  (Below 2^-90 the reciprocal could overflow.)
    float by = fmaxf(a, kTinyMax);
    if (OP == I8_NORM && a >= kTinyMax && __uint_as_float(mx) >= 8.077935669463161e-28f) {
        by = __uint_as_float(mx);
        rs = 1.f;
    }
    const Factor factor = factor_127_over(finite ? by : 1.f);
    a = fmaxf(a, kTinyMax);
    if (tid == 0) p.scale[row] = finite ? a / 127.f : __int_as_float(0x7FC00000);
    int8_t* const q = p.q + row * p.ldq;
    if (!LONG) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * NT + tid) * 8;
            if (c < p.cols) {
                if (!finite) zero(y[k], rs);
                store_q<OP, GRID>(q, c, p.cols, p.q_vec, y[k], rs, factor);
            }
        }
    } else {
        for (int c0 = (tid - lane) * 8; c0 < p.cols; c0 += NT * 8) {
            const int c = c0 + lane * 8;
            RowVec<OP, TX, TD, GRID> in;
            if (c < p.cols) {
                in.load(p, row, c);
                in.sum(y[0]);
            }
            if (OP == I8_NORM) store_resid<TX, TD, GRID>(p, row, c, c0, stage, lane, y[0]);
            if (c < p.cols) {
                if (OP == I8_SWIGLU) in.far_values(y[0]);
                else in.values(y[0], ss);
                if (!finite) zero(y[0], rs);
                store_q<OP, GRID>(q, c, p.cols, p.q_vec, y[0], rs, factor);
            }
        }
    }
}

// SwiGLU's parameters stay where the launch put them, for far_row to read; with __grid_constant__ the others are slower (quantise
// 22016 x 4096 and its values 90.5 instead of 84.6 us).
template <int OP, typename TX, typename TD, bool GRID, int NV, bool WARP, bool LONG>
__global__ void __launch_bounds__(WARP ? 128 : row_threads<OP, NV>()) k_i8_rows(const I8RowsDev p) { i8_rows<OP, TX, TD, GRID, NV, WARP, LONG>(p); }
template <typename TX, bool GRID, int NV, bool WARP, bool LONG>
__global__ void __launch_bounds__(WARP ? 128 : row_threads<I8_SWIGLU, NV>()) k_i8_swiglu_rows(const __grid_constant__ I8RowsDev p) {
    i8_rows<I8_SWIGLU, TX, TX, GRID, NV, WARP, LONG>(p);
}
template <int OP, typename TX, typename TD, bool GRID, int NV, bool WARP, bool LONG>
cudaError_t launch_rows_k(dim3 grid, int threads, cudaStream_t st, const I8RowsDev& p) {
    if constexpr (OP == I8_SWIGLU) return launch_i8(k_i8_swiglu_rows<TX, GRID, NV, WARP, LONG>, grid, dim3(threads), 0, st, p);
    else return launch_i8(k_i8_rows<OP, TX, TD, GRID, NV, WARP, LONG>, grid, dim3(threads), 0, st, p);
}

// q * scale, rounded to bf16 or as fp32.  One block per (row, 4096 columns), eight elements per thread and step, both steps loaded
// before the first is stored.  The second kernel is for rows off the grid and ragged ends; q_vec says whether rows of q start on
// 8 bytes.  q and scale come from the kernel in front, which may still run when this one starts: no read-only loads (__ldg, const
// __restrict__), here and wherever a kernel of this path waits for the one in front.
__device__ __forceinline__ void eight_values(const uint2& w, float s, float* v) {
    // a byte b as the float 2^23 + (b + 128), then minus 2^23 + 128: exact, and no conversion instruction
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = (__uint_as_float(__byte_perm((i < 4 ? w.x : w.y) ^ 0x80808080u, 0x4B000000u, 0x7440u + (i & 3))) - 8388736.f) * s;
}
__global__ void __launch_bounds__(256) k_i8_dequantize(const int8_t* q, long long ldq, const float* scale, int cols, void* out, int out_f32,
                                                       long long ldo) {
    pdl_launch_dependents();
    pdl_wait();
    const long long row = blockIdx.x;
    const float s = scale[row];
    const int c_end = min(cols, ((int)blockIdx.y + 1) * 4096), c0 = blockIdx.y * 4096 + threadIdx.x * 8;
    uint2 w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (c0 + k * 2048 < c_end) w[k] = __ldcg(reinterpret_cast<const uint2*>(q + row * ldq + c0 + k * 2048));
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = c0 + k * 2048;
        if (c >= c_end) break;
        float v[8];
        eight_values(w[k], s, v);
        if (out_f32) store_vec((float*)out + row * ldo + c, v);
        else store_vec((uint16_t*)out + row * ldo + c, v);
    }
}
__global__ void __launch_bounds__(256) k_i8_dequantize_any(const int8_t* q, long long ldq, const float* scale, int cols, int q_vec, void* out,
                                                           int out_f32, long long ldo) {
    __shared__ __align__(16) float stage_s[8 * 256];
    pdl_launch_dependents();
    pdl_wait();
    const long long row = blockIdx.x;
    const int lane = threadIdx.x & 31;
    float* const stage = stage_s + (threadIdx.x >> 5) * 256;
    const float s = scale[row];
    const int8_t* const qr = q + row * ldq;
    const int c_end = min(cols, ((int)blockIdx.y + 1) * 4096), c_warp = blockIdx.y * 4096 + (threadIdx.x - lane) * 8;
    uint2 w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = c_warp + k * 2048 + lane * 8;
        w[k] = make_uint2(0, 0);
        if (q_vec && c + 8 <= c_end) {
            w[k] = __ldcg(reinterpret_cast<const uint2*>(qr + c));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < c_end) (i < 4 ? w[k].x : w[k].y) |= (uint32_t)(uint8_t)qr[c + i] << (8 * (i & 3));
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c0 = c_warp + k * 2048;
        if (c0 >= c_end) break;
        float v[8];
        eight_values(w[k], s, v);
        if (out_f32) warp_store((float*)out + row * ldo, c0, c_end, stage, lane, v);
        else warp_store((uint16_t*)out + row * ldo, c0, c_end, stage, lane, v);
    }
}

// The QKV projection's rows [3 * D] fp32 to what the tree attention reads: q rotated, bf16; k rotated and v appended to cache
// rows prefix_len + t (rotate-half pairs (i, i + hd / 2), angle pos[t] * base^(-2i/hd) in fp64 so that far positions lose
// nothing; every value is rounded once, from the unrounded sums).  Grid (nodes, shares of the heads); a thread takes four
// pairs of q, k and v.  The angles need only pos, which was there before the call: they are computed before the wait for
// the projection (the fp64 sine is what would take longest here).
__global__ void __launch_bounds__(256) k_i8_qkv(const float* qkv, const int32_t* pos, int nh, int hd, float rope_base, int prefix_len,
                                                uint16_t* q, uint16_t* kc, uint16_t* vc) {
    __shared__ __align__(16) float cos_s[64], sin_s[64];
    pdl_launch_dependents();
    const int t = blockIdx.x, half = hd / 2, D = nh * hd;
    if ((int)threadIdx.x < half) {
        const double inv_freq = pow((double)rope_base, -2.0 * (double)threadIdx.x / (double)hd);
        double s, c;
        sincos((double)pos[t] * inv_freq, &s, &c);
        cos_s[threadIdx.x] = (float)c;
        sin_s[threadIdx.x] = (float)s;
    }
    __syncthreads();
    pdl_wait();
    const float* const row = qkv + (size_t)t * 3 * D;
    const size_t cache_row = (size_t)(prefix_len + t) * D;
    const int quads = nh * half / 4;
    auto load4 = [](const float* p) { return __ldcg(reinterpret_cast<const float4*>(p)); };
    auto store4 = [](uint16_t* p, float a, float b, float c, float d) { *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d)); };
    for (int i = blockIdx.y * 256 + threadIdx.x; i < quads; i += gridDim.y * 256) {
        const int h = i * 4 / half, r = i * 4 - h * half, lo = h * hd + r, hi = lo + half;
        const float4 c = *reinterpret_cast<const float4*>(cos_s + r), s = *reinterpret_cast<const float4*>(sin_s + r);
        const float4 q0 = load4(row + lo), q1 = load4(row + hi), k0 = load4(row + D + lo), k1 = load4(row + D + hi);
        const float4 v0 = load4(row + 2 * D + lo), v1 = load4(row + 2 * D + hi);
        uint16_t* const qo = q + (size_t)t * D;
        store4(qo + lo, q0.x * c.x - q1.x * s.x, q0.y * c.y - q1.y * s.y, q0.z * c.z - q1.z * s.z, q0.w * c.w - q1.w * s.w);
        store4(qo + hi, q1.x * c.x + q0.x * s.x, q1.y * c.y + q0.y * s.y, q1.z * c.z + q0.z * s.z, q1.w * c.w + q0.w * s.w);
        store4(kc + cache_row + lo, k0.x * c.x - k1.x * s.x, k0.y * c.y - k1.y * s.y, k0.z * c.z - k1.z * s.z, k0.w * c.w - k1.w * s.w);
        store4(kc + cache_row + hi, k1.x * c.x + k0.x * s.x, k1.y * c.y + k0.y * s.y, k1.z * c.z + k0.z * s.z, k1.w * c.w + k0.w * s.w);
        store4(vc + cache_row + lo, v0.x, v0.y, v0.z, v0.w);
        store4(vc + cache_row + hi, v1.x, v1.y, v1.z, v1.w);
    }
}

// Few vectors per thread make the shortest chain for a row, many keep more bytes in flight and fewer threads waiting: the
// former while all rows are on the SMs at once.  Measured, one or two against four vectors, us: norm of 64 / 592 / 1024 / 8192 x
// 4096 2.3 / 4.2 / 7.1 / 44.1 against 2.8 / 5.5 / 6.8 / 39.4; quantise 1.6 / 2.4 / 3.4 / 25.0 against 1.9 / 3.0 / 3.4 / 18.3; SwiGLU of
// 64 / 148 / 300 / 8192 x 11008 2.6 / 2.7 / 6.3 / 122 against 3.2 / 3.0 / 5.2 / 75.5.
inline bool rows_fit(const I8RowsDev& p, int threads) { return p.rows <= 148 * (2048 / threads); }

template <int OP, typename TX, typename TD, bool GRID>
cudaError_t launch_rows_v(const I8RowsDev& p, cudaStream_t st) {
    const int vecs = (p.cols + 7) / 8;              // vectors of a row
    // up to 1024 columns a warp holds a row: no barrier (64 x 1000: 1.6 us)
    if (vecs <= 32 * 4) return launch_rows_k<OP, TX, TD, GRID, 4, true, false>(dim3(((unsigned)p.rows + 3u) / 4u), 128, st, p);
    const dim3 grid((unsigned)p.rows);
    auto threads = [&](int nv) { return (vecs + nv * 32 - 1) / (nv * 32) * 32; };
    if (threads(1) <= row_threads<OP, 1>() && rows_fit(p, threads(1)))
        return launch_rows_k<OP, TX, TD, GRID, 1, false, false>(grid, threads(1), st, p);
    // off the grid also for many rows: a thread holds twice the words until they are shifted
    if (threads(2) <= row_threads<OP, 2>() && (!GRID || rows_fit(p, threads(2))))
        return launch_rows_k<OP, TX, TD, GRID, 2, false, false>(grid, threads(2), st, p);
    if (threads(4) <= row_threads<OP, 4>()) return launch_rows_k<OP, TX, TD, GRID, 4, false, false>(grid, threads(4), st, p);
    return launch_rows_k<OP, TX, TD, GRID, 1, false, true>(grid, 512, st, p);
}

template <int OP, typename TX, typename TD>
cudaError_t launch_rows_t(I8RowsDev p, cudaStream_t st) {
    auto on_grid = [](const void* q, long long ld, size_t size) { return q == nullptr || (((uintptr_t)q % 16) == 0 && (ld * (long long)size) % 16 == 0); };
    p.q_vec = ((uintptr_t)p.q % 8) == 0 && p.ldq % 8 == 0;
    const bool grid = p.cols % 8 == 0 && p.q_vec && on_grid(p.resid_out, p.ldo, sizeof(TX)) && on_grid(p.x, p.ldx, sizeof(TX)) && on_grid(p.delta, p.ldd, p.d_f32 ? 4 : 2) &&
                      ((uintptr_t)p.gain % 16) == 0;
    return grid ? launch_rows_v<OP, TX, TD, true>(p, st) : launch_rows_v<OP, TX, TD, false>(p, st);
}

}  // namespace

cudaError_t launch_i8_rows(int op, const I8RowsDev& p, cudaStream_t st) {
    typedef uint16_t bf16;
    if (op == I8_SWIGLU) return p.x_f32 ? launch_rows_t<I8_SWIGLU, float, float>(p, st) : launch_rows_t<I8_SWIGLU, bf16, bf16>(p, st);
    if (op == I8_QUANTIZE) return p.x_f32 ? launch_rows_t<I8_QUANTIZE, float, NoDelta>(p, st) : launch_rows_t<I8_QUANTIZE, bf16, NoDelta>(p, st);
    if (p.delta == nullptr) return p.x_f32 ? launch_rows_t<I8_NORM, float, NoDelta>(p, st) : launch_rows_t<I8_NORM, bf16, NoDelta>(p, st);
    if (p.d_f32) return p.x_f32 ? launch_rows_t<I8_NORM, float, float>(p, st) : launch_rows_t<I8_NORM, bf16, float>(p, st);
    return p.x_f32 ? launch_rows_t<I8_NORM, float, bf16>(p, st) : launch_rows_t<I8_NORM, bf16, bf16>(p, st);
}

cudaError_t launch_i8_qkv(const float* qkv, const int32_t* pos, int T, int nh, int hd, float rope_base, int prefix_len, void* q, void* kc,
                          void* vc, cudaStream_t st) {
    return launch_i8(k_i8_qkv, dim3(T, (nh * hd / 8 + 255) / 256), dim3(256), 0, st, qkv, pos, nh, hd, rope_base, prefix_len, (uint16_t*)q, (uint16_t*)kc,
                      (uint16_t*)vc);
}

cudaError_t launch_i8_dequantize(const int8_t* q, long long ldq, const float* scale, int rows, int cols, void* out, int out_f32,
                                 long long ldo, cudaStream_t st) {
    const bool q_vec = ((uintptr_t)q % 8) == 0 && ldq % 8 == 0;
    const bool on_grid = cols % 8 == 0 && q_vec && ((uintptr_t)out % 16) == 0 && (ldo * (out_f32 ? 4 : 2)) % 16 == 0;
    const dim3 grid((unsigned)rows, (unsigned)((cols + 4095) / 4096));
    return on_grid ? launch_i8(k_i8_dequantize, grid, dim3(256), 0, st, q, ldq, scale, cols, out, out_f32, ldo)
                   : launch_i8(k_i8_dequantize_any, grid, dim3(256), 0, st, q, ldq, scale, cols, q_vec, out, out_f32, ldo);
}

}  // namespace cats
