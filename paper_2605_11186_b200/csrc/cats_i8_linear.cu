// Matrix product in 8-bit integers with one scale per token and one per output channel:
//
//   out[t][n] = (sum_k x[t][k] w[n][k]) * sx[t] * sw[n]        (int32 sums, exact; scales applied in fp32)
//
// Tokens are the MMA's M dimension (128 per tile, lane = token), output channels its N dimension (R per tile, a multiple
// of 16 up to 256).  For the few tokens of a tree the product is bound by reading w once from HBM:
//   * w is packed (cats_pack_weights_i8) K block by K block: [K / 128][outs / 8] groups of 8 rows x 128 bytes, each group
//     in the 128-byte-swizzle layout tcgen05.mma reads.  Any R rows of one K block, R a multiple of 8, are one
//     contiguous run, so R is free and is chosen so that the tiles fill the SMs evenly (linear_plan).
//   * x is row-major as the row kernels leave it; TMA boxes of 128 bytes x ceil8(tokens) rows bring it in, zeros beyond the
//     last row and column.
// Warp 0 (one thread) copies w, warp 1 (one thread) copies x into a ring of shared-memory stages with mbarrier completion;
// warp 2 issues tcgen05.mma into one of two TMEM accumulators; warps 4-7 drain the other one: int32 -> fp32 * sx * sw ->
// bf16 or fp32 rows.  Rows of a stage that no copy writes (tokens beyond the last, channels beyond the last) hold
// leftovers; they only reach accumulator rows and columns that are not stored.
// Every wait is bounded; on expiry the CTA reports CATS_ERR_TIMEOUT, lets its copies land, frees its TMEM and returns.
#include <cuda.h>

#include "cats_kernels.cuh"

namespace cats {
namespace {

constexpr int kThreads = 256;
constexpr int kKb = 128;              // int8 columns of a K block: one swizzled row of 128 bytes
constexpr int kMaxStages = 16;
constexpr int kCtrl = 1024;
constexpr int kSmemMax = 227 * 1024;
constexpr int kSms = 148;

struct LinearDev {
    int rows, outs, n_kb;
    int R;                  // output channels per tile
    int m_blocks;           // blocks of 128 tokens
    int n_tiles;            // m_blocks * ceil(outs / R), token blocks fastest
    int x_rows;             // rows of an x box
    int unit;               // K blocks per stage
    int stages;
    uint32_t w_chunk;       // bytes of a tile's rows in one K block
    uint32_t x_chunk;
    uint32_t stage_bytes;
    uint32_t tail;          // bytes behind the last stage that its last x chunk is read over as 128 rows
    uint32_t tmem_cols;
    const uint8_t* w;
    const float *sx, *sw;
    void* out;
    int out_f32, vec_out;   // vec_out: rows and columns allow 16-byte stores
    long long ldo;
    int32_t* d_status;
};

struct Ctrl {
    uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(Ctrl) <= kCtrl, "control block too large");

// Instruction descriptor: D int32, A and B signed 8-bit, both K-major, M = 128, N = n.
__device__ __forceinline__ uint32_t idesc_i8_m128(int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
__device__ __forceinline__ void umma_i8(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
__device__ __forceinline__ void bulk_copy(void* smem_dst, const void* gsrc, uint32_t bytes, uint64_t* bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
        ::"r"(smem_u32(smem_dst)), "l"(gsrc), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
        : "memory");
}

// 16 accumulator columns of one token to out[t][n0 .. n0 + 16).
__device__ __forceinline__ void store16(const LinearDev& p, long long t, int n0, const float* acc, float sx, const float* sw) {
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = (float)__float_as_int(acc[i]) * sx * sw[i];
    if (p.vec_out && n0 + 16 <= p.outs) {
        if (p.out_f32) {
            float4* o = reinterpret_cast<float4*>((float*)p.out + t * p.ldo + n0);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        } else {
            uint4* o = reinterpret_cast<uint4*>((uint16_t*)p.out + t * p.ldo + n0);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                o[i] = make_uint4(pack_bf16x2(v[8 * i], v[8 * i + 1]), pack_bf16x2(v[8 * i + 2], v[8 * i + 3]),
                                  pack_bf16x2(v[8 * i + 4], v[8 * i + 5]), pack_bf16x2(v[8 * i + 6], v[8 * i + 7]));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        if (n0 + i >= p.outs) break;
        if (p.out_f32) ((float*)p.out)[t * p.ldo + n0 + i] = v[i];
        else ((uint16_t*)p.out)[t * p.ldo + n0 + i] = float_to_bf16_bits(v[i]);
    }
}

__global__ void __launch_bounds__(kThreads) k_linear_i8(const LinearDev p, const __grid_constant__ CUtensorMap tm_x) {
    extern __shared__ __align__(1024) uint8_t smem[];      // [stages][stage_bytes], the tail, channel scales, control block
    float* const sw_s = reinterpret_cast<float*>(smem + (size_t)p.stages * p.stage_bytes + p.tail);
    Ctrl* const ctrl = reinterpret_cast<Ctrl*>(sw_s + 4 * 256);
    volatile int* const abort_flag = &ctrl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((smem_u32(smem) & 1023u) != 0) {      // the swizzled tiles need this alignment
        if (threadIdx.x == 0) report(p.d_status, CATS_ERR_UNSUPPORTED);
        return;
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(&ctrl->full[s], 2);     // one arrive.expect_tx from each copying thread
            mbar_init(&ctrl->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&ctrl->acc_full[b], 1);
            mbar_init(&ctrl->acc_empty[b], 128);
        }
        ctrl->abort_flag = 0;
        mbar_fence_init();
        tma_prefetch_desc(&tm_x);
    }
    if (warp == 2) {
        tmem_alloc(&ctrl->tmem_base, p.tmem_cols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = ctrl->tmem_base;
    pdl_launch_dependents();
    const int S = p.stages, G = (int)gridDim.x;
    const int n_units = (p.n_kb + p.unit - 1) / p.unit;
    const size_t kb_stride = (size_t)((p.outs + 7) / 8) * 1024;       // packed bytes of one K block
    // stage layout: unit chunks of w, then unit chunks of x
    if (warp <= 1) {
        if (lane == 0) {
            const bool is_w = warp == 0;
            // many token blocks read the same rows of w soon after one another; a tree reads them once
            const uint64_t pol = is_w && p.m_blocks == 1 ? l2_policy_evict_first() : l2_policy_evict_last();
            if (!is_w) pdl_wait();            // x comes from the kernel before; w never does
            int s = 0, issued = 0;
            uint32_t par = 1;
            bool ok = true;
            for (int tile = blockIdx.x; tile < p.n_tiles && ok; tile += G) {
                const int nt = tile / p.m_blocks, mb = tile - nt * p.m_blocks;
                const int n0 = nt * p.R;
                const uint32_t w_bytes = (uint32_t)min(p.R, (p.outs - n0 + 7) / 8 * 8) * kKb;
                const uint8_t* src = p.w + (size_t)(n0 >> 3) * 1024;
                for (int u = 0, kb = 0; u < n_units; ++u) {
                    if (issued >= S && !mbar_wait(&ctrl->empty[s], par, abort_flag)) { ok = false; break; }
                    uint8_t* stage = smem + (size_t)s * p.stage_bytes;
                    const int nk = min(p.unit, p.n_kb - kb);
                    if (is_w) {
                        mbar_expect_tx(&ctrl->full[s], w_bytes * nk);
                        for (int j = 0; j < nk; ++j, ++kb, src += kb_stride) bulk_copy(stage + j * p.w_chunk, src, w_bytes, &ctrl->full[s], pol);
                    } else {
                        mbar_expect_tx(&ctrl->full[s], p.x_chunk * nk);
                        for (int j = 0; j < nk; ++j, ++kb)
                            tma_load_2d(stage + p.unit * p.w_chunk + j * p.x_chunk, &tm_x, kb * kKb, mb * 128, &ctrl->full[s], pol);
                    }
                    ++issued;
                    if (++s == S) { s = 0; par ^= 1u; }
                }
            }
            if (*abort_flag) {                // let the copies in flight land before the CTA goes away
                volatile int ignore = 0;
                for (int j = max(0, issued - S); j < issued; ++j) mbar_wait(&ctrl->full[j % S], (j / S) & 1, &ignore);
            }
        }
    } else if (warp == 2) {
        if (lane == 0) {
            const uint32_t idesc = idesc_i8_m128(p.R);
            int s = 0, seg = 0;
            uint32_t par = 0;
            bool ok = true;
            for (int tile = blockIdx.x; tile < p.n_tiles && ok; tile += G, ++seg) {
                const int b = seg & 1;
                if (seg >= 2) ok = mbar_wait(&ctrl->acc_empty[b], ((seg >> 1) - 1) & 1, abort_flag);
                tc_fence_after_sync();
                const uint32_t d = tmem + (uint32_t)(b * p.R);
                for (int u = 0, kb = 0; u < n_units && ok; ++u) {
                    ok = mbar_wait(&ctrl->full[s], par, abort_flag);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const int nk = min(p.unit, p.n_kb - kb);
                    const uint32_t w_addr = smem_u32(smem + (size_t)s * p.stage_bytes);
                    const uint32_t x_addr = w_addr + p.unit * p.w_chunk;
                    for (int j = 0; j < nk; ++j, ++kb) {
                        const uint64_t da = umma_desc_sw128(x_addr + j * p.x_chunk), db = umma_desc_sw128(w_addr + j * p.w_chunk);
#pragma unroll
                        for (int k = 0; k < 4; ++k) umma_i8(d, da + 2 * k, db + 2 * k, idesc, kb > 0 || k > 0);
                    }
                    umma_commit(&ctrl->empty[s]);
                    if (++s == S) { s = 0; par ^= 1u; }
                }
                umma_commit(&ctrl->acc_full[b]);      // also on abort, so that the epilogue warps wake up
            }
        }
    } else if (warp >= 4) {
        pdl_wait();
        const int q4 = warp & 3;
        float* const sw = sw_s + q4 * 256;       // one copy of the tile's channel scales per warp: no barrier needed
        int seg = 0;
        bool ok = true;
        for (int tile = blockIdx.x; tile < p.n_tiles && ok; tile += G, ++seg) {
            const int nt = tile / p.m_blocks, mb = tile - nt * p.m_blocks;
            const int n0 = nt * p.R, b = seg & 1;
            const long long t = (long long)mb * 128 + q4 * 32 + lane;
            __syncwarp();
            for (int i = lane; i < p.R; i += 32) sw[i] = n0 + i < p.outs ? __ldg(p.sw + n0 + i) : 0.f;
            __syncwarp();
            const float sx = t < p.rows ? __ldg(p.sx + t) : 0.f;
            ok = mbar_wait(&ctrl->acc_full[b], (seg >> 1) & 1, abort_flag) && !*abort_flag;
            tc_fence_after_sync();
            if (ok && mb * 128 + q4 * 32 < p.rows) {
                const uint32_t taddr = tmem + ((uint32_t)(q4 * 32) << 16) + (uint32_t)(b * p.R);
                for (int c = 0; c < p.R && n0 + c < p.outs; c += 16) {
                    float acc[16];
                    tmem_ld16(taddr + c, acc);
                    if (t < p.rows) store16(p, t, n0 + c, acc, sx, sw + c);
                }
            }
            tc_fence_before_sync();
            mbar_arrive(&ctrl->acc_empty[b]);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 2) {
        __syncwarp();
        tc_fence_after_sync();
        tmem_dealloc(tmem, p.tmem_cols);
    }
    if (threadIdx.x == 0 && *abort_flag) report(p.d_status, CATS_ERR_TIMEOUT);
}

// int8 [rows][cols] -> [K block][8-row group][8 x 128 bytes], 128-byte swizzle, zeros beyond the matrix.  One thread per 16 bytes.
__global__ void __launch_bounds__(256) k_pack_weights_i8(const int8_t* __restrict__ src, long long ld, int rows, int cols, int n8,
                                                         long long n, uint4* __restrict__ dst) {
    const long long g = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (g >= n) return;
    const int c = (int)(g & 7), r = (int)((g >> 3) & 7);
    const long long group = g >> 6;
    const int kb = (int)(group / n8), row = (int)(group - (long long)kb * n8) * 8 + r;
    const int col = kb * kKb + c * 16;
    uint32_t w[4] = {0, 0, 0, 0};
    if (row < rows) {
        const int8_t* s = src + row * ld + col;
        for (int i = 0; i < 16 && col + i < cols; ++i) w[i >> 2] |= ((uint32_t)(uint8_t)s[i]) << (8 * (i & 3));
    }
    dst[group * 64 + r * 8 + (c ^ r)] = make_uint4(w[0], w[1], w[2], w[3]);
}

typedef CUresult (*TensorMapEncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                      const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                      CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
TensorMapEncodeFn tensor_map_encoder() {
    static const TensorMapEncodeFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
            f = nullptr;
        return (TensorMapEncodeFn)f;
    }();
    return fn;
}

// The 8-bit operand x in boxes of 128 bytes x box_rows rows.  The innermost coordinate of every box is a multiple of 128.
bool x_tensor_map(const I8Linear& p, int box_rows, CUtensorMap* out) {
    TensorMapEncodeFn enc = tensor_map_encoder();
    if (enc == nullptr) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)p.cols, (cuuint64_t)p.rows};
    const cuuint64_t strides[1] = {(cuuint64_t)p.ldx};
    const cuuint32_t box[2] = {kKb, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return enc(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(p.x), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Opts a kernel into large shared memory, once per device.
template <typename K> cudaError_t allow_smem(K kernel, bool (&done)[64]) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64 && done[dev]) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
    if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;
    return e;
}

inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Channels per tile: the multiple of 16 that gives the busiest SM the least to read, w rows and x rows together.
int linear_tile(const I8Linear& p, int m_blocks, int x_rows) {
    int best = 256;
    long long best_cost = 1ll << 62;
    for (int R = 256; R >= 16; R -= 16) {
        const long long tiles = (long long)m_blocks * ceil_div(p.outs, R);
        const long long cost = (tiles + kSms - 1) / kSms * (R + x_rows);
        if (cost < best_cost) { best_cost = cost; best = R; }
    }
    return best;
}

}  // namespace

size_t packed_weight_i8_bytes(int rows, int cols) { return (size_t)ceil_div(cols, kKb) * ceil_div(rows, 8) * 1024; }

cudaError_t launch_pack_weights_i8(const int8_t* src, long long ld, int rows, int cols, void* dst, cudaStream_t st) {
    const long long n = (long long)(packed_weight_i8_bytes(rows, cols) / 16);
    ++g_launch_count;
    k_pack_weights_i8<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(src, ld, rows, cols, ceil_div(rows, 8), n, (uint4*)dst);
    return cudaGetLastError();
}

cudaError_t launch_linear_i8(const I8Linear& p, cudaStream_t st) {
    static bool done[64];
    cudaError_t e = allow_smem(k_linear_i8, done);
    if (e != cudaSuccess) return e;
    LinearDev d = {};
    d.rows = p.rows; d.outs = p.outs; d.n_kb = ceil_div(p.cols, kKb);
    d.m_blocks = ceil_div(p.rows, 128);
    d.x_rows = p.rows >= 128 ? 128 : ceil_div(p.rows, 8) * 8;
    d.R = linear_tile(p, d.m_blocks, d.x_rows);
    const long long tiles = (long long)d.m_blocks * ceil_div(p.outs, d.R);
    if (tiles > (1ll << 30)) return cudaErrorInvalidValue;
    d.n_tiles = (int)tiles;
    d.w_chunk = (uint32_t)d.R * kKb;
    d.x_chunk = (uint32_t)d.x_rows * kKb;
    // K blocks per stage: about 24 KB, so that one barrier round trip carries enough bytes
    d.unit = max(1, min(8, 24 * 1024 / (int)(d.w_chunk + d.x_chunk)));
    d.stage_bytes = d.unit * (d.w_chunk + d.x_chunk);
    d.tail = 128u * kKb - d.x_chunk;
    const int fixed = (int)d.tail + 4 * 256 * 4 + kCtrl;
    d.stages = min(kMaxStages, (kSmemMax - fixed) / (int)d.stage_bytes);
    if (d.stages < 2) return cudaErrorInvalidConfiguration;
    d.tmem_cols = 32;
    while (d.tmem_cols < 2u * d.R) d.tmem_cols *= 2;
    d.w = (const uint8_t*)p.w; d.sx = p.sx; d.sw = p.sw;
    d.out = p.out; d.out_f32 = p.out_f32; d.ldo = p.ldo;
    d.vec_out = ((uintptr_t)p.out % 16) == 0 && (p.ldo * (p.out_f32 ? 4 : 2)) % 16 == 0;
    d.d_status = p.d_status;
    CUtensorMap tm;
    if (!x_tensor_map(p, d.x_rows, &tm)) return cudaErrorNotSupported;
    const int grid = d.n_tiles < kSms ? d.n_tiles : kSms;
    return launch_pdl(k_linear_i8, dim3(grid), dim3(kThreads), (size_t)d.stages * d.stage_bytes + fixed, st, d, tm);
}

cudaError_t set_wait_limit_i8(unsigned long long ns) { return cudaMemcpyToSymbol(g_wait_limit_ns, &ns, sizeof(ns)); }

}  // namespace cats
