// Matrix product in 8-bit integers with one scale per token and one per output channel:
//
//   out[t][n] = (sum_k x[t][k] w[n][k]) * sx[t] * sw[n]        (int32 sums, exact; scales applied in fp32)
//
// Tokens are the MMA's M dimension (128 per tile, lane = token), output channels its N dimension (R per tile, a multiple
// of 16 up to 256).  For the few tokens of a tree the product is bound by reading w once from HBM:
//   * w is packed (cats_pack_weights_i8) K block by K block: [K / 128][outs / 8] groups of 8 rows x 128 bytes, each group
//     in the 128-byte-swizzle layout tcgen05.mma reads.  Any R rows of one K block, R a multiple of 8, are one
//     contiguous run, so R is free and is chosen so that the tiles fill the SMs evenly (linear_tiling).
//   * x is row-major as the row kernels leave it; TMA boxes of 128 bytes x ceil8(tokens) rows bring it in, zeros beyond the
//     last row and column.
// Warp 0 copies w, warp 1 copies x into a ring of shared-memory stages with mbarrier completion; warp 2 issues tcgen05.mma
// into one of two TMEM accumulators; warps 4-11 drain the other one: int32 -> fp32 * sx * sw -> bf16 or fp32 rows.  Rows of
// a stage that no copy writes (tokens beyond the last, channels beyond the last) hold leftovers; they only reach accumulator
// rows and columns that are not stored.
// With few tiles the K blocks are cut into `split` shares, one CTA of a cluster each.  The partial sums meet in distributed
// shared memory: the accumulator's 16-channel groups are dealt out to the CTAs, every CTA stores its int32 partial of a group
// into the memory of the group's owner (each sender has its own place there), one cluster barrier publishes them, and the
// owners add and store.  Whole numbers: the order of the sums does not matter, and nothing is left in global memory.
// Every wait is bounded; on expiry the CTA reports CATS_ERR_TIMEOUT, lets its copies land and its MMAs end, frees its TMEM and returns.
#include <cuda.h>

#include <mutex>

#include "cats_kernels.cuh"

namespace cats {
namespace {

constexpr int kEpiWarps = 8;
constexpr int kThreads = 128 + 32 * kEpiWarps;
constexpr int kKb = 128;              // int8 columns of a K block: one swizzled row of 128 bytes
constexpr int kMaxStages = 16;
constexpr int kCtrl = 1024;
constexpr int kSmemMax = 227 * 1024;
constexpr int kSms = 148;

struct LinearDev {
    int rows, outs, n_kb;
    int R;                  // output channels per tile
    int split, kb_share;    // CTAs per tile (one cluster), K blocks of each
    int m_blocks;           // blocks of 128 tokens
    int n_tiles;            // m_blocks * ceil(outs / R), token blocks fastest
    int x_rows;             // rows of an x box
    int unit;               // K blocks per stage
    int stages;
    uint32_t w_chunk;       // bytes of a tile's rows in one K block
    uint32_t x_chunk;
    uint32_t stage_bytes;
    uint32_t tail;          // bytes behind the last stage that its last x chunk is read over as 128 rows
    uint32_t recv_bytes;    // partial sums from the other CTAs of the cluster: [own groups][split - 1 senders]
    uint32_t tmem_cols;
    const uint8_t* w;
    const float *sx, *sw;
    void* out;
    int out_f32, vec_out;   // vec_out: rows and columns allow 16-byte stores
    long long ldo;
    int w_early;            // w may be read before the kernel in front has finished
    int drop_x;             // fault injection: the x copy of a CTA's last stage is announced but never made
    int give_up;            // fault injection: the MMA warp raises the abort flag in place of its first wait
    int32_t* d_status;
};

struct Ctrl {
    uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    int abort_flag;
    int issued[4], segs;      // after an abort: stages issued by each copying warp (a pair: of both CTAs), accumulators committed
};
static_assert(sizeof(Ctrl) <= kCtrl, "control block too large");

// Instruction descriptor: D int32, A and B signed 8-bit, both K-major, M = 128, N = n.
__device__ __forceinline__ uint32_t idesc_i8_m128(int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
// The low word of a shared-memory descriptor changes from MMA to MMA, the high word (8-row groups 1024 bytes apart,
// descriptor version, 128-byte swizzle) never does; see umma_desc_sw128.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t smem_addr) { return ((smem_addr & 0x3FFFFu) >> 4) | (1u << 16); }
__device__ __forceinline__ void umma_i8(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %5};\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi)
        : "memory");
}
// One lane of the warp, the same one every time.
__device__ __forceinline__ bool elect_one() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}
// Bounded wait of a whole warp: the answer is the same for every lane.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}
// NC accumulator columns of this thread's lane; the values may be used after tmem_loaded().
template <int NC> __device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t* r) {
#pragma unroll
    for (int h = 0; h < NC / 16; ++h)
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
            : "=r"(r[16 * h]), "=r"(r[16 * h + 1]), "=r"(r[16 * h + 2]), "=r"(r[16 * h + 3]), "=r"(r[16 * h + 4]), "=r"(r[16 * h + 5]),
              "=r"(r[16 * h + 6]), "=r"(r[16 * h + 7]), "=r"(r[16 * h + 8]), "=r"(r[16 * h + 9]), "=r"(r[16 * h + 10]), "=r"(r[16 * h + 11]),
              "=r"(r[16 * h + 12]), "=r"(r[16 * h + 13]), "=r"(r[16 * h + 14]), "=r"(r[16 * h + 15])
            : "r"(taddr + 16 * h)
            : "memory");
}
template <int NC> __device__ __forceinline__ void tmem_loaded(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < NC; ++i) asm volatile("" : "+r"(r[i]));       // no use of r moves above the wait
}
__device__ __forceinline__ uint32_t cluster_addr(uint32_t local_smem, int rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local_smem), "r"(rank));
    return r;
}
__device__ __forceinline__ void st_cluster_v4(uint32_t addr, const uint32_t* v) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_id() {
    uint32_t r;
    asm("mov.u32 %0, %%clusterid.x;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Partial sums of one 16-channel group from one sender: [4 channel quadruples][x_rows tokens][4] int32, so that a warp's
// store into a peer is 512 contiguous bytes (16-byte pieces of 64-byte token rows took four times as long: 12 bytes per ns).
__device__ __forceinline__ uint32_t part_bytes(int x_rows) { return (uint32_t)x_rows * 64u; }
__device__ __forceinline__ uint32_t part_piece(int x_rows, int t, int i) { return (uint32_t)(i * x_rows + t) * 16u; }

__device__ __forceinline__ void bulk_copy(void* smem_dst, const void* gsrc, uint32_t bytes, uint64_t* bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
        ::"r"(smem_u32(smem_dst)), "l"(gsrc), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
        : "memory");
}

// The way of NC accumulator columns of a warp's 32 tokens (one per lane) to out[t0 + lane][n0 .. n0 + NC), through the warp's
// staging tile: a store instruction then covers whole runs of a few rows (from the lanes directly, every lane's 16 bytes are a
// cache line of their own).  The sums are staged as they are and scaled on the way out, where a lane keeps its columns' scales.
// 16-byte pieces are permuted by row so that neither side has bank conflicts.
template <int NC> __device__ __forceinline__ uint32_t* staged(uint32_t* stage, int row, int piece) {
    return stage + row * NC + ((piece ^ (NC == 32 ? row & 7 : (row >> 1) & 3)) << 2);
}
template <int NC> __device__ __forceinline__ void stage_cols(const uint32_t* acc, uint32_t* stage, int lane) {
#pragma unroll
    for (int i = 0; i < NC / 4; ++i)
        *reinterpret_cast<uint4*>(staged<NC>(stage, lane, i)) = make_uint4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]);
    __syncwarp();
}
// n_tokens: valid tokens from t0 on; n_cols <= NC: valid columns; sx: the 32 token scales; sw: scales of the columns.
template <int NC>
__device__ __forceinline__ void store_cols(const LinearDev& p, long long t0, int n_tokens, int n0, int n_cols, const float* sx, const float* sw,
                                           const uint32_t* stage, int lane) {
    constexpr int NP = NC / 4;                       // pieces of 4 columns per row
    auto scale4 = [](const uint4& a, float s, const float4& w) {
        return make_float4((float)(int)a.x * s * w.x, (float)(int)a.y * s * w.y, (float)(int)a.z * s * w.z, (float)(int)a.w * s * w.w);
    };
    if (p.vec_out && n_cols % 8 == 0) {
        // A lane keeps its columns and steps through the rows: the permutation of its pieces repeats every 8 rows.
        if (p.out_f32) {
            constexpr int RI = 32 / NP;              // rows per instruction
            const int r0 = lane / NP, piece = lane % NP;
            const float4 w = *reinterpret_cast<const float4*>(sw + piece * 4);
            float* o = (float*)p.out + (t0 + r0) * p.ldo + n0 + piece * 4;
            uint4 a[NP];                             // all loads before the first store: the compiler keeps their order
            float s[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                a[i] = *reinterpret_cast<const uint4*>(staged<NC>(const_cast<uint32_t*>(stage), r0 + i * RI, piece));
                s[i] = sx[r0 + i * RI];
            }
            if (piece * 4 < n_cols)
#pragma unroll
                for (int i = 0; i < NP; ++i, o += RI * p.ldo)
                    if (r0 + i * RI < n_tokens) *reinterpret_cast<float4*>(o) = scale4(a[i], s[i], w);
        } else {
            constexpr int RI = 64 / NP;
            const int r0 = lane / (NP / 2), piece = lane % (NP / 2) * 2;
            const float4 w0 = *reinterpret_cast<const float4*>(sw + piece * 4), w1 = *reinterpret_cast<const float4*>(sw + piece * 4 + 4);
            uint16_t* o = (uint16_t*)p.out + (t0 + r0) * p.ldo + n0 + piece * 4;
            uint4 a[NP / 2], b[NP / 2];
            float s[NP / 2];
#pragma unroll
            for (int i = 0; i < NP / 2; ++i) {
                a[i] = *reinterpret_cast<const uint4*>(staged<NC>(const_cast<uint32_t*>(stage), r0 + i * RI, piece));
                b[i] = *reinterpret_cast<const uint4*>(staged<NC>(const_cast<uint32_t*>(stage), r0 + i * RI, piece + 1));
                s[i] = sx[r0 + i * RI];
            }
            if (piece * 4 < n_cols)
#pragma unroll
                for (int i = 0; i < NP / 2; ++i, o += RI * p.ldo) {
                    const float4 u = scale4(a[i], s[i], w0), v = scale4(b[i], s[i], w1);
                    if (r0 + i * RI < n_tokens)
                        *reinterpret_cast<uint4*>(o) = make_uint4(pack_bf16x2(u.x, u.y), pack_bf16x2(u.z, u.w), pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
                }
        }
    } else {
        const int col = lane % NC;
        if (col < n_cols) {
            const float w = sw[col];
            long long o = (t0 + lane / NC) * p.ldo + n0 + col;
#pragma unroll 4
            for (int row = lane / NC; row < n_tokens; row += 32 / NC, o += (32 / NC) * p.ldo) {
                const float v = (float)(int)staged<NC>(const_cast<uint32_t*>(stage), row, col >> 2)[col & 3] * sx[row] * w;
                if (p.out_f32) ((float*)p.out)[o] = v;
                else ((uint16_t*)p.out)[o] = float_to_bf16_bits(v);
            }
        }
    }
    __syncwarp();
}

// "The accumulator has been read": its loads have completed (tcgen05.wait::ld) before this is issued, and nothing else is handed
// over.  A releasing arrive would wait for the output stores in flight as well (in a pair, whose barrier is a cluster away:
// 4096 x 1024 x 8192 35.8 instead of 32.0 us).
__device__ __forceinline__ void arrive_read(uint64_t* bar) {
    asm volatile("mbarrier.arrive.relaxed.cta.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// After an abort: what is still in flight into this CTA's memories ends before the CTA goes away.  By all threads, when none of them
// waits on a barrier of the pipeline any more, so that nothing is issued after this.  Copies: the stages issued last, at most S of them,
// are waited for on their barriers.  A copying warp that gave up before the other one arrives in its place, without bytes
// (it is less than S stages behind: the other one's stage j needed stage j - S whole).  MMAs: the last commit.  The limit is for
// what never comes, such as a withheld copy; copies and MMAs take microseconds.
constexpr unsigned long long kDrainNs = 10000000ull;
__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity, unsigned long long t0) {
    while (!mbar_try_wait(bar, parity) && globaltimer_ns() - t0 < kDrainNs) {}
}
__device__ __noinline__ void drain(Ctrl* ctrl, int S, int issued, int segs) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned long long t0 = globaltimer_ns();
    if (warp <= 1 && lane == 0) ctrl->issued[warp] = issued;
    __syncthreads();
    if (warp <= 1) {
        const int last = max(ctrl->issued[0], ctrl->issued[1]);
        if (lane == 0)
            for (int j = issued; j < last; ++j) mbar_arrive(&ctrl->full[j % S]);
        __syncwarp();
        for (int j = max(0, last - S); j < last; ++j) drain_wait(&ctrl->full[j % S], (j / S) & 1, t0);
    } else if (warp == 2 && segs > 0) {
        drain_wait(&ctrl->acc_full[(segs - 1) & 1], ((segs - 1) >> 1) & 1, t0);
    }
    __syncthreads();
}

// The scales of a tile, fetched a tile ahead into registers and from there to the warp's copy in shared memory.
struct TileScales {
    float w[8], x;
    __device__ __forceinline__ void fetch(const LinearDev& p, int n0, long long t0, int lane) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = lane + 32 * j < p.R && n0 + lane + 32 * j < p.outs ? __ldcg(p.sw + n0 + lane + 32 * j) : 0.f;
        x = t0 + lane < p.rows ? __ldcg(p.sx + t0 + lane) : 0.f;
    }
    __device__ __forceinline__ void put(float* sw, float* sx, int lane) const {
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) sw[lane + 32 * j] = w[j];
        sx[lane] = x;
        __syncwarp();
    }
};

// This warp's share (32 columns, every other time) of a whole accumulator: the next columns are on their way while these are
// scaled and stored.  n_tokens > 0.  release(): called once when the warp has read its last columns.
template <typename F>
__device__ __forceinline__ void store_tile(const LinearDev& p, uint32_t taddr, int group, long long t0, int n_tokens, int n0, const float* sx,
                                           const float* sw, uint32_t* stage, int lane, F release) {
    uint32_t acc[32];
    const int n_cols = min(p.R, p.outs - n0);
    if (group * 32 < n_cols) tmem_load<32>(taddr + group * 32, acc);
    else release();
#pragma unroll 1
    for (int c = group * 32; c < n_cols; c += 64) {
        tmem_loaded<32>(acc);
        stage_cols<32>(acc, stage, lane);
        if (c + 64 < n_cols) tmem_load<32>(taddr + c + 64, acc);
        else release();
        store_cols<32>(p, t0, n_tokens, n0 + c, min(32, n_cols - c), sx, sw + c, stage, lane);
    }
}

__global__ void __launch_bounds__(kThreads) k_linear_i8(const LinearDev p, const __grid_constant__ CUtensorMap tm_x) {
    extern __shared__ __align__(1024) uint8_t smem[];      // [stages][stage_bytes], the tail, received partials, staging tiles, channel scales, control block
    uint8_t* const recv = smem + (size_t)p.stages * p.stage_bytes + p.tail;
    uint32_t* const stage_s = reinterpret_cast<uint32_t*>(recv + p.recv_bytes);      // one 32 x 32 tile per epilogue warp
    float* const sw_s = reinterpret_cast<float*>(stage_s + kEpiWarps * 1024);        // 256 channel scales, 32 token scales per epilogue warp
    Ctrl* const ctrl = reinterpret_cast<Ctrl*>(sw_s + kEpiWarps * 288);
    volatile int* const abort_flag = &ctrl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((smem_u32(smem) & 1023u) != 0) {      // the swizzled tiles need this alignment
        if (threadIdx.x == 0) report(p.d_status, CATS_ERR_UNSUPPORTED);
        return;
    }
    if (warp == 0) {                          // one stage's barriers per lane
        if (lane < p.stages) {
            mbar_init(&ctrl->full[lane], 2);  // one arrive.expect_tx from each copying warp
            mbar_init(&ctrl->empty[lane], 1);
        } else if (lane >= 30) {
            mbar_init(&ctrl->acc_full[lane - 30], 1);
            mbar_init(&ctrl->acc_empty[lane - 30], kEpiWarps);
        }
        if (lane == 0) ctrl->abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 1 && lane == 0) tma_prefetch_desc(&tm_x);
    if (warp == 2) {
        tmem_alloc(&ctrl->tmem_base, p.tmem_cols);
        tmem_relinquish();
    }
    // split == 1: tiles blockIdx.x, + gridDim.x, ...; else exactly one tile, K blocks [kb0, kb0 + n_kb)
    const int rank = p.split > 1 ? (int)cluster_rank() : 0;
    const int first = p.split > 1 ? (int)cluster_id() : (int)blockIdx.x, G = p.split > 1 ? p.n_tiles : (int)gridDim.x;
    const int kb0 = rank * p.kb_share, n_kb = min(p.n_kb - kb0, p.kb_share);
    const int S = p.stages;
    const int n_units = p.unit == 1 ? n_kb : (n_kb + p.unit - 1) / p.unit;
    // Every CTA starts at another place of the K range: in step, all SMs would ask the same few L2 slices for the same rows of
    // x.  Whole numbers: the order of the sums does not matter.
    const int u_first = p.m_blocks == 1 ? (int)blockIdx.x % n_units : 0;
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = ctrl->tmem_base;
    int issued = 0, segs = 0;                 // stages issued by this copying warp; tiles whose accumulator the MMA warp has committed
    if (p.split > 1) cluster_arrive();        // waited for before the first store into a peer: every CTA of the cluster has started
    pdl_launch_dependents();
    // stage layout: unit chunks of w, then unit chunks of x.  All lanes of a role's warp run its loop and one of them issues:
    // addresses and descriptors stay in uniform registers, where the copy and MMA instructions want them.
    if (warp <= 1) {
        const bool is_w = warp == 0;
        // many token blocks read the same rows of w soon after one another; a tree reads them once
        const uint64_t pol = is_w && p.m_blocks == 1 ? l2_policy_evict_first() : l2_policy_evict_last();
        const size_t kb_stride = (size_t)((p.outs + 7) / 8) * 1024;       // packed bytes of one K block
        // x comes from the kernel before; w does not where this launch follows others of the same call: the ring is filled with
        // it at once.  No clock of a bounded wait starts before the kernel in front has finished.
        if (!is_w || !p.w_early) pdl_wait();
        int s = 0;
        uint32_t par = 1;
        bool ok = true;
        for (int tile = first; tile < p.n_tiles && ok; tile += G) {
            const int nt = p.m_blocks == 1 ? tile : tile / p.m_blocks, mb = tile - nt * p.m_blocks;
            const int n0 = nt * p.R;
            const uint32_t w_bytes = (uint32_t)min(p.R, (p.outs - n0 + 7) / 8 * 8) * kKb;
            const uint8_t* const w_tile = p.w + (size_t)kb0 * kb_stride + (size_t)(n0 >> 3) * 1024;
            for (int i = 0, u = u_first; i < n_units; ++i) {
                if (issued == S) pdl_wait();
                if (issued >= S && !warp_wait(&ctrl->empty[s], par, abort_flag)) { ok = false; break; }
                uint8_t* const stage = smem + (size_t)s * p.stage_bytes;
                const int kb = u * p.unit, nk = min(p.unit, n_kb - kb);
                if (elect_one()) {
                    if (is_w) {
                        mbar_expect_tx(&ctrl->full[s], w_bytes * nk);
                        for (int j = 0; j < nk; ++j) bulk_copy(stage + j * p.w_chunk, w_tile + (size_t)(kb + j) * kb_stride, w_bytes, &ctrl->full[s], pol);
                    } else {
                        mbar_expect_tx(&ctrl->full[s], p.x_chunk * nk);
                        for (int j = 0; j < nk && !(p.drop_x && i == n_units - 1); ++j)
                            tma_load_2d(stage + p.unit * p.w_chunk + j * p.x_chunk, &tm_x, (kb0 + kb + j) * kKb, mb * 128, &ctrl->full[s], pol);
                    }
                }
                __syncwarp();
                ++issued;
                if (++s == S) { s = 0; par ^= 1u; }
                if (++u == n_units) u = 0;
            }
        }
    } else if (warp == 2) {
        pdl_wait();
        const uint32_t idesc = idesc_i8_m128(p.R);
        int s = 0;
        uint32_t par = 0;
        bool ok = !p.give_up;
        if (!ok) *abort_flag = 1;
        for (int tile = first; tile < p.n_tiles && ok; tile += G, ++segs) {
            const int b = segs & 1;
            if (segs >= 2) ok = warp_wait(&ctrl->acc_empty[b], ((segs >> 1) - 1) & 1, abort_flag);
            tc_fence_after_sync();
            const uint32_t d = tmem + (uint32_t)(b * p.R);
            uint32_t more = 0;                // the first MMA of a tile overwrites the accumulator
            for (int i = 0, u = u_first; i < n_units && ok; ++i) {
                ok = warp_wait(&ctrl->full[s], par, abort_flag);
                if (!ok) break;
                tc_fence_after_sync();
                const int nk = min(p.unit, n_kb - u * p.unit);
                const uint32_t w_addr = smem_u32(smem) + (uint32_t)s * p.stage_bytes;
                uint32_t db = desc_lo(w_addr), da = desc_lo(w_addr + p.unit * p.w_chunk);
                if (elect_one()) {
                    for (int j = 0; j < nk; ++j) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            umma_i8(d, da + 2 * k, db + 2 * k, idesc, more);
                            more = 1;
                        }
                        da += p.x_chunk >> 4;
                        db += p.w_chunk >> 4;
                    }
                    umma_commit(&ctrl->empty[s]);
                }
                more = 1;
                __syncwarp();
                if (++s == S) { s = 0; par ^= 1u; }
                if (++u == n_units) u = 0;
            }
            if (elect_one()) umma_commit(&ctrl->acc_full[b]);      // also on abort, so that the epilogue warps wake up
            __syncwarp();
        }
    } else if (warp == 3) {
        // A call of its own may not read w before the kernel in front has finished (it may be what writes w), but HBM need not
        // idle until then: the first copies' bytes are requested into L2, which is where any later write of theirs lands too
        // (64 x 4096 x 22016, calls back to back: 17.3 -> 16.2 us).
        if (!p.w_early && p.m_blocks == 1 && first < p.n_tiles) {
            const int n0 = first * p.R;
            const uint32_t w_bytes = (uint32_t)min(p.R, (p.outs - n0 + 7) / 8 * 8) * kKb;
            const size_t kb_stride = (size_t)((p.outs + 7) / 8) * 1024;
            const uint8_t* const w_tile = p.w + (size_t)kb0 * kb_stride + (size_t)(n0 >> 3) * 1024;
            if (elect_one())
                for (int i = 0, u = u_first; i < min(S, n_units); ++i) {
                    for (int j = 0; j < p.unit && u * p.unit + j < n_kb; ++j)
                        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(w_tile + (size_t)(u * p.unit + j) * kb_stride), "r"(w_bytes) : "memory");
                    if (++u == n_units) u = 0;
                }
            __syncwarp();
        }
    } else {
        pdl_wait();
        const int q4 = warp & 3, group = (warp - 4) >> 2;         // TMEM lane quadrant; two warps share it and take turns
        uint32_t* const stage = stage_s + (warp - 4) * 1024;
        float* const sw = sw_s + (warp - 4) * 288;                // a copy of the tile's scales per warp: no barrier needed
        float* const sx = sw + 256;
        const int tl = q4 * 32 + lane;
        int seg = 0;
        bool ok = true;
        TileScales scales;
        auto place = [&](int tile, int& n0, long long& t0) {
            const int nt = p.m_blocks == 1 ? tile : tile / p.m_blocks;
            n0 = nt * p.R;
            t0 = (long long)(tile - nt * p.m_blocks) * 128 + q4 * 32;
        };
        int n0 = 0;
        long long t0 = 0;
        if (first < p.n_tiles) {
            place(first, n0, t0);
            scales.fetch(p, n0, t0, lane);
        }
        for (int tile = first; tile < p.n_tiles && ok; tile += G, ++seg) {
            const int b = seg & 1;
            place(tile, n0, t0);
            const long long t = t0 + lane;
            const int n_tokens = (int)min(32ll, p.rows - t0);      // valid tokens of this warp (negative: none)
            scales.put(sw, sx, lane);
            if (tile + G < p.n_tiles) {
                int n1;
                long long t1;
                place(tile + G, n1, t1);
                scales.fetch(p, n1, t1, lane);
            }
            ok = warp_wait(&ctrl->acc_full[b], (seg >> 1) & 1, abort_flag) && !__any_sync(0xffffffffu, *abort_flag);
            tc_fence_after_sync();
            const bool busy = n_tokens > 0;
            const uint32_t taddr = tmem + ((uint32_t)(q4 * 32) << 16) + (uint32_t)(b * p.R);
            if (p.split > 1) {
                const int n_groups = p.R / 16;
                cluster_wait();
                if (busy) {
                    int turn = 0;
                    for (int g = 0, owner = 0, slot = 0; g < n_groups; ++g) {
                        if (owner != rank && (turn++ & 1) == group) {
                            uint32_t acc[16];
                            tmem_load<16>(taddr + g * 16, acc);
                            tmem_loaded<16>(acc);
                            if (tl < p.x_rows) {
                                const int from = rank < owner ? rank : rank - 1;
                                const uint32_t dst = cluster_addr(smem_u32(recv), owner) + (uint32_t)(slot * (p.split - 1) + from) * part_bytes(p.x_rows);
#pragma unroll
                                for (int i = 0; i < 4; ++i) st_cluster_v4(dst + part_piece(p.x_rows, tl, i), acc + 4 * i);
                            }
                            __syncwarp();
                        }
                        if (++owner == p.split) { owner = 0; ++slot; }
                    }
                }
                __syncwarp();
                cluster_arrive();
                cluster_wait();
                if (ok && busy) {
                    for (int slot = group, g = rank + group * p.split; g < n_groups && n0 + g * 16 < p.outs; slot += 2, g += 2 * p.split) {
                        uint32_t acc[16];
                        tmem_load<16>(taddr + g * 16, acc);
                        tmem_loaded<16>(acc);
                        if (t < p.rows) {
                            for (int from = 0; from < p.split - 1; ++from) {
                                const uint8_t* src = recv + (size_t)(slot * (p.split - 1) + from) * part_bytes(p.x_rows);
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const uint4 v = *reinterpret_cast<const uint4*>(src + part_piece(p.x_rows, tl, i));
                                    acc[4 * i] += v.x;
                                    acc[4 * i + 1] += v.y;
                                    acc[4 * i + 2] += v.z;
                                    acc[4 * i + 3] += v.w;
                                }
                            }
                        }
                        stage_cols<16>(acc, stage, lane);
                        store_cols<16>(p, t0, n_tokens, n0 + g * 16, min(16, p.outs - n0 - g * 16), sx, sw + g * 16, stage, lane);
                    }
                }
            }
            auto release = [&] {                                   // the accumulator may be overwritten as far as this warp goes
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) arrive_read(&ctrl->acc_empty[b]);
            };
            if (p.split == 1 && ok && busy) store_tile(p, taddr, group, t0, n_tokens, n0, sx, sw, stage, lane, release);
            else release();
        }
    }
    if (p.split > 1 && warp < 4) {            // the other warps' part in the two phases of the cluster barrier
        __syncwarp();
        cluster_wait();
        cluster_arrive();
        cluster_wait();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) drain(ctrl, S, issued, segs);      // whoever raised the flag did so before this barrier
    if (warp == 2) {
        __syncwarp();
        tc_fence_after_sync();
        tmem_dealloc(tmem, p.tmem_cols);
    }
    if (threadIdx.x == 0 && *abort_flag) report(p.d_status, CATS_ERR_TIMEOUT);
}

// ---------------------------------------------------------------------------------------------------------------------
// The same product for many tokens, where it is bound by the tensor cores and by what an SM takes in: a pair of CTAs on two
// SMs works on one tile of 256 tokens x R channels (tcgen05 cta_group::2).  Each CTA brings its 128 tokens and half of the
// tile's channels, (128 + R / 2) rows per K block for 128 x R sums, where a CTA on its own takes in 128 + R; that is what lets
// the tensor cores keep up their rate (4093 x 4096 x 22016: 220 to 240 us, 3360 to 3080 TOP/s as the power limit allows; single CTAs on
// 128 x 256 tiles 301 us beside the former).
// Copies of both CTAs count on the first CTA's barrier, whose warp 2 issues the MMAs for both; commits arrive at both.
// ---------------------------------------------------------------------------------------------------------------------
constexpr uint32_t kFirstOfPair = 0xFEFFFFFFu;       // a shared-memory address in the pair's first CTA

__device__ __forceinline__ uint32_t idesc_i8_m256(int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(256 >> 4) << 24);
}
__device__ __forceinline__ void umma_i8_pair(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %5};\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], da, db, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi)
        : "memory");
}
__device__ __forceinline__ void commit_pair(uint64_t* bar) {      // arrives at this barrier of both CTAs
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(smem_u32(bar)), "h"((uint16_t)3)
                 : "memory");
}
__device__ __forceinline__ void tma_load_pair(void* smem_dst, const void* tmap, int32_t x, int32_t y, uint64_t* bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%2, %3}], [%4], %5;"
        ::"r"(smem_u32(smem_dst)), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(smem_u32(bar) & kFirstOfPair), "l"(policy)
        : "memory");
}
__device__ __forceinline__ void arrive_first(uint64_t* bar) {     // at the first CTA's barrier; relaxed as arrive_read
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(smem_u32(bar) & kFirstOfPair) : "memory");
}

__device__ __forceinline__ void mbar_complete_tx(uint64_t* bar, uint32_t bytes) {      // as if a copy of so many bytes had landed
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// As drain, for a pair.  The barriers of all copies are the first CTA's, whose two copying warps announce both CTAs' bytes.  They
// make up for stages that not all four copying warps came to issue: an arrival with the bytes that the other CTA
// did ask for, or the bytes that it did not ask for.  (All four have issued whatever stage was consumed, so again less than S stages.)
__device__ __noinline__ void drain_pair(Ctrl* ctrl, int S, int rank, int issued, int segs, uint32_t w_chunk, uint32_t x_chunk) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned long long t0 = globaltimer_ns();
    if (lane == 0 && warp <= 1) st_cluster(cluster_addr(smem_u32(&ctrl->issued[2 * rank + warp]), 0), (uint32_t)issued);
    if (lane == 0 && warp == 2 && rank == 0)
        for (int r = 0; r < 2; ++r) st_cluster(cluster_addr(smem_u32(&ctrl->segs), r), (uint32_t)segs);
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    if (rank == 0 && warp <= 1) {
        const volatile int* const n = ctrl->issued;
        const int peer = n[2 + warp], last = max(max(n[0], n[1]), max(n[2], n[3]));
        const uint32_t chunk = warp == 0 ? w_chunk : x_chunk;
        if (lane == 0)
            for (int j = max(0, last - S); j < last; ++j) {
                uint64_t* const bar = &ctrl->full[j % S];
                if (j < issued) {
                    if (j >= peer) mbar_complete_tx(bar, chunk);
                } else if (j < peer) {
                    mbar_expect_tx(bar, chunk);
                } else {
                    mbar_arrive(bar);
                }
            }
        __syncwarp();
        for (int j = max(0, last - S); j < last; ++j) drain_wait(&ctrl->full[j % S], (j / S) & 1, t0);
    } else if (warp == 2) {                   // commits arrive at both CTAs
        segs = *(const volatile int*)&ctrl->segs;
        if (segs > 0) drain_wait(&ctrl->acc_full[(segs - 1) & 1], ((segs - 1) >> 1) & 1, t0);
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();
}

__global__ void __launch_bounds__(kThreads) k_linear_i8_pair(const LinearDev p, const __grid_constant__ CUtensorMap tm_x,
                                                             const __grid_constant__ CUtensorMap tm_w) {
    extern __shared__ __align__(1024) uint8_t smem[];      // [stages][128 tokens, R / 2 channels], staging tiles, scales, control block
    uint32_t* const stage_s = reinterpret_cast<uint32_t*>(smem + (size_t)p.stages * p.stage_bytes);
    float* const sw_s = reinterpret_cast<float*>(stage_s + kEpiWarps * 1024);
    Ctrl* const ctrl = reinterpret_cast<Ctrl*>(sw_s + kEpiWarps * 288);
    volatile int* const abort_flag = &ctrl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank();
    if ((smem_u32(smem) & 1023u) != 0) {      // the swizzled tiles need this alignment (the same address in both CTAs)
        if (threadIdx.x == 0) report(p.d_status, CATS_ERR_UNSUPPORTED);
        return;
    }
    if (warp == 0) {                          // one stage's barriers per lane
        if (lane < p.stages) {
            mbar_init(&ctrl->full[lane], 2);  // the first CTA's: one arrive.expect_tx from each of its copying warps, for both CTAs' bytes
            mbar_init(&ctrl->empty[lane], 1);
        } else if (lane >= 30) {
            mbar_init(&ctrl->acc_full[lane - 30], 1);
            mbar_init(&ctrl->acc_empty[lane - 30], 2 * kEpiWarps);        // the first CTA's: the epilogue warps of both
        }
        if (lane == 0) ctrl->abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 1 && lane == 0) {
        tma_prefetch_desc(&tm_x);
        tma_prefetch_desc(&tm_w);
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctrl->tmem_base)), "r"(p.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_arrive();                         // the peer's barriers are set up and its tensor memory is there
    cluster_wait();
    tc_fence_after_sync();
    const uint32_t tmem = ctrl->tmem_base;
    pdl_launch_dependents();
    const int S = p.stages, G = (int)gridDim.x / 2, first = (int)cluster_id();
    const int n8 = (p.outs + 7) / 8;
    int issued = 0, segs = 0;                 // as in k_linear_i8
    if (warp <= 1) {
        const bool is_w = warp == 0;
        const uint64_t pol = l2_policy_evict_last();
        if (!is_w || !p.w_early) pdl_wait();
        int s = 0;
        uint32_t par = 1;
        bool ok = true;
        for (int tile = first; tile < p.n_tiles && ok; tile += G) {
            const int nt = tile / p.m_blocks, mb = tile - nt * p.m_blocks;
            const int w_row = nt * p.R / 8 + rank * (p.R / 16), x_row = mb * 256 + rank * 128;
            for (int kb = 0; kb < p.n_kb; ++kb) {
                if (issued == S) pdl_wait();
                if (issued >= S && !warp_wait(&ctrl->empty[s], par, abort_flag)) { ok = false; break; }
                uint8_t* const stage = smem + (size_t)s * p.stage_bytes;
                if (elect_one()) {
                    if (is_w) {
                        if (rank == 0) mbar_expect_tx(&ctrl->full[s], 2 * p.w_chunk);
                        tma_load_pair(stage + p.x_chunk, &tm_w, 0, kb * n8 + w_row, &ctrl->full[s], pol);
                    } else {
                        if (rank == 0) mbar_expect_tx(&ctrl->full[s], 2 * p.x_chunk);
                        if (!(p.drop_x && kb == p.n_kb - 1)) tma_load_pair(stage, &tm_x, kb * kKb, x_row, &ctrl->full[s], pol);
                    }
                }
                __syncwarp();
                ++issued;
                if (++s == S) { s = 0; par ^= 1u; }
            }
        }
    } else if (warp == 2) {
        if (rank == 0) {
            pdl_wait();
            const uint32_t idesc = idesc_i8_m256(p.R);
            int s = 0;
            uint32_t par = 0;
            bool ok = !p.give_up;
            if (!ok) *abort_flag = 1;
            for (int tile = first; tile < p.n_tiles && ok; tile += G, ++segs) {
                const int b = segs & 1;
                if (segs >= 2) ok = warp_wait(&ctrl->acc_empty[b], ((segs >> 1) - 1) & 1, abort_flag);
                tc_fence_after_sync();
                const uint32_t d = tmem + (uint32_t)(b * p.R);
                for (int kb = 0; kb < p.n_kb && ok; ++kb) {
                    ok = warp_wait(&ctrl->full[s], par, abort_flag);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint32_t x_addr = smem_u32(smem) + (uint32_t)s * p.stage_bytes;
                    const uint32_t da = desc_lo(x_addr), db = desc_lo(x_addr + p.x_chunk);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) umma_i8_pair(d, da + 2 * k, db + 2 * k, idesc, kb > 0 || k > 0);
                        commit_pair(&ctrl->empty[s]);
                    }
                    __syncwarp();
                    if (++s == S) { s = 0; par ^= 1u; }
                }
                if (elect_one()) commit_pair(&ctrl->acc_full[b]);      // also on abort, so that the epilogue warps wake up
                __syncwarp();
            }
        }
    } else if (warp >= 4) {
        pdl_wait();
        const int q4 = warp & 3, group = (warp - 4) >> 2;         // TMEM lane quadrant; two warps share it and take turns
        uint32_t* const stage = stage_s + (warp - 4) * 1024;
        float* const sw = sw_s + (warp - 4) * 288;
        float* const sx = sw + 256;
        int seg = 0;
        bool ok = true;
        TileScales scales;
        auto place = [&](int tile, int& n0, long long& t0) {
            const int nt = tile / p.m_blocks;
            n0 = nt * p.R;
            t0 = (long long)(tile - nt * p.m_blocks) * 256 + rank * 128 + q4 * 32;
        };
        int n0 = 0;
        long long t0 = 0;
        if (first < p.n_tiles) {
            place(first, n0, t0);
            scales.fetch(p, n0, t0, lane);
        }
        for (int tile = first; tile < p.n_tiles && ok; tile += G, ++seg) {
            const int b = seg & 1;
            place(tile, n0, t0);
            const int n_tokens = (int)min(32ll, p.rows - t0);      // valid tokens of this warp (negative: none)
            scales.put(sw, sx, lane);
            if (tile + G < p.n_tiles) {
                int n1;
                long long t1;
                place(tile + G, n1, t1);
                scales.fetch(p, n1, t1, lane);
            }
            ok = warp_wait(&ctrl->acc_full[b], (seg >> 1) & 1, abort_flag) && !__any_sync(0xffffffffu, *abort_flag);
            tc_fence_after_sync();
            const uint32_t taddr = tmem + ((uint32_t)(q4 * 32) << 16) + (uint32_t)(b * p.R);
            auto release = [&] {
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) arrive_first(&ctrl->acc_empty[b]);
            };
            if (ok && n_tokens > 0) store_tile(p, taddr, group, t0, n_tokens, n0, sx, sw, stage, lane, release);
            else release();
        }
    }
    // An abort concerns both CTAs: the warp that raised the flag, if no other, sees it here and raises the peer's too.
    if (lane == 0 && *abort_flag) st_cluster(cluster_addr(smem_u32(&ctrl->abort_flag), rank ^ 1), 1);
    tc_fence_before_sync();
    __syncwarp();
    cluster_arrive();                         // nobody leaves while its peer may still reach into its memory
    cluster_wait();
    if (*abort_flag) drain_pair(ctrl, S, rank, issued, segs, p.w_chunk, p.x_chunk);
    if (warp == 2) {
        tc_fence_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.tmem_cols) : "memory");
    }
    if (threadIdx.x == 0 && *abort_flag) report(p.d_status, CATS_ERR_TIMEOUT);
}

// ---------------------------------------------------------------------------------------------------------------------
// The same product for very few tokens (one-token passes): there the tensor-core kernel above is a chain of latencies -- set-up,
// copy, MMA, exchange, store -- around a copy of 2 to 3 us.  Here a block of eight warps takes one 8-row group of w (several, if
// there are fewer K blocks than warps); its warps take the K blocks in turn, a lane one 16-byte piece of rows r and r + 4 per K block straight into registers, four-way
// products on the ordinary cores (dp4a), T times as many as there are tokens.
// ---------------------------------------------------------------------------------------------------------------------
struct FewDev {
    const int8_t* x;
    long long ldx;
    const float *sx, *sw;
    const uint8_t* w;
    int rows, cols, outs, n_kb;
    int kw;                 // warps that share a group's K blocks: 1, 2, 4 or 8
    void* out;
    int out_f32;
    long long ldo;
};

// 16 columns of a row; columns from cols on are not read and count as zero
__device__ __forceinline__ int4 load_x16(const int8_t* row, int col, int cols) {
    if (col + 16 <= cols) return *reinterpret_cast<const int4*>(row + col);
    int v[4] = {0, 0, 0, 0};
    for (int i = 0; col + i < cols; ++i) v[i >> 2] |= (int)((uint32_t)(uint8_t)row[col + i] << (8 * (i & 3)));
    return make_int4(v[0], v[1], v[2], v[3]);
}

template <int T> __global__ void __launch_bounds__(256) k_linear_i8_few(const FewDev p) {
    constexpr int U = T <= 2 ? 2 : 1;         // K blocks per step: 2 U loads of w in flight per lane
    __shared__ int red[8][8][T];
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = lane & 7, r = lane >> 3;
    const int kw = p.kw, groups = 8 / kw, n8 = (p.outs + 7) / 8;
    const int group = (int)blockIdx.x * groups + warp / kw, first = warp % kw;
    const size_t kb_stride = (size_t)n8 * 1024;
    const int n_kb = group < n8 ? p.n_kb : 0;
    const uint8_t* const w0 = p.w + (size_t)group * 1024 + r * 128 + ((c ^ r) << 4);
    const uint8_t* const w1 = p.w + (size_t)group * 1024 + (r + 4) * 128 + ((c ^ (r + 4)) << 4);
    // into L2 while the kernel in front finishes, as in k_linear_i8 (1 x 4096 x 4096, calls back to back: 4.2 -> 3.7 us)
    if (c == 0)
        for (int u = 0; u < 4 && first + kw * u < n_kb; ++u) {
            asm volatile("prefetch.global.L2 [%0];" ::"l"(w0 + (first + kw * u) * kb_stride));
            asm volatile("prefetch.global.L2 [%0];" ::"l"(w1 + (first + kw * u) * kb_stride));
        }
    pdl_wait();
    int acc[2][T] = {};
    for (int kb = first; kb < n_kb; kb += kw * U) {
        int4 a[U][2], b[U][T];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = kb + kw * u;
            const bool in = k < n_kb;
            a[u][0] = in ? __ldcs(reinterpret_cast<const int4*>(w0 + k * kb_stride)) : make_int4(0, 0, 0, 0);
            a[u][1] = in ? __ldcs(reinterpret_cast<const int4*>(w1 + k * kb_stride)) : make_int4(0, 0, 0, 0);
#pragma unroll
            for (int t = 0; t < T; ++t)
                b[u][t] = in && t < p.rows ? load_x16(p.x + t * p.ldx, k * kKb + c * 16, p.cols) : make_int4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    acc[h][t] = __dp4a(a[u][h].x, b[u][t].x, acc[h][t]);
                    acc[h][t] = __dp4a(a[u][h].y, b[u][t].y, acc[h][t]);
                    acc[h][t] = __dp4a(a[u][h].z, b[u][t].z, acc[h][t]);
                    acc[h][t] = __dp4a(a[u][h].w, b[u][t].w, acc[h][t]);
                }
    }
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) acc[h][t] += __shfl_xor_sync(0xffffffffu, acc[h][t], o);
            if (c == 0) red[warp][r + 4 * h][t] = acc[h][t];
        }
    __syncthreads();
    if (threadIdx.x < 8 * T * groups) {       // consecutive threads: consecutive channels of one token
        const int ch = threadIdx.x % (8 * groups), t = threadIdx.x / (8 * groups), n = (int)blockIdx.x * 8 * groups + ch;
        int sum = 0;
        for (int i = 0; i < kw; ++i) sum += red[(ch >> 3) * kw + i][ch & 7][t];
        if (t < p.rows && n < p.outs) {
            const float v = (float)sum * p.sx[t] * p.sw[n];
            if (p.out_f32) ((float*)p.out)[t * p.ldo + n] = v;
            else ((uint16_t*)p.out)[t * p.ldo + n] = float_to_bf16_bits(v);
        }
    }
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
        if (col + 16 <= cols && ((uintptr_t)s & 15) == 0) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(s));
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else for (int i = 0; i < 16 && col + i < cols; ++i) w[i >> 2] |= ((uint32_t)(uint8_t)s[i]) << (8 * (i & 3));
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

inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// The packed weights as rows of one 8-row group (1 KB) each, K block by K block, in boxes of box_groups groups.
bool w_tensor_map(const I8Linear& p, int box_groups, CUtensorMap* out) {
    TensorMapEncodeFn enc = tensor_map_encoder();
    if (enc == nullptr) return false;
    const cuuint64_t dims[2] = {256, (cuuint64_t)ceil_div(p.cols, kKb) * (cuuint64_t)ceil_div(p.outs, 8)};
    const cuuint64_t strides[1] = {1024};
    const cuuint32_t box[2] = {256, (cuuint32_t)box_groups};
    const cuuint32_t estr[2] = {1, 1};
    return enc(out, CU_TENSOR_MAP_DATA_TYPE_INT32, 2, const_cast<void*>(p.w), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Tiling {
    int R, split, pair;
    float ns;
};

// Channels per tile, CTAs per tile, or CTA pairs, by the time of the busiest SM.  Measured: an SM takes in 95 bytes of w and x
// per ns (128 x 11008 x 4096, from L2), all of them together move 6500 bytes of w and out per ns (HBM); the four MMAs of a K
// block cost their issuing warp 0.15 us however small they are (1 x 4096 x 4096 as 128 whole tiles 8.4 us, as 32 tiles in
// four shares 6.5); exchanging partial sums costs 1.2 us and 1 ns per 40 bytes sent (77 x 5120 x 15360: whole tiles 15.8,
// halves 17.2 us; 128 x 11008 x 4096: whole tiles 18.9, halves 15.6, quarters 13.4 us); a call ends 6 ns per channel of a tile
// after its last sum; a tile cannot follow another in less than its epilogue takes (4096 x 128 x 8192: 32, 64, 128, 256
// channels 67.9, 40.1, 30.3, 25.5 us, in pairs of 64, 128, 256 35.3, 28.4, 25.2); a pair takes 1 us more to set up and gains
// from a few hundred tokens on (160 x 4096 x 4096: 10.6 against 9.5 us, 300: 12.0 against 11.5, 1000: 17.1 against 20.5;
// 4093 x 4096 x 22016: 219 against 301).  clusters[i]: clusters of 2^i CTAs that fit the device at once.
Tiling linear_tiling(const I8Linear& p, int m_blocks, int x_rows, const int (&clusters)[4]) {
    const int n_kb = ceil_div(p.cols, kKb);
    const float hbm_ns = ((float)p.outs * p.cols + (float)p.rows * p.outs * (p.out_f32 ? 4 : 2)) / 6500.f;
    Tiling best = {256, 1, 0, 1e30f};
    for (int i = 0; i < 4; ++i) {
        const int c = 1 << i;
        const int share = ceil_div(n_kb, c);
        if ((c - 1) * share >= n_kb) break;                         // a CTA without K blocks
        for (int R = 256; R >= 16; R -= 16) {
            const long long tiles = (long long)m_blocks * ceil_div(p.outs, R);
            if (c > 1 && tiles > clusters[i]) break;
            if (ceil_div(R / 16, c) * (c - 1) * (x_rows * 64) > 64 * 1024) continue;      // received partials: 64 KB at most
            const float waves = (float)((tiles + clusters[i] - 1) / clusters[i]);
            const float kb_ns = fmaxf((float)(R + x_rows) * (kKb / 95.f), 150.f);
            const float sent_ns = c > 1 ? 1200.f + (float)(R * (c - 1) / c) * (float)x_rows * (4.f / 40.f) : 0.f;
            const float tile_ns = (float)share * kb_ns;
            const float sm_ns = tile_ns + (waves - 1.f) * fmaxf(tile_ns, 950.f + 10.5f * R);
            // the two overlap, but not quite: of tilings that HBM bounds, the one that leaves the SMs the most slack is best
            const float ns = fmaxf(sm_ns, hbm_ns) + 0.25f * fminf(sm_ns, hbm_ns) + sent_ns + 6.f * R / c;
            if (ns < best.ns) best = {R, c, 0, ns};
        }
    }
    // CTA pairs on 256 tokens: half the channels to take in, and 2 R clocks of the tensor cores
    if (p.rows > 128 && clusters[1] > 0)
        for (int R = 256; R >= 64; R -= 32) {
            const long long tiles = (long long)ceil_div(p.rows, 256) * ceil_div(p.outs, R);
            const float waves = (float)((tiles + clusters[1] - 1) / clusters[1]);
            const float tile_ns = (float)n_kb * fmaxf(fmaxf((float)(R / 2 + 128) * (kKb / 95.f), 2.f * R / 1.7f), 150.f);
            const float sm_ns = tile_ns + (waves - 1.f) * fmaxf(tile_ns, 500.f + 12.f * R);
            const float ns = fmaxf(sm_ns, hbm_ns) + 0.25f * fminf(sm_ns, hbm_ns) + 1000.f + 6.f * R;
            if (ns < best.ns) best = {R, 1, 1, ns};
        }
    return best;
}

// The same for the kernel for few tokens; the tensor cores' kernels take 1.5 us more than linear_tiling counts.  A block
// takes the time of its weights at 6500 bytes per ns for all blocks together, or of its instructions, about 2 ns.  Measured, it
// against the tensor cores, us: one token 3.8 / 6.7 (4096 x 4096), 8.5 / 10.3 (11008 x 4096), 14.1 / 16.2 (4096 x 22016), 10.5 /
// 8.0 (1024 x 32000), 26.6 / 11.9 (640 x 100000); two tokens 4.1 / 6.7, 8.6 / 10.4 (11008 x 4096), 10.0 / 10.3 (4096 x 12288);
// four tokens 5.0 / 6.8, 10.5 / 10.3, 12.5 / 10.2.
inline int few_warps(int n_kb) { return n_kb > 4 ? 8 : (n_kb > 2 ? 4 : n_kb); }     // that share a group's K blocks
float few_ns(const I8Linear& p) {
    if (p.rows > 4) return 1e30f;
    const int n_kb = ceil_div(p.cols, kKb), groups = 8 / few_warps(n_kb);
    const float blocks = (float)ceil_div(ceil_div(p.outs, 8), groups);
    const float work = 1.8f + 0.25f * p.rows + (p.cols % 16 ? 1.5f * p.rows : 0.f);
    const float bytes = (float)n_kb * groups * (1024.f / 6500.f) * (1.f + 0.13f * (p.rows - 1));
    return 1500.f + blocks * fmaxf(work, bytes);
}
cudaError_t launch_few(const I8Linear& p, cudaStream_t st) {
    const int n_kb = ceil_div(p.cols, kKb), kw = few_warps(n_kb);
    const FewDev f = {p.x, p.ldx, p.sx, p.sw, (const uint8_t*)p.w, p.rows, p.cols, p.outs, n_kb, kw, p.out, p.out_f32, p.ldo};
    const dim3 grid((unsigned)ceil_div(ceil_div(p.outs, 8), 8 / kw));
    if (p.rows == 1) return launch_i8(k_linear_i8_few<1>, grid, dim3(256), 0, st, f);
    if (p.rows == 2) return launch_i8(k_linear_i8_few<2>, grid, dim3(256), 0, st, f);
    return launch_i8(k_linear_i8_few<4>, grid, dim3(256), 0, st, f);
}

template <typename... Maps>
cudaError_t launch_clusters(void (*kernel)(LinearDev, Maps...), int cluster, int grid, size_t smem, cudaStream_t st, const LinearDev& d,
                            const Maps&... maps) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)cluster, 1, 1};
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = g_call_boundary && !g_call_overlaps ? 1 : 2;
    g_call_boundary = false;
    ++g_launch_count;
    return cudaLaunchKernelEx(&cfg, kernel, d, maps...);
}

// Per device, once: large shared memory for the kernel, and how many clusters of 2, 4 and 8 CTAs (one CTA per SM) fit at once.
cudaError_t linear_device(const int (**clusters)[4]) {
    static int known[64][4];
    static std::mutex mu;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(mu);
    *clusters = &known[dev];
    if (known[dev][0] != 0) return cudaSuccess;
    e = cudaFuncSetAttribute(k_linear_i8, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_linear_i8_pair, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
    if (e != cudaSuccess) return e;
    for (int i = 1; i < 4; ++i) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(kSms / (1 << i) * (1 << i));
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = kSmemMax;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {1u << i, 1, 1};
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&known[dev][i], k_linear_i8, &cfg);
        if (e != cudaSuccess) return e;
    }
    known[dev][0] = kSms;
    return cudaSuccess;
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
    const int(*clusters)[4];
    cudaError_t e = linear_device(&clusters);
    if (e != cudaSuccess) return e;
    LinearDev d = {};
    d.rows = p.rows; d.outs = p.outs; d.n_kb = ceil_div(p.cols, kKb);
    d.m_blocks = ceil_div(p.rows, 128);
    d.x_rows = p.rows >= 128 ? 128 : ceil_div(p.rows, 8) * 8;
    const Tiling tiling = linear_tiling(p, d.m_blocks, d.x_rows, *clusters);
    if (few_ns(p) < tiling.ns + 1500.f) return launch_few(p, st);
    d.R = tiling.R;
    d.split = tiling.split;
    d.kb_share = ceil_div(d.n_kb, d.split);
    if (tiling.pair) d.m_blocks = ceil_div(p.rows, 256);
    const long long tiles = (long long)d.m_blocks * ceil_div(p.outs, d.R);
    if (tiles > (1ll << 30)) return cudaErrorInvalidValue;
    d.n_tiles = (int)tiles;
    d.w_chunk = (uint32_t)(tiling.pair ? d.R / 2 : d.R) * kKb;
    d.x_chunk = (uint32_t)d.x_rows * kKb;
    // K blocks per stage: up to 40 KB, so that one barrier round trip carries enough bytes
    d.unit = tiling.pair ? 1 : max(1, min(8, 40 * 1024 / (int)(d.w_chunk + d.x_chunk)));
    d.stage_bytes = d.unit * (d.w_chunk + d.x_chunk);
    d.tail = 128u * kKb - d.x_chunk;
    d.recv_bytes = (uint32_t)(ceil_div(d.R / 16, d.split) * (d.split - 1) * d.x_rows * 64);
    const int fixed = (int)(d.tail + d.recv_bytes) + kEpiWarps * (1024 + 288) * 4 + kCtrl;
    d.stages = min(kMaxStages, (kSmemMax - fixed) / (int)d.stage_bytes);
    if (d.stages < 2) return cudaErrorInvalidConfiguration;
    d.tmem_cols = 32;           // two accumulators; the second one's last columns are read 32 at a time
    while (d.tmem_cols < (uint32_t)(d.R + (d.R + 31) / 32 * 32)) d.tmem_cols *= 2;
    d.w = (const uint8_t*)p.w; d.sx = p.sx; d.sw = p.sw;
    d.out = p.out; d.out_f32 = p.out_f32; d.ldo = p.ldo;
    d.vec_out = ((uintptr_t)p.out % 16) == 0 && (p.ldo * (p.out_f32 ? 4 : 2)) % 16 == 0;
    d.d_status = p.d_status;
    d.drop_x = g_debug_fault == 3;
    d.give_up = g_debug_fault == 4;
    d.w_early = !g_call_boundary;       // not as a call of its own (g_call_overlaps)
    const size_t smem = (size_t)d.stages * d.stage_bytes + fixed;
    CUtensorMap tm_x, tm_w;
    if (!x_tensor_map(p, d.x_rows, &tm_x)) return cudaErrorNotSupported;
    if (tiling.pair) {
        if (!w_tensor_map(p, d.R / 16, &tm_w)) return cudaErrorNotSupported;
        return launch_clusters(k_linear_i8_pair, 2, 2 * (d.n_tiles < kSms / 2 ? d.n_tiles : kSms / 2), smem, st, d, tm_x, tm_w);
    }
    return launch_clusters(k_linear_i8, d.split, d.split > 1 ? d.n_tiles * d.split : (d.n_tiles < kSms ? d.n_tiles : kSms), smem, st, d, tm_x);
}

cudaError_t set_wait_limit_i8(unsigned long long ns) { return cudaMemcpyToSymbol(g_wait_limit_ns, &ns, sizeof(ns)); }

}  // namespace cats
