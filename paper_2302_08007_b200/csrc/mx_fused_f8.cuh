// The fused product kernel (mx_fused_gemm.cuh) for MX4 / MX6 operands re-encoded as E4M3 bytes with a scale per 32 elements
// (bdr_reencode_f8.cu): the same Jobs on tcgen05.mma.kind::mxf8f6f4.block_scale, at twice the bf16 rate and half the operand bytes.
// Products and scales are exact, so results differ from the bf16 kernel's in summation order only.  The pipeline is that of mx_gemm_f8.cuh:
// stages of 128 K with their scale atoms, a warp of the leader CTA that copies the atoms to tensor memory, one accumulator of 256 columns (the
// scales take the rest), which the epilogue warps pull into registers at once so that the next item can begin.  It does nothing when *gate is not
// zero: some element was not representable, and the bf16 kernel, launched behind it with the same gate, computes the product instead (with nothing to do that takes
// 4 us, and 2.6 us the decoding in front of it).
//
// Additionally to mx_fused_gemm.cuh a Job has
//   load8(p, it, kk, rank, dst, bar)   loads of K step kk of 128: A, B, and 512 bytes of scales of A and twice 512 of B behind them
//   column(half, q)                    first of the 32 accumulator columns that finish() gets as v[q]
#pragma once

#include "mx_fused_gemm.cuh"

namespace bdr {
namespace fused {

constexpr int kK8 = 128;                             // K elements (bytes) of a stage
constexpr int kStages8 = 6;
constexpr int kTiles8 = 2 * kRows * kK8;             // A 16 KB + B half 16 KB
constexpr int kStage8Bytes = kTiles8 + 2048;         // tiles, then the scales (1024-byte multiple)
constexpr int kTx8Bytes = kTiles8 + 3 * 512;
constexpr int kThreads8 = (3 + kEpiWarps) * 32;      // producer, MMA / relay, 8 epilogue warps, scale copier
constexpr int kCopyWarp8 = 2 + kEpiWarps;
constexpr size_t kSmem8 = (size_t)kStages8 * kStage8Bytes + kEpiWarps * kTileBytes + 1024 /*bookkeeping*/ + 1024 /*alignment*/;
constexpr uint32_t kScaleCol0 = 256, kScaleCols = 12;  // of tensor memory: first scale column, columns per stage (4 for A, 8 for B)

struct Bars8 {
    uint64_t full[kStages8], full_local[kStages8], empty[kStages8], sf_ready[kStages8], tmem_full, tmem_empty;
    uint32_t tmem_base;
    int failed;
};

template <class Job>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads8, 1) fused_f8_kernel(const __grid_constant__ typename Job::Params p) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* stages = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* const tiles = stages + kStages8 * kStage8Bytes;
    Bars8& bars = *reinterpret_cast<Bars8*>(tiles + kEpiWarps * kTileBytes);
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int cluster_id = blockIdx.x >> 1, n_clusters = gridDim.x >> 1, steps = p.f8.steps;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages8; ++s) {
            mbar_init(&bars.full[s], 2);        // leader: its own bytes (arrive.expect_tx) + the peer's relay
            mbar_init(&bars.full_local[s], 1);  // peer: its own bytes
            mbar_init(&bars.empty[s], 1);       // multicast commit of the MMAs that read the stage
            mbar_init(&bars.sf_ready[s], 1);    // leader: commit of the stage's scale copies
        }
        mbar_init(&bars.tmem_full, 1);                  // multicast commit after an item's last K step
        mbar_init(&bars.tmem_empty, 2 * kEpiWarps);     // leader: every epilogue warp of both CTAs
        bars.failed = 0;
        fence_barrier_init();
    }
    if (warp == 1) tmem_alloc2_cols(&bars.tmem_base, 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = bars.tmem_base;

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const bool open = *p.gate == 0;  // the same for every thread of the grid

    if (!open) {
        // nothing to do but to give the tensor memory back
    } else if (warp == 0) {
        uint64_t* const my_full = rank == 0 ? bars.full : bars.full_local;
        bool ok = true;
        int stage = 0, turn = 0;
        for (int i = cluster_id; i < p.n_items && ok; i += n_clusters) {
            const typename Job::Item item = Job::item(p, i);
            for (int kk = 0; kk < steps; ++kk) {
                if (turn > 0) {
                    ok = mbar_wait_warp(&bars.empty[stage], (turn - 1) & 1);
                    if (!ok) break;
                }
                if (elect_one()) {
                    mbar_expect_tx(&my_full[stage], kTx8Bytes);
                    Job::load8(p, item, kk, (int)rank, stages + stage * kStage8Bytes, &my_full[stage]);
                }
                __syncwarp();
                if (++stage == kStages8) { stage = 0; ++turn; }
            }
        }
        if (!ok) {
            bars.failed = 1;
            // the copies still on their way: one more bounded wait for each
            for (int s = 0; s < kStages8; ++s)
                if (s < stage || turn > 0) mbar_wait(&my_full[s], (s < stage ? turn : turn - 1) & 1);
        }
        __syncwarp();
    } else if (warp == 1) {
        bool ok = true;
        int stage = 0, turn = 0;
        if (rank == 0) {
            int tcount = 0;
            for (int i = cluster_id; i < p.n_items && ok; i += n_clusters, ++tcount) {
                if (tcount >= 1) {  // the epilogues of both CTAs hold the item before in registers
                    ok = mbar_wait_warp(&bars.tmem_empty, (tcount - 1) & 1);
                    if (!ok) break;
                    tc_fence_after();
                }
                for (int kk = 0; kk < steps; ++kk) {
                    ok = mbar_wait_warp(&bars.sf_ready[stage], turn & 1);  // data landed, scales copied
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sa = smem_u32(stages + stage * kStage8Bytes);
                    const uint32_t tsfa = tmem_base + kScaleCol0 + (uint32_t)stage * kScaleCols, tsfb = tsfa + 4;
                    const uint64_t da = make_smem_desc(sa), db = make_smem_desc(sa + kRows * kK8);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < kK8 / 32; ++k)  // 32 bytes of K per MMA; scale byte k of the columns
                            umma2_mxf8(tmem_base, da + (uint64_t)(2 * k), db + (uint64_t)(2 * k), kF8InstrDesc | ((uint32_t)k << 29) | ((uint32_t)k << 4),
                                       (kk | k) != 0, tsfa, tsfb);
                        umma_commit2(&bars.empty[stage]);
                    }
                    __syncwarp();
                    if (++stage == kStages8) { stage = 0; ++turn; }
                }
                if (ok && elect_one()) umma_commit2(&bars.tmem_full);
                __syncwarp();
            }
        } else {
            for (int i = cluster_id; i < p.n_items && ok; i += n_clusters)
                for (int kk = 0; kk < steps; ++kk) {
                    ok = mbar_wait_warp(&bars.full_local[stage], turn & 1);
                    if (!ok) break;
                    if (elect_one()) mbar_arrive_cluster(&bars.full[stage], 0);
                    __syncwarp();
                    if (++stage == kStages8) { stage = 0; ++turn; }
                }
        }
        if (!ok) bars.failed = 1;
        __syncwarp();
        tc_fence_before();
    } else if (warp == kCopyWarp8) {
        if (rank == 0) {
            bool ok = true;
            int stage = 0, turn = 0;
            for (int i = cluster_id; i < p.n_items && ok; i += n_clusters)
                for (int kk = 0; kk < steps; ++kk) {
                    // (the stage's previous MMAs are done: the producer refilled it only after their commit)
                    ok = mbar_wait_warp(&bars.full[stage], turn & 1);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sf = smem_u32(stages + stage * kStage8Bytes) + kTiles8;
                    const uint32_t tsfa = tmem_base + kScaleCol0 + (uint32_t)stage * kScaleCols;
                    if (elect_one()) {
                        sf_copy2(tsfa, make_sf_desc(sf));
                        sf_copy2(tsfa + 4, make_sf_desc(sf + 512));
                        sf_copy2(tsfa + 8, make_sf_desc(sf + 1024));
                        umma_commit2_leader(&bars.sf_ready[stage]);
                    }
                    __syncwarp();
                    if (++stage == kStages8) { stage = 0; ++turn; }
                }
            if (!ok) bars.failed = 1;
        }
        __syncwarp();
        tc_fence_before();
    } else {
        Epi e;
        e.r0 = (int)rank * kRows + (warp & 3) * 32;
        e.half = (warp - 2) >> 2;
        e.lane = lane;
        e.tile = smem_u32(tiles + (warp - 2) * kTileBytes);
        e.tmem = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
        bool ok = true;
        int tcount = 0;
        for (int i = cluster_id; i < p.n_items; i += n_clusters, ++tcount) {
            const typename Job::Item item = Job::item(p, i);
            ok = ok && mbar_wait_warp(&bars.tmem_full, tcount & 1);
            if (!ok) break;
            tc_fence_after();
            uint32_t u[4][32];
#pragma unroll
            for (int q = 0; q < 4; ++q) tmem_ld32_nowait(e.tmem + (uint32_t)Job::column(e.half, q), u[q]);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(&bars.tmem_empty, 0);  // the next item may overwrite the accumulator
            float v[4][32];
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int j = 0; j < 32; ++j) v[q][j] = __uint_as_float(u[q][j]);
            Job::finish(p, item, e, v);
        }
        if (!ok) bars.failed = 1;
        tc_fence_before();
    }
    __syncthreads();
    cluster_sync_all();  // the peer may still be signalling this CTA's barriers
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc2(tmem_base, 512);
    }
    if (threadIdx.x == 0 && bars.failed) atomicCAS(p.status, 0, (int)BDR_ERR_TIMEOUT);
}

// E4M3 bytes [z][rows][K], contiguous: boxes of 128 K x 128 rows, 128-byte swizzle
inline bool make_map8(CUtensorMap* out, const void* base, int64_t K, int64_t rows, int64_t z) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)K, (cuuint64_t)rows, (cuuint64_t)z};
    const cuuint64_t strides[2] = {(cuuint64_t)K, (cuuint64_t)(K * rows)};
    const cuuint32_t box[3] = {(cuuint32_t)kK8, (cuuint32_t)kRows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class Job>
int launch_f8(const typename Job::Params& p, cudaStream_t st) {
    static PerDevice once;
    if (once.get(current_device(), [&]() -> int {  // no occupancy query: cluster kernel, one CTA per SM
            return cudaFuncSetAttribute(fused_f8_kernel<Job>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem8) == cudaSuccess ? 1 : 0;
        }) < 1)
        return BDR_ERR_CUDA;
    return launch_clusters(fused_f8_kernel<Job>, p, kThreads8, kSmem8, st);
}

// Whether a product A [M, K] x W [lines, K] (lines in groups of `group` rows that start on a tile) takes the 8-bit path: formats that E4M3 holds, whole
// tiles, enough work that half the product's time outweighs four more launches (the re-encoding, and the bf16 kernels that look at the flag), and no
// longer a reduction than the re-encoding takes.
inline bool takes_f8(int m_a, int m_w, int64_t M, int64_t lines, int64_t group, int64_t K) {
    return m_a <= 4 && m_w <= 4 && M % 256 == 0 && group % 128 == 0 && K % 128 == 0 && K <= kMostReencodeK && lines % 256 == 0 && M * lines >= (1ll << 35) / K;
}
// Bytes of the re-encoded operands and their scales.
inline int64_t f8_bytes(int64_t M, int64_t lines, int64_t K) { return round_up((M + lines) * K + (M + lines) * K / 32, 256); }

// What the 8-bit kernel needs beside the rest of a Job's parameters.
struct F8 {
    CUtensorMap a, w;
    const uint8_t *sf_a, *sf_w;   // [K / 128][rows / 128][512]
    int row_tiles_a, row_tiles_w, steps;
};
// Re-encodes both operands into `space` (f8_bytes) and describes them; the flag becomes *gate: 0 when the 8-bit kernel is to run.
inline int encode_f8(const bdr_planes_t& a, int m_a, int64_t M, const bdr_planes_t& w, int m_w, int64_t lines, int64_t z, int64_t K, uint8_t* space, int* flag,
                     F8* out, const int** gate, cudaStream_t st) {
    uint8_t *const wa = space, *const ww = wa + M * K, *const sa = ww + lines * K, *const sw = sa + M * K / 32;
    if (cudaMemsetAsync(flag, 0, sizeof(int), st) != cudaSuccess) return BDR_ERR_CUDA;
    const ZeroTiles none = {nullptr, 0, 1, 0, 0, 1, 1};
    const int rc = reencode_rowwise_e4m3(a, m_a, w, m_w, M, lines, K, wa, ww, sa, sw, flag, none, st);
    if (rc) return rc;
    if (!make_map8(&out->a, wa, K, M, 1) || !make_map8(&out->w, ww, K, lines / z, z)) return BDR_ERR_CUDA;
    out->sf_a = sa;
    out->sf_w = sw;
    out->row_tiles_a = (int)(M / 128);
    out->row_tiles_w = (int)(lines / 128);
    out->steps = (int)(K / kK8);
    *gate = flag;
    return BDR_OK;
}

}  // namespace fused
}  // namespace bdr
