// The product kernel behind the fused operators: a persistent, TMA-fed tcgen05 kernel over 256 x 256 accumulators, one cluster of
// two CTAs per SM pair, whose operands and epilogue come from a Job.  The pipeline is that of the dense phase of mx_gemm_ws:
//   warp 0   : one lane issues the TMA loads of this CTA's 128 rows of A and its 128 columns of B (64 K elements, 32 KB) into a ring
//   warp 1   : leader CTA: one lane issues tcgen05.mma.cta_group::2 (M 256, N 256, K 16) into one of two accumulator buffers;
//              peer CTA: relays "my stage is full" to the leader's barrier
//   warps 2-9: epilogue of this CTA's 128 x 256 block of the item, overlapping the next item's main loop
// Ragged sizes cost nothing in the main loop: the tensor maps carry the true extents, what lies beyond them arrives as zeros, and the
// epilogues mask rows and columns.  Every wait is bounded; one that runs out sets the status word and the role leaves its loop.
//
// A Job has
//   Params                         kernel argument (tensor maps and sizes)
//   Item item(p, i)                work item i of p.n_items; Item::steps is its number of K steps of 64
//   load(p, it, kk, rank, dst, bar)   TMA loads of K step kk: exactly kFuStageBytes bytes
//   a_mn(it), b_mn                 whether an operand lies with its rows (M or N) contiguous instead of K
//   kSpan                          K steps after which the accumulator is handed to the epilogue: 0 = at the end of the item
//   epilogue(p, it, r, half, tmem)    (kSpan == 0) row r of 256, columns 128 half .. of the accumulator; `tmem` addresses this warp's lanes
//   finish(p, it, r, half, v)         (kSpan > 0) the same, with the 128 sums in registers
// The tensor core cuts its fp32 additions off instead of rounding them, toward zero: over a chain of n instructions of 16 K each the sum
// loses about n 2^-25 of itself.  That is nothing beside 16-bit results, nor for operands of few bits, whose sums are mostly exact; sums of full-width values for
// 32-bit results are taken kSpan steps at a time and added with rounded additions in the epilogue's registers, while the next span runs.
#pragma once

#include "bdr_host.h"
#include "mx_fused.h"
#include "mx_tc.cuh"

namespace bdr {
namespace fused {

constexpr int kRows = 128;                          // rows of A, and columns of B, per CTA
constexpr int kStages = 6;
constexpr int kOperandBytes = kRows * kBK * 2;      // 16 KB
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kEpiWarps = 8;
constexpr int kThreads = (2 + kEpiWarps) * 32;
constexpr size_t kSmem = (size_t)kStages * kStageBytes + 1024 /*bookkeeping*/ + 1024 /*alignment*/;

struct Bars {
    uint64_t full[kStages], full_local[kStages], empty[kStages], tmem_full[2], tmem_empty[2];
    uint32_t tmem_base;
    int failed;
};

// Descriptor of an operand with its rows contiguous: chunks of 64 rows x 64 K (one TMA box, K rows of 128 bytes, 128-byte swizzle),
// chunks 8 KB apart; eight K rows make 1024 bytes.
__device__ __forceinline__ uint64_t make_mn_desc(uint32_t smem_addr) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(64 * 128 >> 4) << 16;  // between chunks of 64 rows
    d |= (uint64_t)(1024 >> 4) << 32;      // between groups of eight K
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
constexpr uint32_t kMnA = 1u << 15, kMnB = 1u << 16;  // instruction descriptor: the operand's rows are contiguous

template <class Job>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) fused_gemm_kernel(const __grid_constant__ typename Job::Params p) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* stages = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Bars& bars = *reinterpret_cast<Bars*>(stages + kStages * kStageBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int cluster_id = blockIdx.x >> 1, n_clusters = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&bars.full[s], 2);        // leader: its own TMA bytes (arrive.expect_tx) + the peer's relay
            mbar_init(&bars.full_local[s], 1);  // peer: its own TMA bytes
            mbar_init(&bars.empty[s], 1);       // multicast commit of the MMAs that read the stage
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&bars.tmem_full[b], 1);                 // multicast commit after an item's last K step
            mbar_init(&bars.tmem_empty[b], 2 * kEpiWarps);    // leader: every epilogue warp of both CTAs
        }
        bars.failed = 0;
        fence_barrier_init();
    }
    if (warp == 1) tmem_alloc2_cols(&bars.tmem_base, 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = bars.tmem_base;

    // nothing above touched global memory: launched as a programmatic dependent, it overlaps the tail of the kernel before
    asm volatile("griddepcontrol.wait;" ::: "memory");

    if (warp == 0) {
        if (lane == 0) {
            uint64_t* const my_full = rank == 0 ? bars.full : bars.full_local;
            bool ok = true;
            uint32_t it = 0;
            for (int i = cluster_id; i < p.n_items && ok; i += n_clusters) {
                const typename Job::Item item = Job::item(p, i);
                for (int kk = 0; kk < item.steps; ++kk, ++it) {
                    const int stage = it % kStages;
                    if (it >= kStages) {
                        ok = mbar_wait(&bars.empty[stage], ((it / kStages) - 1) & 1);
                        if (!ok) break;
                    }
                    mbar_expect_tx(&my_full[stage], kStageBytes);
                    Job::load(p, item, kk, (int)rank, stages + stage * kStageBytes, &my_full[stage]);
                }
            }
            if (!ok) bars.failed = 1;
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            bool ok = true;
            uint32_t it = 0;
            if (rank == 0) {
                int tcount = 0;
                for (int i = cluster_id; i < p.n_items && ok; i += n_clusters, ++tcount) {
                    const typename Job::Item item = Job::item(p, i);
                    const bool a_mn = Job::a_mn(item);
                    const uint32_t idesc = kPairInstrDesc | (a_mn ? kMnA : 0u) | (Job::b_mn ? kMnB : 0u);
                    const uint64_t a_step = a_mn ? 128 : 2;  // 16 K: two groups of eight K rows, or 32 bytes along a row
                    const uint64_t b_step = Job::b_mn ? 128 : 2;
                    const int span = Job::kSpan ? Job::kSpan : item.steps;
                    int buf = 0, left = 0;  // K steps that the current buffer still takes
                    uint32_t acc = 0;
                    for (int kk = 0; kk < item.steps; ++kk, ++it, --left) {
                        if (left == 0) {
                            if (kk > 0) { umma_commit2(&bars.tmem_full[buf]); ++tcount; }
                            left = span;
                            buf = tcount & 1;
                            acc = tmem_base + (uint32_t)buf * 256u;
                            if (tcount >= 2) {  // the epilogues of both CTAs have drained this buffer
                                ok = mbar_wait_cluster(&bars.tmem_empty[buf], ((tcount >> 1) - 1) & 1);
                                if (!ok) break;
                                tc_fence_after();
                            }
                        }
                        const int stage = it % kStages;
                        ok = mbar_wait_cluster(&bars.full[stage], (it / kStages) & 1);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t sa = smem_u32(stages + stage * kStageBytes), sb = sa + kOperandBytes;
                        const uint64_t da = a_mn ? make_mn_desc(sa) : make_smem_desc(sa);
                        const uint64_t db = Job::b_mn ? make_mn_desc(sb) : make_smem_desc(sb);
#pragma unroll
                        for (int k = 0; k < kBK / 16; ++k) umma2_bf16(acc, da + k * a_step, db + k * b_step, idesc, left != span || k != 0);
                        umma_commit2(&bars.empty[stage]);
                    }
                    if (ok) umma_commit2(&bars.tmem_full[buf]);
                }
            } else {
                for (int i = cluster_id; i < p.n_items && ok; i += n_clusters) {
                    const typename Job::Item item = Job::item(p, i);
                    for (int kk = 0; kk < item.steps; ++kk, ++it) {
                        const int stage = it % kStages;
                        ok = mbar_wait(&bars.full_local[stage], (it / kStages) & 1);
                        if (!ok) break;
                        mbar_arrive_cluster(&bars.full[stage], 0);
                    }
                }
            }
            if (!ok) bars.failed = 1;
        }
        __syncwarp();
        tc_fence_before();
    } else {
        const int ew = warp - 2;
        const uint32_t my_lanes = (uint32_t)((warp & 3) * 32) << 16;  // the tensor-memory lanes this warp may read
        bool ok = true;
        int tcount = 0;
        for (int i = cluster_id; i < p.n_items; i += n_clusters, ++tcount) {
            const typename Job::Item item = Job::item(p, i);
            const int r = (int)rank * kRows + (warp & 3) * 32 + lane, half = ew >> 2;
            auto next = [&](int buf) {  // waits for the next accumulator
                ok = ok && mbar_wait(&bars.tmem_full[buf], (tcount >> 1) & 1);
                ok = __all_sync(0xFFFFFFFFu, ok);
                tc_fence_after();
                return ok;
            };
            auto done = [&](int buf) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(&bars.tmem_empty[buf], 0);
            };
            if constexpr (Job::kSpan == 0) {
                const int buf = tcount & 1;
                if (!next(buf)) break;
                Job::epilogue(p, item, r, half, tmem_base + my_lanes + (uint32_t)buf * 256u);
                done(buf);
            } else {
                float v[4][32];
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[q][j] = 0.f;
                for (int k0 = 0; k0 < item.steps; k0 += Job::kSpan) {
                    if (k0 > 0) ++tcount;
                    const int buf = tcount & 1;
                    if (!next(buf)) break;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t u[32];
                        tmem_ld32(tmem_base + my_lanes + (uint32_t)(buf * 256 + half * 128 + 32 * q), u);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[q][j] += __uint_as_float(u[j]);
                    }
                    done(buf);
                }
                if (!ok) break;
                Job::finish(p, item, r, half, v);
                __syncwarp();
            }
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

// bf16 [z][rows][cols], row pitch `pitch`, z pitch `z_pitch` (elements, multiples of 8): boxes of 64 columns x box_rows, 128-byte swizzle
inline bool make_map(CUtensorMap* out, const void* base, int64_t cols, int64_t rows, int64_t z, int64_t pitch, int64_t z_pitch, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)z};
    const cuuint64_t strides[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)z_pitch * 2};
    const cuuint32_t box[3] = {(cuuint32_t)kBK, (cuuint32_t)box_rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class Job>
int launch(const typename Job::Params& p, cudaStream_t st) {
    static PerDevice once;
    if (once.get(current_device(), [&]() -> int {  // no occupancy query: cluster kernel, one CTA per SM
            return cudaFuncSetAttribute(fused_gemm_kernel<Job>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem) == cudaSuccess ? 1 : 0;
        }) < 1)
        return BDR_ERR_CUDA;
    const int n_clusters = p.n_items < sm_count() / 2 ? p.n_items : sm_count() / 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * n_clusters));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, fused_gemm_kernel<Job>, p);
    return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

// ---- epilogue pieces ----------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// n (at most 32) values of a row, from column `at` of row pointer `row`, rounded once to the type; vec: 16-byte stores are possible
__device__ __forceinline__ void store_run(void* row, int64_t at, const float (&v)[32], int n, bool f32, bool vec) {
    if (f32) {
        float* to = static_cast<float*>(row) + at;
        if (vec && n == 32) {
#pragma unroll
            for (int q = 0; q < 8; ++q) *reinterpret_cast<float4*>(to + 4 * q) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < n) to[j] = v[j];
        }
    } else {
        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(row) + at;
        if (vec && n == 32) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<uint4*>(to + 8 * q) = make_uint4(bf16x2(v[8 * q], v[8 * q + 1]), bf16x2(v[8 * q + 2], v[8 * q + 3]),
                                                                   bf16x2(v[8 * q + 4], v[8 * q + 5]), bf16x2(v[8 * q + 6], v[8 * q + 7]));
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < n) to[j] = __float2bfloat16_rn(v[j]);
        }
    }
}
__device__ __forceinline__ void load_run(const void* row, int64_t at, float (&v)[32], int n, bool f32, bool vec) {
    if (f32) {
        const float* from = static_cast<const float*>(row) + at;
        if (vec && n == 32) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float4 x = *reinterpret_cast<const float4*>(from + 4 * q);
                v[4 * q] = x.x; v[4 * q + 1] = x.y; v[4 * q + 2] = x.z; v[4 * q + 3] = x.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = j < n ? from[j] : 0.f;
        }
    } else {
        const __nv_bfloat16* from = static_cast<const __nv_bfloat16*>(row) + at;
        if (vec && n == 32) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint4 x = *reinterpret_cast<const uint4*>(from + 8 * q);
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[8 * q + 2 * e] = __uint_as_float(w[e] << 16);
                    v[8 * q + 2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = j < n ? __bfloat162float(from[j]) : 0.f;
        }
    }
}
// whether rows of `width`-byte elements at p, ld apart, allow 16-byte accesses at multiples of 32 elements (host)
inline bool rows_aligned(const void* p, int64_t ld, int width) { return (uintptr_t)p % 16 == 0 && ld * width % 16 == 0; }

// The gradient of a product enters the tensor core as bf16.  Gradients of 16 bits take its nearest value: off by 2^-8 of it at most, half a step
// of the results' own type, in every term of their sums.  Gradients of 32 bits take three parts, each the nearest value of
// what the ones before leave: 24 bits, all that the 32-bit value has (unless its last part falls below 2^-133).
constexpr int kPartsF32 = 3;
__device__ __forceinline__ void store_parts(__nv_bfloat16* to, int64_t part_pitch, int parts, float (&v)[32], int n) {
    store_run(to, 0, v, n, false, true);
#pragma unroll 1
    for (int i = 1; i < parts; ++i) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] -= __bfloat162float(__float2bfloat16_rn(v[j]));
        store_run(to + i * part_pitch, 0, v, n, false, true);
    }
}

}  // namespace fused
}  // namespace bdr
