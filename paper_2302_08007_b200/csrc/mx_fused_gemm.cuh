// The product kernel behind the fused operators: a persistent, TMA-fed tcgen05 kernel over 256 x (64, 128, 192 or 256) accumulators, one
// cluster of two CTAs per SM pair, whose operands and epilogue come from a Job.  The pipeline is that of the dense phase of mx_gemm_ws:
//   warp 0   : one lane issues the TMA loads of this CTA's 128 rows of A and its half of B's columns (64 K elements) into a ring
//   warp 1   : leader CTA: one lane issues tcgen05.mma.cta_group::2 (M 256, N the accumulator's columns, K 16) into one of two accumulator
//              buffers;  peer CTA: relays "my stage is full" to the leader's barrier
//   warps 2-9: epilogue of this CTA's 128 rows of the item, overlapping the next item's main loop
// Ragged sizes cost nothing in the main loop: the tensor maps carry the true extents, what lies beyond them arrives as zeros, and the
// epilogues mask rows and columns.  Every wait is bounded; one that runs out sets the status word and the role leaves its loop.
//
// A Job has
//   Params                         kernel argument: tensor maps, sizes, n_items, bn (the accumulator's columns), status; gate: NULL, or device
//                                  flag without which the kernel does nothing
//   Item item(p, i)                work item i of p.n_items; Item::steps is its number of K steps of 64 (p.n_long, p.extra: see Deal)
//   load(p, it, kk, rank, dst, bar)   TMA loads of K step kk: A at dst, B kOperandBytes behind it, 16384 + 64 bn bytes in all
//   a_mn(it), b_mn                 whether an operand lies with its rows (M or N) contiguous instead of K
//   kSpan                          K steps after which the accumulator is handed to the epilogue: 0 = at the end of the item
//   kBack                          (kSpan > 0) the total of the spans goes back to tensor memory; else it stays in registers
//   epilogue(p, it, e)             (kSpan == 0 or kBack) reads the accumulator through e.tmem
//   finish(p, it, e, v)            (kSpan > 0, not kBack) the same, with the sums of a thread's row and half of the columns in registers
//   prefetch(p)                    the tensor maps that load() uses
//   kCut                           whether a tile's K steps may be cut into p.splits items (Item::tile, Item::split): the parts' sums go to
//                                  p.partials, and the warp that comes last (p.counters) adds them in order, puts the total back into its tensor
//                                  memory and runs the epilogue
//   rows(p), chunks(bn, half), chunk(bn, half, i)   (kCut or kBack) the rows that are there, and the 32-column pieces of the accumulator that the
//                                  epilogue of a half reads, four at most
// The tensor core cuts its fp32 additions off instead of rounding them, toward zero: over a chain of n instructions of 16 K each the sum
// loses up to n 2^-25 of itself.  That is nothing beside 16-bit results.  Sums of full-width values for 32-bit results are taken kSpan steps at a
// time and added with rounded additions in the epilogue's registers, while the next span runs.  Products of packed values are sums of 4 to 14
// bits times powers of two, exact as long as 24 bits hold the sum: one_chain says up to where.
#pragma once

#include <algorithm>

#include "bdr_host.h"
#include "mx_fused.h"
#include "mx_tc.cuh"

namespace bdr {
namespace fused {

constexpr int kRows = 128;                          // rows of A, and columns of B, per CTA
constexpr int kStages = 6, kMostStages = 9;          // of 256 columns; narrower ones leave room for more, and a ring's turn takes the same time
constexpr int kOperandBytes = kRows * kBK * 2;      // 16 KB
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kEpiWarps = 8;
constexpr int kThreads = (2 + kEpiWarps) * 32;
constexpr int kTileBytes = 32 * 64;                 // of an epilogue warp, see store_tile
constexpr size_t kSmem = (size_t)kStages * kStageBytes + kEpiWarps * kTileBytes + 1024 /*bookkeeping*/ + 1024 /*alignment*/;

struct Bars {
    uint64_t full[kMostStages], full_local[kMostStages], empty[kMostStages], tmem_full[2], tmem_empty[2];
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
// Instruction descriptor: D = fp32, A = B = bf16, M = 256, N = bn; bits 15 and 16: A's, B's rows are contiguous.
constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(256 >> 4) << 24), kMnA = 1u << 15, kMnB = 1u << 16;

// Which items a cluster takes.  The first n_long items are as long as `extra` of the others, rounded down.  They are dealt out in rounds; the clusters that
// a last round of them does not reach take `extra` of the others each, and the rest is dealt out in rounds again, from the other end.
struct Deal {
    int n_items, n_long, extra, cluster, clusters;
    __device__ __forceinline__ int reached() const { return n_long % clusters; }
    __device__ __forceinline__ int extras() const { return reached() ? (clusters - reached()) * extra : 0; }
    __device__ __forceinline__ int rest() const { return n_long + extras() + clusters - 1 - cluster; }
    __device__ __forceinline__ int others() const {
        return extras() && cluster >= reached() && n_long + (cluster - reached()) * extra < n_items ? n_long + (cluster - reached()) * extra : rest();
    }
    __device__ __forceinline__ int first() const { return cluster < n_long ? cluster : others(); }
    __device__ __forceinline__ int next(int i) const {
        if (i < n_long) return i + clusters < n_long ? i + clusters : others();
        if (i >= n_long + extras()) return i + clusters;
        return (i + 1 - n_long) % extra && i + 1 < n_items ? i + 1 : rest();
    }
};

// What an epilogue warp works on.
struct Epi {
    uint32_t tmem;   // its 32 lanes of the accumulator, column 0
    int r0;          // their first row of the item's 256
    int half, lane;  // two warps share the lanes: half of the columns each
    uint32_t tile;   // shared-memory address of the warp's own 2 KB
};

// A cut tile: stores this part's sums of the warp's rows and columns; true for the warp that finds all parts there, with the total in its
// tensor memory.  Nobody waits.  Slots are 256 x bn floats in pieces of 32 rows x 32 columns, four columns of 32 rows together.
template <class Job>
__device__ __forceinline__ bool last_part(const typename Job::Params& p, const typename Job::Item& it, const Epi& e) {
    const int64_t slot = 256 * p.bn;
    float* const base = p.partials + (int64_t)it.tile * p.splits * slot + e.r0 * p.bn + 4 * e.lane;
    const int n = Job::chunks(p.bn, e.half);
    for (int i = 0; i < n; ++i) {
        const int col = Job::chunk(p.bn, e.half, i);
        __syncwarp();
        uint32_t u[32];
        tmem_ld32(e.tmem + (uint32_t)col, u);
        float* const to = base + it.split * slot + col * 32;
#pragma unroll
        for (int j = 0; j < 8; ++j) __stcg(reinterpret_cast<uint4*>(to + 128 * j), make_uint4(u[4 * j], u[4 * j + 1], u[4 * j + 2], u[4 * j + 3]));
    }
    __threadfence();
    __syncwarp();
    int before = 0;
    if (e.lane == 0) before = atomicAdd(&p.counters[it.tile * 16 + (e.r0 >> 5) * 2 + e.half], 1);
    before = __shfl_sync(0xFFFFFFFFu, before, 0);
    if (before != p.splits - 1) return false;
    __threadfence();
    for (int i = 0; i < n; ++i) {
        const int col = Job::chunk(p.bn, e.half, i);
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = 0.f;
#pragma unroll 2
        for (int s = 0; s < p.splits; ++s) {
            const float* const from = base + s * slot + col * 32;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float4 x = __ldcg(reinterpret_cast<const float4*>(from + 128 * j));
                v[4 * j] += x.x; v[4 * j + 1] += x.y; v[4 * j + 2] += x.z; v[4 * j + 3] += x.w;
            }
        }
        uint32_t u[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) u[j] = __float_as_uint(v[j]);
        __syncwarp();
        tmem_st32(e.tmem + (uint32_t)col, u);
    }
    return true;
}

template <class Job>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) fused_gemm_kernel(const __grid_constant__ typename Job::Params p) {
    static_assert(Job::kSpan == 0 || Job::kBack || !Job::kCut, "the parts of a cut tile are read from tensor memory");
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* stages = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* const tiles = stages + kStages * kStageBytes;
    Bars& bars = *reinterpret_cast<Bars*>(tiles + kEpiWarps * kTileBytes);
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int cluster_id = blockIdx.x >> 1, n_clusters = gridDim.x >> 1;
    const Deal deal = {p.n_items, p.n_long, p.extra, cluster_id, n_clusters};
    const int stage_bytes = kOperandBytes + 64 * p.bn, n_stages = min(kMostStages, kStages * kStageBytes / stage_bytes);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kMostStages; ++s) {
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
    if (threadIdx.x == 32 * kEpiWarps) Job::prefetch(p);
    if (warp == 1) tmem_alloc2_cols(&bars.tmem_base, 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = bars.tmem_base;

    // nothing above touched global memory: launched as a programmatic dependent, it overlaps the tail of the kernel before; and the kernel
    // behind may be set up already
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const bool open = !p.gate || *p.gate != 0;  // the same for every thread of the grid

    if (!open) {
        // the 8-bit kernel has done it
    } else if (warp == 0) {
        // The roles' warps run their loops together, and one elected thread issues: what the instructions take from uniform registers (descriptors,
        // addresses) then stays there.  With one lane in a branch of its own a K step took at least 560 clocks, whatever the columns.
        uint64_t* const my_full = rank == 0 ? bars.full : bars.full_local;
        bool ok = true;
        int stage = 0, turn = 0;  // of the ring
        for (int i = deal.first(); i < p.n_items && ok; i = deal.next(i)) {
            const typename Job::Item item = Job::item(p, i);
            for (int kk = 0; kk < item.steps; ++kk) {
                if (turn > 0) {
                    ok = mbar_wait_warp(&bars.empty[stage], (turn - 1) & 1);
                    if (!ok) break;
                }
                if (elect_one()) {
                    mbar_expect_tx(&my_full[stage], stage_bytes);
                    Job::load(p, item, kk, (int)rank, stages + stage * stage_bytes, &my_full[stage]);
                }
                __syncwarp();
                if (++stage == n_stages) { stage = 0; ++turn; }
            }
        }
        if (!ok) {
            bars.failed = 1;
            // the copies still on their way: one more bounded wait for each
            for (int s = 0; s < n_stages; ++s)
                if (s < stage || turn > 0) mbar_wait(&my_full[s], (s < stage ? turn : turn - 1) & 1);
        }
        __syncwarp();
    } else if (warp == 1) {
        bool ok = true;
        int stage = 0, turn = 0;
        if (rank == 0) {
            int tcount = 0;
            for (int i = deal.first(); i < p.n_items && ok; i = deal.next(i), ++tcount) {
                const typename Job::Item item = Job::item(p, i);
                const bool a_mn = Job::a_mn(item);
                const uint32_t idesc = kIdesc | ((uint32_t)(p.bn >> 3) << 17) | (a_mn ? kMnA : 0u) | (Job::b_mn ? kMnB : 0u);
                const uint64_t a_step = a_mn ? 128 : 2;  // 16 K: two groups of eight K rows, or 32 bytes along a row
                const uint64_t b_step = Job::b_mn ? 128 : 2;
                const int span = Job::kSpan ? Job::kSpan : item.steps;
                int buf = 0, left = 0;  // K steps that the current buffer still takes
                uint32_t acc = 0;
                for (int kk = 0; kk < item.steps; ++kk, --left) {
                    if (left == 0) {
                        if (kk > 0) {
                            if (elect_one()) umma_commit2(&bars.tmem_full[buf]);
                            ++tcount;
                        }
                        left = span;
                        buf = tcount & 1;
                        acc = tmem_base + (uint32_t)buf * 256u;
                        if (tcount >= 2) {  // the epilogues of both CTAs have drained this buffer
                            ok = mbar_wait_warp(&bars.tmem_empty[buf], ((tcount >> 1) - 1) & 1);
                            if (!ok) break;
                            tc_fence_after();
                        }
                    }
                    ok = mbar_wait_warp(&bars.full[stage], turn & 1);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sa = smem_u32(stages + stage * stage_bytes), sb = sa + kOperandBytes;
                    const uint64_t da = a_mn ? make_mn_desc(sa) : make_smem_desc(sa);
                    const uint64_t db = Job::b_mn ? make_mn_desc(sb) : make_smem_desc(sb);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < kBK / 16; ++k) umma2_bf16(acc, da + k * a_step, db + k * b_step, idesc, left != span || k != 0);
                        umma_commit2(&bars.empty[stage]);
                    }
                    __syncwarp();
                    if (++stage == n_stages) { stage = 0; ++turn; }
                }
                if (ok && elect_one()) umma_commit2(&bars.tmem_full[buf]);
                __syncwarp();
            }
        } else {
            for (int i = deal.first(); i < p.n_items && ok; i = deal.next(i)) {
                const typename Job::Item item = Job::item(p, i);
                for (int kk = 0; kk < item.steps; ++kk) {
                    ok = mbar_wait_warp(&bars.full_local[stage], turn & 1);
                    if (!ok) break;
                    if (elect_one()) mbar_arrive_cluster(&bars.full[stage], 0);
                    __syncwarp();
                    if (++stage == n_stages) { stage = 0; ++turn; }
                }
            }
        }
        if (!ok) bars.failed = 1;
        __syncwarp();
        tc_fence_before();
    } else {
        const int ew = warp - 2;
        const uint32_t my_lanes = (uint32_t)((warp & 3) * 32) << 16;  // the tensor-memory lanes this warp may read
        bool ok = true;
        int tcount = 0;
        for (int i = deal.first(); i < p.n_items; i = deal.next(i), ++tcount) {
            const typename Job::Item item = Job::item(p, i);
            Epi e;
            e.r0 = (int)rank * kRows + (warp & 3) * 32;
            e.half = ew >> 2;
            e.lane = lane;
            e.tile = smem_u32(tiles + ew * kTileBytes);
            auto next = [&](int buf) {  // waits for the next accumulator
                ok = ok && mbar_wait_warp(&bars.tmem_full[buf], (tcount >> 1) & 1);
                tc_fence_after();
                return ok;
            };
            auto done = [&](int buf) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(&bars.tmem_empty[buf], 0);
            };
            if constexpr (Job::kSpan == 0 || Job::kBack) {
                if constexpr (Job::kSpan > 0) {
                    const int n = Job::chunks(p.bn, e.half);
                    float v[4][32];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[q][j] = 0.f;
                    auto take = [&](uint32_t from) {
#pragma unroll
                        for (int q = 0; q < 8; ++q) {  // sixteen columns at a time, as below
                            if (q >= 2 * n) break;
                            uint32_t u[16];
                            tmem_ld16(from + (uint32_t)(Job::chunk(p.bn, e.half, q >> 1) + 16 * (q & 1)), u);
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[q >> 1][16 * (q & 1) + j] += __uint_as_float(u[j]);
                        }
                    };
                    for (int k0 = Job::kSpan; k0 < item.steps; k0 += Job::kSpan) {
                        const int buf = tcount & 1;
                        if (!next(buf)) break;
                        take(tmem_base + my_lanes + (uint32_t)buf * 256u);
                        done(buf);
                        ++tcount;
                    }
                    if (!ok) break;
                    if (!next(tcount & 1)) break;
                    if (item.steps > Job::kSpan) {  // the last span's sums give way to the total
                        const uint32_t last = tmem_base + my_lanes + (uint32_t)(tcount & 1) * 256u;
                        take(last);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            if (q >= n) break;
                            uint32_t u[32];
#pragma unroll
                            for (int j = 0; j < 32; ++j) u[j] = __float_as_uint(v[q][j]);
                            __syncwarp();
                            tmem_st32(last + (uint32_t)Job::chunk(p.bn, e.half, q), u);
                        }
                    }
                } else {
                    if (!next(tcount & 1)) break;
                }
                const int buf = tcount & 1;
                e.tmem = tmem_base + my_lanes + (uint32_t)buf * 256u;
                bool mine = true;
                if constexpr (Job::kCut) {
                    mine = item.tm * 256 + e.r0 < Job::rows(p);
                    if (mine && p.splits > 1) mine = last_part<Job>(p, item, e);
                }
                if (mine) Job::epilogue(p, item, e);
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
                    for (int q = 0; q < 8; ++q) {  // sixteen columns at a time: more would not fit beside the sums
                        if (32 * q >= p.bn) break;
                        uint32_t u[16];
                        tmem_ld16(tmem_base + my_lanes + (uint32_t)(buf * 256 + e.half * (p.bn >> 1) + 16 * q), u);
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[q >> 1][16 * (q & 1) + j] += __uint_as_float(u[j]);
                    }
                    done(buf);
                }
                if (!ok) break;
                Job::finish(p, item, e, v);
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

template <class Params>
int launch_clusters(void (*kern)(Params), const Params& p, int threads, size_t smem, cudaStream_t st) {
    const int n_clusters = p.n_items < sm_count() / 2 ? p.n_items : sm_count() / 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * n_clusters));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, p);
    return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

template <class Job>
int launch(const typename Job::Params& p, cudaStream_t st) {
    static PerDevice once;
    if (once.get(current_device(), [&]() -> int {  // no occupancy query: cluster kernel, one CTA per SM
            return cudaFuncSetAttribute(fused_gemm_kernel<Job>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem) == cudaSuccess ? 1 : 0;
        }) < 1)
        return BDR_ERR_CUDA;
    return launch_clusters(fused_gemm_kernel<Job>, p, kThreads, kSmem, st);
}

// ---- epilogue pieces ----------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// A row-major tensor as an epilogue sees it.  align: 16, 4 or 2, the bytes that every row start (and so every multiple of 32 columns) is
// aligned to.
struct Rows {
    void* p;
    int64_t ld;  // bytes
    int f32, align;
    __device__ __forceinline__ char* at(int64_t row, int64_t col) const { return static_cast<char*>(p) + row * ld + col * (f32 ? 4 : 2); }
};
inline Rows make_rows(const void* p, int64_t ld, bool f32) {  // ld in elements (host)
    const int64_t bytes = ld * (f32 ? 4 : 2);
    const uint64_t both = (uintptr_t)p | (uint64_t)bytes;
    return {const_cast<void*>(p), bytes, f32, both % 16 == 0 ? 16 : (both % 4 == 0 ? 4 : 2)};
}

// Tiles of 32 rows x 32 columns between the lanes of a warp (a lane holds a row, as tensor memory gives it) and global memory.  They pass
// through 64 bytes per row of shared memory, the 16-byte pieces of rows 2i and 2i + 1 exchanged by i so that neither side meets in a bank, and
// so that a warp's accesses to global memory run along rows, whatever the rows' alignment.
__device__ __forceinline__ uint32_t tile_at(uint32_t tile, int row, int piece) { return tile + row * 64 + ((piece ^ ((row >> 1) & 3)) << 4); }
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void sts32(uint32_t addr, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ uint16_t lds16(uint32_t addr) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void sts16(uint32_t addr, uint16_t v) { asm volatile("st.shared.u16 [%0], %1;" ::"r"(addr), "h"(v) : "memory"); }

// shared -> global: `rows` rows of n elements (16 fp32 or 32 bf16 at most) to `to`, ld bytes apart
template <bool F32>
__device__ __forceinline__ void flush_tile(const Epi& e, char* to, int64_t ld, int rows, int n, int align) {
    __syncwarp();
    if (align == 16 && n == (F32 ? 16 : 32)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 8 * i + (e.lane >> 2);
            const uint4 v = lds128(tile_at(e.tile, row, e.lane & 3));
            if (row < rows) *reinterpret_cast<uint4*>(to + row * ld + 16 * (e.lane & 3)) = v;
        }
    } else if (F32 || align >= 4) {
        const int w = e.lane & 15, have = F32 ? n - w : n - 2 * w;
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
            const int row = 2 * i + (e.lane >> 4);
            const uint32_t v = lds32(tile_at(e.tile, row, w >> 2) + 4 * (w & 3));
            char* const at = to + row * ld + 4 * w;
            if (row >= rows || have <= 0) continue;
            if (F32 || have >= 2) *reinterpret_cast<uint32_t*>(at) = v;
            else *reinterpret_cast<uint16_t*>(at) = (uint16_t)v;
        }
    } else {
#pragma unroll 4
        for (int row = 0; row < 32; ++row) {
            const uint16_t v = lds16(tile_at(e.tile, row, e.lane >> 3) + 2 * (e.lane & 7));
            if (row < rows && e.lane < n) *reinterpret_cast<uint16_t*>(to + row * ld + 2 * e.lane) = v;
        }
    }
    __syncwarp();
}
// global -> shared, zeros where there is nothing
template <bool F32>
__device__ __forceinline__ void fetch_tile(const Epi& e, const char* from, int64_t ld, int rows, int n, int align) {
    __syncwarp();
    if (align == 16 && n == (F32 ? 16 : 32)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 8 * i + (e.lane >> 2);
            uint4 v = make_uint4(0, 0, 0, 0);
            if (row < rows) v = *reinterpret_cast<const uint4*>(from + row * ld + 16 * (e.lane & 3));
            sts128(tile_at(e.tile, row, e.lane & 3), v.x, v.y, v.z, v.w);
        }
    } else if (F32 || align >= 4) {
        const int w = e.lane & 15, have = F32 ? n - w : n - 2 * w;
#pragma unroll 8
        for (int i = 0; i < 16; ++i) {
            const int row = 2 * i + (e.lane >> 4);
            const char* const at = from + row * ld + 4 * w;
            uint32_t v = 0;
            if (row < rows && have > 0) v = F32 || have >= 2 ? *reinterpret_cast<const uint32_t*>(at) : *reinterpret_cast<const uint16_t*>(at);
            sts32(tile_at(e.tile, row, w >> 2) + 4 * (w & 3), v);
        }
    } else {
#pragma unroll 8
        for (int row = 0; row < 32; ++row) {
            uint16_t v = 0;
            if (row < rows && e.lane < n) v = *reinterpret_cast<const uint16_t*>(from + row * ld + 2 * e.lane);
            sts16(tile_at(e.tile, row, e.lane >> 3) + 2 * (e.lane & 7), v);
        }
    }
    __syncwarp();
}

// The warp's 32 x 32 values v to t at (row, col), rounded once to t's type; rows, n: how many of them are there.  All lanes take part.
__device__ __forceinline__ void store_tile(const Epi& e, const Rows& t, int64_t row, int64_t col, int rows, int n, const float (&v)[32]) {
    if (rows <= 0 || n <= 0) return;
    char* const to = t.at(row, col);
    if (t.f32) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (n <= 16 * h) break;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int j = 16 * h + 4 * q;
                sts128(tile_at(e.tile, e.lane, q), __float_as_uint(v[j]), __float_as_uint(v[j + 1]), __float_as_uint(v[j + 2]), __float_as_uint(v[j + 3]));
            }
            flush_tile<true>(e, to + 64 * h, t.ld, rows, min(16, n - 16 * h), t.align);
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            sts128(tile_at(e.tile, e.lane, q), bf16x2(v[8 * q], v[8 * q + 1]), bf16x2(v[8 * q + 2], v[8 * q + 3]), bf16x2(v[8 * q + 4], v[8 * q + 5]),
                   bf16x2(v[8 * q + 6], v[8 * q + 7]));
        flush_tile<false>(e, to, t.ld, rows, n, t.align);
    }
}
__device__ __forceinline__ void load_tile(const Epi& e, const Rows& t, int64_t row, int64_t col, int rows, int n, float (&v)[32]) {
    const char* const from = t.at(row, col);
    if (t.f32) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            fetch_tile<true>(e, from + 64 * h, t.ld, rows, max(0, min(16, n - 16 * h)), t.align);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint4 x = lds128(tile_at(e.tile, e.lane, q));
                const int j = 16 * h + 4 * q;
                v[j] = __uint_as_float(x.x); v[j + 1] = __uint_as_float(x.y); v[j + 2] = __uint_as_float(x.z); v[j + 3] = __uint_as_float(x.w);
            }
        }
    } else {
        fetch_tile<false>(e, from, t.ld, rows, n, t.align);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint4 x = lds128(tile_at(e.tile, e.lane, q));
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[8 * q + 2 * i] = __uint_as_float(w[i] << 16);
                v[8 * q + 2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        }
    }
    __syncwarp();
}

// The gradient of a product enters the tensor core as bf16.  Gradients of 16 bits take its nearest value: off by 2^-8 of it at most, half a step
// of the results' own type, in every term of their sums.  Gradients of 32 bits take three parts, each the nearest value of
// what the ones before leave: 24 bits, all that the 32-bit value has (unless its last part falls below 2^-133).
constexpr int kPartsF32 = 3;
// d: bf16 parts of part_rows rows each, pitch a multiple of 64 columns (what lies beyond the last column is never read)
__device__ __forceinline__ void store_parts(const Epi& e, const Rows& d, int64_t part_rows, int64_t row, int64_t col, int rows, int parts, float (&v)[32]) {
    store_tile(e, d, row, col, rows, 32, v);
#pragma unroll 1
    for (int i = 1; i < parts; ++i) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] -= __bfloat162float(__float2bfloat16_rn(v[j]));
        store_tile(e, d, i * part_rows + row, col, rows, 32, v);
    }
}

// Whether the products of formats with m_a and m_w magnitude bits may be summed in one chain of that many K steps: as long as 24 bits hold the sum of
// products of one size, or the chain is short; else they are taken kBackSpan steps at a time.  Largest relative error of 32-bit results whose terms have
// one sign, in one chain, in spans, and of plain fp32 sums: MX9 x MX9 of 4096 K 3.1e-6, 4.6e-7, 3.1e-6, of 8192 8.8e-6, 3.7e-7, 5.9e-6, of 16384 2.8e-5,
// 3.7e-7, 1e-5; with a hundredth of the channels, the first, 64 times as large as the others 7.2e-6, 3e-6, 5.5e-6; 2.2e-5, 2.9e-6, 8.8e-6; 7e-5, 4.5e-6,
// 1.3e-5.  MX9 x MX6 of 8192 K in one chain 2.2e-7 (plain 2.8e-7), with the large channels 1.6e-6 (1.4e-6); MX6 x MX6 is exact there.  Spans cost 1 %
// (4096 x 32000 x 4096 693 -> 699 us, 4096 x 4096 x 4096 gated 189 -> 190), 16 steps 3 %.
constexpr int kBackSpan = 32;
inline bool one_chain(int m_a, int m_w, int64_t steps) { return steps <= kBackSpan || steps * kBK << (m_a + m_w) <= 1ll << 24; }

// How a product of tiles_m x cols is shared out: the accumulator's columns (cols_div of them for each of the product's) and the items that a
// tile's K steps are cut into.  Measured, a step takes about 650, 527, 370 and 340 clocks at 256, 192, 128 and 64 columns when all clusters are at it (the SMs'
// intake of 50 bytes a clock; 300 with 64 or 128 columns and few clusters: barriers and issue), an item's start and epilogue 1500 at 256: narrower tiles pay
// where they save a round or fill idle clusters (256, 192, 128, 64 columns: 256 x 7000 x 1024 13.1, 12.0, 13.2, 16.4 us; 1003 x 2747 x 1500 24.2, 21.2, 22.2,
// 30.7; 600 x 1500 x 3000 22.7, 19.0, 16.1, 23.7; 2048 x 2304 x 1024 18.7, 19.2, 20.6, 32.3).  A cut pays where few tiles have long sums: it costs the way through
// memory and back, and the last warp's reading of all parts (64 columns, 300 x 300 x 8192 26.1 us, in three 17.2; 256 x 256 x 3584 13.7, 11.8; 256 x 256 x 1280
// 8.0, 10.1).
constexpr int kClusters = 74;  // (the workspaces' sizes follow from it, without a GPU)
struct Share {
    int bn, tiles_n, splits, span;
    int64_t items(int64_t tiles_m) const { return tiles_m * tiles_n * splits; }
    int64_t partial_bytes(int64_t tiles_m) const { return splits > 1 ? items(tiles_m) * 256 * bn * 4 : 0; }
    int64_t counters(int64_t tiles_m) const { return splits > 1 ? tiles_m * tiles_n * 16 : 0; }
};
inline Share share_product(int64_t tiles_m, int64_t cols, int cols_div, int64_t steps, bool whole = false) {
    Share best = {};
    if (tiles_m == 0 || cols == 0 || steps == 0) return {256, 0, 1, 0};  // no items
    double least = 0;
    for (int bn = 256; bn >= (whole ? 256 : 64); bn -= 64) {
        const int64_t n = bn / cols_div, tiles_n = (cols + n - 1) / n, tiles = tiles_m * tiles_n;
        const int64_t most = whole || tiles > kClusters / 2 ? 1 : std::min<int64_t>(16, kClusters / tiles);
        for (int64_t want = 1; want <= most; ++want) {
            const int64_t span = (steps + want - 1) / want, splits = (steps + span - 1) / span;
            if (splits != want) continue;
            const double rounds = (double)((tiles * splits + kClusters - 1) / kClusters);
            const double t = rounds * (span * (bn == 256 ? 650.0 : (bn == 192 ? 527.0 : (bn == 128 ? 370.0 : 340.0))) + 1500.0 * bn / 256) + (splits < 2 ? 0.0 : (bn == 256 ? 7000.0 + 2200.0 * splits : 3500.0 + 1600.0 * splits));
            if (!best.bn || t < 0.97 * least) {
                best = {bn, (int)tiles_n, (int)splits, (int)span};
                least = t;
            }
        }
    }
    return best;
}

}  // namespace fused
}  // namespace bdr
