// The two gradient products of a layer whose operands are packed along K: with D = dLoss / d(A W^T) in bf16,
//     dA[M, K] = D W        (sum over the layer's outputs)       dW[N, K] = D^T A     (sum over tokens)
// Both reduce over a dimension along which their operands are not contiguous in memory: W and A are decoded once, row by row,
// and D^T is D.  Nothing is transposed for it: the tensor core reads an operand with its rows contiguous just as well (descriptors of
// rows-contiguous chunks, see mx_fused_gemm.cuh), so TMA fetches boxes of 64 columns x 64 K from the matrices as they lie.
// Both products run in one launch: their tiles share the clusters, and a last round that is half empty is paid for once.
//
// Measured, bf16: 4096 x 16384 outputs x 2048 159 us = 1726 TFLOP/s, the tensor pipe busy for 86 % of it; 4096 x 32000 x 4096 1412 us = 1520 TFLOP/s; in a long run the power
// limit, 1333 TFLOP/s.  Three parts for 32-bit results take 2.8 times as long.
#include <algorithm>

#include "bdr_async.cuh"
#include "bdr_x2.cuh"
#include "mx_fused_gemm.cuh"
#include "mx_frag.cuh"

namespace bdr {
namespace {

using fused::kRows;
using fused::Rows;

// Where the sums of one of the products go: to the result itself, or, of a part of the K steps, to fp32 sums of the workspace.
struct Target {
    Rows out;        // the result (or the running sum of several calls)
    Rows sums;       // [splits * rows of all segments][K]; NULL: not split
    const float* read;  // running sum of earlier calls to add, or NULL
    int64_t ld_read;
    int rows;        // of a segment
    int splits, span;   // K steps of a part
    int steps;
    int scaled;      // `out` is the result, which takes the factor
    const int64_t* targets;  // NULL, or the rows of the result that do not count are zeros
    int64_t vocab;
    __device__ __forceinline__ bool nothing(int64_t row) const { return targets && !row_counts(targets[row], vocab); }
};

template <bool F32>
struct GradJob {
    struct Params {
        CUtensorMap d_k;   // D, boxes of 64 (K) x 128 rows: A operand of dA
        CUtensorMap d_mn;  // D, boxes of 64 (rows of dW) x 64 (K)
        CUtensorMap w, a;  // boxes of 64 columns x 64 K
        Target da, dw;
        int n_items, n_long, extra, bn, dw_first, items_da_split, items_dw_split, items_dw_seg;
        int tiles_m, tiles_n, tiles_k;
        int steps_n, steps_m;  // K steps over one segment's columns of D, over tokens
        int segs, parts;
        const float* scale;
        int cols;              // K
        const int* gate;
        int* status;
    };
    struct Item {
        int steps, tm, tk, seg;  // seg < 0: dA
        int split, k0;           // first K step
    };
    static constexpr bool b_mn = true;
    static constexpr bool kCut = false, kBack = false;
    static __device__ __forceinline__ void prefetch(const Params& p) { prefetch_map(&p.d_k); prefetch_map(&p.d_mn); prefetch_map(&p.w); prefetch_map(&p.a); }
    static constexpr int kSpan = F32 ? 4 : 0;  // 16 instructions in a chain (32: 4 % faster; 2.6e-7 of a result lost, 5e-7 with 32)
    static __device__ __forceinline__ bool a_mn(const Item& it) { return it.seg >= 0; }
    static __device__ __forceinline__ Item item(const Params& p, int i) {
        Item it;
        const bool first = i < p.n_long;  // the longer items come first
        if (!first) i -= p.n_long;
        if (first != (bool)p.dw_first) {
            it.split = i / p.items_da_split;
            it.seg = -1;
            gemm_tile_coords(i - it.split * p.items_da_split, p.tiles_m, p.tiles_k, 8, it.tm, it.tk);
        } else {
            it.split = i / p.items_dw_split;
            i -= it.split * p.items_dw_split;
            it.seg = i / p.items_dw_seg;
            gemm_tile_coords(i - it.seg * p.items_dw_seg, p.tiles_n, p.tiles_k, 8, it.tm, it.tk);
        }
        const Target& t = it.seg < 0 ? p.da : p.dw;
        it.k0 = it.split * t.span;
        it.steps = min(t.span, t.steps - it.k0);
        return it;
    }
    static __device__ __forceinline__ void load(const Params& p, const Item& it, int kk, int rank, uint8_t* dst, uint64_t* bar) {
        const int row = (it.tm * 2 + rank) * kRows, col = it.tk * p.bn + rank * (p.bn >> 1);
        const bool wide = p.bn == 256;  // else half of the columns: one box of 64 of them
        kk += it.k0;
        uint8_t* const b = dst + fused::kOperandBytes;
        constexpr int kChunk = fused::kOperandBytes / 2;
        if (it.seg < 0) {
            const int i = kk / p.steps_n, k = (kk - i * p.steps_n) * kBK;
            const int z = p.segs * p.parts - 1 - i, seg = z % p.segs;  // z = part * segs + segment; the smallest part first
            tma_load_3d(dst, &p.d_k, k, row, z, bar);
            tma_load_3d(b, &p.w, col, k, seg, bar);
            if (wide) tma_load_3d(b + kChunk, &p.w, col + 64, k, seg, bar);
        } else {
            const int i = kk / p.steps_m, k = (kk - i * p.steps_m) * kBK, z = (p.parts - 1 - i) * p.segs + it.seg;
            tma_load_3d(dst, &p.d_mn, row, k, z, bar);
            tma_load_3d(dst + kChunk, &p.d_mn, row + 64, k, z, bar);
            tma_load_3d(b, &p.a, col, k, 0, bar);
            if (wide) tma_load_3d(b + kChunk, &p.a, col + 64, k, 0, bar);
        }
    }
    // a warp's 32 x 32 sums, from column c of the accumulator
    static __device__ __forceinline__ void put(const Params& p, const Item& it, const fused::Epi& e, int c, float (&v)[32]) {
        const Target& t = it.seg < 0 ? p.da : p.dw;
        const int64_t row = (int64_t)it.tm * 256 + e.r0;
        const int col = it.tk * p.bn + c, rows = (int)min((int64_t)32, t.rows - row), n = min(32, p.cols - col);
        if (rows <= 0 || n <= 0) return;
        const int64_t segs = it.seg < 0 ? 1 : p.segs, out_row = row + (it.seg > 0 ? (int64_t)it.seg * t.rows : 0);
        if (t.sums.p) {
            fused::store_tile(e, t.sums, it.split * segs * t.rows + out_row, col, rows, n, v);
            return;
        }
        if (t.read) {
            float old[32];
            const Rows from = {const_cast<float*>(t.read), t.ld_read, 1, 16};
            fused::load_tile(e, from, out_row, col, rows, n, old);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += old[j];
        }
        if (t.scaled && p.scale) {
            const float s = *p.scale;
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] *= s;
        }
        if (e.lane < rows && t.nothing(out_row + e.lane)) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0.f;
        }
        fused::store_tile(e, t.out, out_row, col, rows, n, v);
    }
    static __device__ __forceinline__ void epilogue(const Params& p, const Item& it, const fused::Epi& e) {
#pragma unroll 1
        for (int c = e.half * (p.bn >> 1); c < (e.half + 1) * (p.bn >> 1); c += 32) {
            __syncwarp();
            uint32_t u[32];
            tmem_ld32(e.tmem + (uint32_t)c, u);
            float v[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(u[j]);
            put(p, it, e, c, v);
        }
    }
    static __device__ __forceinline__ void finish(const Params& p, const Item& it, const fused::Epi& e, float (&v)[4][32]) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (64 * q < p.bn) put(p, it, e, e.half * (p.bn >> 1) + 32 * q, v[q]);
    }
};

// Adds the parts of a split product in order, and what earlier calls left, and writes the result: four columns per thread.  blockIdx.z: dA, dW
__global__ void __launch_bounds__(128) grad_join_kernel(Target da, Target dw, int64_t rows_da, int64_t rows_dw, int cols, const float* scale) {
    asm volatile("griddepcontrol.wait;" ::: "memory");  // launched as a programmatic dependent of the products
    const Target& t = blockIdx.z ? dw : da;
    const int64_t rows = blockIdx.z ? rows_dw : rows_da;
    const int col = ((int)blockIdx.x * 128 + (int)threadIdx.x) * 4, n = min(4, cols - col);
    if (!t.sums.p || n <= 0) return;
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);  // (the pitch of the sums has room for whole groups)
        for (int s = 0; s < t.splits; ++s) {
            const float4 x = *reinterpret_cast<const float4*>(t.sums.at(s * rows + row, col));
            v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
        }
        if (t.read) {
            const float4 x = *reinterpret_cast<const float4*>(reinterpret_cast<const char*>(t.read) + row * t.ld_read + col * 4);
            v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
        }
        if (t.scaled && scale) {
            const float s = *scale;
            v.x *= s; v.y *= s; v.z *= s; v.w *= s;
        }
        if (t.nothing(row)) v = make_float4(0.f, 0.f, 0.f, 0.f);
        const float w[4] = {v.x, v.y, v.z, v.w};
        char* const to = t.out.at(row, col);
        if (t.out.f32) {
            if (t.out.align == 16 && n == 4) *reinterpret_cast<float4*>(to) = v;
            else
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < n) reinterpret_cast<float*>(to)[j] = w[j];
        } else {
            if (t.out.align == 16 && n == 4) *reinterpret_cast<uint2*>(to) = make_uint2(fused::bf16x2(v.x, v.y), fused::bf16x2(v.z, v.w));
            else
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < n) reinterpret_cast<__nv_bfloat16*>(to)[j] = __float2bfloat16_rn(w[j]);
        }
    }
}

// One thread decodes 32 elements of a line (two blocks) straight from the planes and writes 64 bytes.  Bound by memory: 15547 lines of 3417 MX6 27 us = 5.4 TB/s.
// targets: NULL, or blocks out of the ordinary (all those without values among them) of rows that do not count are zeros.
template <int W>
__device__ __forceinline__ void decode_items(const bdr_planes_t& in, __nv_bfloat16* out, int64_t pitch, int64_t n_items, uint32_t items_per_row, int nb,
                                             int64_t first, int64_t stride, const int64_t* targets, int64_t vocab) {
    for (int64_t g = first; g < n_items; g += stride) {
        const int64_t row = (uint64_t)n_items >> 32 ? g / items_per_row : (uint32_t)g / items_per_row;
        const uint32_t it = (uint32_t)(g - row * items_per_row);
        const int64_t at = (int64_t)it * 4 * W;
        const uint8_t* codes = in.elems + row * in.ld_elems + at;
        uint32_t s[W], yw[16];
        if constexpr (W == 8) {
            const uint4 a = __ldg(reinterpret_cast<const uint4*>(codes));
            uint4 b = make_uint4(0, 0, 0, 0);
            if (2 * (int)it + 1 < nb) b = __ldg(reinterpret_cast<const uint4*>(codes) + 1);  // the line may end with the first block
            s[0] = a.x; s[1] = a.y; s[2] = a.z; s[3] = a.w;
            s[4] = b.x; s[5] = b.y; s[6] = b.z; s[7] = b.w;
        } else {
#pragma unroll
            for (int k = 0; k < W; ++k) s[k] = at + 4 * k < in.ld_elems ? __ldg(reinterpret_cast<const uint32_t*>(codes) + k) : 0u;
        }
        // (pitches are multiples of 16 bytes: the second of the two scale bytes is in the line's pitch even where there is no such block)
        const uint32_t Fw = __ldg(reinterpret_cast<const uint16_t*>(in.exps + row * in.ld_exps) + it);
        const uint32_t mw = __ldg(reinterpret_cast<const uint16_t*>(in.micro + row * in.ld_micro) + it);
        // (a block that is not there takes the other's exponent: whatever its padding holds must not send the warp the slow way)
        const uint32_t F0 = Fw & 0xFFu, F1 = 2 * (int)it + 1 < nb ? Fw >> 8 : F0;
        if ((F0 - x2::kMinF <= (uint32_t)(x2::kMaxDecodeF - x2::kMinF)) && (F1 - x2::kMinF <= (uint32_t)(x2::kMaxDecodeF - x2::kMinF))) {
            x2::decode_two_blocks_row<W>(s, F0, F1, mw, yw);
        } else if (targets && !row_counts(targets[row], vocab)) {
#pragma unroll
            for (int k = 0; k < 16; ++k) yw[k] = 0u;
        } else {
            x2::TwoBlocks<W> in2;
#pragma unroll
            for (int k = 0; k < W; ++k) in2.s[k] = s[k];
            const x2::TwoBlocksOut o = x2::decode_two_blocks_slow<W>(in2, F0, F1, mw);
#pragma unroll
            for (int k = 0; k < 16; ++k) yw[k] = o.y[k];
        }
        __nv_bfloat16* const to = out + row * pitch + (int64_t)it * 32;
        async::stg256(to, yw);
        async::stg256(to + 16, yw + 8);
    }
}

struct Lines {
    bdr_planes_t in;
    __nv_bfloat16* out;
    int64_t n_items;
    int m;
};
__device__ __forceinline__ void largest_of(const Largest& l) {  // a block of 256
    __shared__ float shared[8];
    constexpr int kAtOnce = 16;  // rows in flight per thread
    float m = 0.f;
    for (int64_t i0 = threadIdx.x; i0 < l.M; i0 += 256 * kAtOnce) {
        int64_t t[kAtOnce];
        float d[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int64_t i = i0 + 256 * j;
            t[j] = i < l.M ? l.targets[i] : -1;
            d[j] = i < l.M ? l.dloss[i] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            if (row_counts(t[j], l.V)) m = fmaxf(m, fabsf(d[j]));
    }
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) m = fmaxf(m, shared[i]);
        *l.out = m > 0.f && m < INFINITY ? m : 1.f;
    }
}
// Both operands in one launch: blocks 0 .. first_blocks - 1 take the first.
__global__ void __launch_bounds__(256) decode_pair_kernel(Lines first, Lines second, unsigned first_blocks, int64_t pitch, uint32_t items_per_row, int nb,
                                                           const int* gate, int* zero, int n_zero, int beside, Largest largest) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the product's set-up may begin
    if (gate && *gate == 0) return;
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < n_zero; i += 256) zero[i] = 0;
    const unsigned blocks = gridDim.x - (largest.out ? 1u : 0u);
    if (blockIdx.x == blocks) {
        largest_of(largest);
        return;
    }
    const bool one = blockIdx.x < first_blocks;
    const Lines& l = one ? first : second;
    const int64_t at = (int64_t)(one ? blockIdx.x : blockIdx.x - first_blocks) * 256 + threadIdx.x, stride = (int64_t)(one ? first_blocks : blocks - first_blocks) * 256;
    const int64_t* const targets = one && largest.out ? largest.targets : nullptr;
    switch (l.m) {
        case 2: decode_items<3>(l.in, l.out, pitch, l.n_items, items_per_row, nb, at, stride, targets, largest.V); break;
        case 4: decode_items<5>(l.in, l.out, pitch, l.n_items, items_per_row, nb, at, stride, targets, largest.V); break;
        default: decode_items<8>(l.in, l.out, pitch, l.n_items, items_per_row, nb, at, stride, targets, largest.V); break;
    }
    if (beside) asm volatile("griddepcontrol.wait;" ::: "memory");  // not before the product in front: whoever waits for this kernel has both
}

}  // namespace

int decode_pair(const bdr_planes_t& a, int m_a, int64_t rows_a, __nv_bfloat16* out_a, const bdr_planes_t& w, int m_w, int64_t rows_w, __nv_bfloat16* out_w,
                int64_t K, int64_t pitch, cudaStream_t st, const int* gate, int* zero, int64_t n_zero, bool beside,
                const Largest* largest) {
    Lines l[2] = {{a, out_a, rows_a, m_a}, {w, out_w, rows_w, m_w}};
    const int64_t per_row = (K + 31) / 32;
    for (Lines& x : l) {
        const bool rows_count = &x == l && largest;  // (the other kernel knows no rows)
        if (!gate && !beside && !rows_count && x.n_items * K >= (1ll << 23)) {
            QParams qp;
            qp.k1 = 16; qp.k2 = 2; qp.d2 = 1; qp.m = x.m; qp.rounding = BDR_ROUND_NEAREST_EVEN; qp.beta = 1; qp.qmax = (1u << x.m) - 1u;
            const int rc = unpack_rowwise_mx_x2(x.in, x.out, x.n_items, K, pitch, qp, st);  // whole runs of 2048 elements: through shared memory
            if (rc == BDR_OK) x.n_items = 0;
            else if (rc != BDR_ERR_UNSUPPORTED) return rc;
        }
        x.n_items *= per_row;
    }
    if (l[0].n_items + l[1].n_items == 0 && !largest) return n_zero == 0 || cudaMemsetAsync(zero, 0, n_zero * 4, st) == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
    // Behind a gate there rarely is anything to do.  Beside a product one block fits on an SM, and stays until it ends: all of the work is theirs.
    const int64_t most = (int64_t)sm_count() * (beside ? 1 : (gate ? 4 : 32));
    unsigned blocks[2];
    for (int i = 0; i < 2; ++i) blocks[i] = (unsigned)std::min<int64_t>((l[i].n_items + 255) / 256, i == 1 && beside ? most - blocks[0] : most);
    const dim3 grid(blocks[0] + blocks[1] + (largest ? 1 : 0));
    const Largest none = {};
    if (beside)
        return launch_dependent(decode_pair_kernel, grid, dim3(256), st, l[0], l[1], blocks[0], pitch, (uint32_t)per_row, (int)((K + 15) / 16), gate, zero, (int)n_zero, 1, none);
    decode_pair_kernel<<<grid, 256, 0, st>>>(l[0], l[1], blocks[0], pitch, (uint32_t)per_row, (int)((K + 15) / 16), gate, zero, (int)n_zero, 0,
                                           largest ? *largest : none);
    return cudaGetLastError() == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

// How the tiles of the two products are shared out: the accumulator's columns, and into how many parts the K steps of each product's tiles are cut.
// Few tiles with long sums (dA of few tokens, dW of a narrow layer) would keep few clusters busy: their steps go to several clusters, whose fp32
// sums another kernel adds in order.  The shares are those that let the last cluster finish first, with what was measured (in 10 ns): a step
// 40 with 256 columns and 33 with 128, the loads (rows that are not there cost none: 34 and 20 up to 128 tokens); an item's epilogue 270, 32-bit results 540, with
// 256 columns, and half of that with 128, 400 for 32-bit results of many tokens; the joining kernel 350.  (With 34 and 20 for any tokens too many products took
// 128 columns: 5888 x 5120 x 512 fp32 245 us, now 193; 1839 x 1605 x 311 fp32 58, 45.  With 40 and 33 for few, 3 x 14809 x 259 30.6 -> 34.4 us.)
// (Always as for both products: a gradient does not depend on whether the other is wanted.)
constexpr int kPlanClusters = 74, kMostCuts = 32;
struct GradPlan {
    int bn = 256, tiles_k = 0, da = 0, dw = 0;       // tiles of each product
    int cut_da = 1, cut_dw = 1, span_da = 0, span_dw = 0;
    bool dw_first = false;
    int n_da() const { return da * cut_da; }
    int n_dw() const { return dw * cut_dw; }
    int extra = 0;                                   // see fused::Deal
};
static int64_t makespan(int n1, int64_t t1, int n2, int64_t t2, int64_t extra) {  // of n1 long items and n2 others, dealt out as Deal does
    const int C = std::min(kPlanClusters, n1 + n2), q = n1 / C, r = n1 % C;
    const int given = r ? (int)std::min<int64_t>(n2, (C - r) * extra) : 0, rest = n2 - given, full = rest / C, part = rest % C;
    const int64_t reached = r ? (q + 1) * t1 + (full + (part > C - r)) * t2 : 0;
    return std::max(reached, q * t1 + ((given > 0 ? std::min<int64_t>(extra, given) : 0) + full + (part > 0)) * t2);
}
static GradPlan plan_grads(int64_t M, int64_t N, int64_t K, int segs, int parts, bool f32) {
    GradPlan best;
    int64_t least = -1;
    const int64_t tiles_m = (M + 255) / 256, tiles_n = segs * ((N + 255) / 256);
    const int64_t steps_da = (N + kBK - 1) / kBK * segs * parts, steps_dw = (M + kBK - 1) / kBK * parts;
    static const int kCuts[] = {1, 2, 3, 4, 6, 10, 16, kMostCuts};  // (of sums of 24 steps at least)
    for (int bn = 256; bn >= 128; bn /= 2) {
        const int64_t tiles_k = (K + bn - 1) / bn, da = tiles_m * tiles_k, dw = tiles_n * tiles_k;
        const bool few = M <= 128;
        const int64_t step = bn == 256 ? (few ? 34 : 40) : (few ? 20 : 33), epilogue = f32 && !few && bn == 128 ? 400 : (f32 ? 540 : 270) * bn / 256;
        for (int i : kCuts) {
            if (i > 1 && (da * i > kPlanClusters || steps_da < 24)) break;
            const int64_t span_da = (steps_da + i - 1) / i, n_da = da * ((steps_da + span_da - 1) / span_da);
            for (int j : kCuts) {
                if (j > 1 && (dw * j > kPlanClusters || steps_dw < 24)) break;
                const int64_t span_dw = (steps_dw + j - 1) / j, n_dw = dw * ((steps_dw + span_dw - 1) / span_dw);
                const int64_t t_da = span_da * step + epilogue, t_dw = span_dw * step + epilogue;
                const bool dw_first = t_dw > t_da;
                const int64_t extra = std::max(t_da, t_dw) / std::min(t_da, t_dw);
                const int64_t t = (dw_first ? makespan(n_dw, t_dw, n_da, t_da, extra) : makespan(n_da, t_da, n_dw, t_dw, extra)) + (i > 1 || j > 1 ? 350 : 0);
                if (least >= 0 && t * 100 >= least * 98) continue;
                least = t;
                best.bn = bn; best.tiles_k = (int)tiles_k; best.da = (int)da; best.dw = (int)dw;
                best.cut_da = (int)(n_da / da); best.cut_dw = (int)(n_dw / dw);
                best.span_da = (int)span_da; best.span_dw = (int)span_dw;
                best.dw_first = dw_first; best.extra = (int)extra;
            }
        }
    }
    return best;
}
// Bytes of the fp32 sums that launch_grad_products may need for M tokens and any number of outputs up to N: at most 2 x 74 tiles of each product.
int64_t grad_sums_bytes(int64_t M, int64_t N, int64_t K, int segs) {
    const int64_t most = 2 * kPlanClusters * 256 / ((K + 255) / 256) + 1;  // (tiles of 128 columns are more, and have as many rows)
    return round_up((std::min(most, kMostCuts * M) + std::min(most, kMostCuts * segs * N)) * line_pitch(K) * 4, 256);
}

template <bool F32>
static int launch_grads(const GradProducts& g, cudaStream_t st) {
    typename GradJob<F32>::Params p = {};
    const int64_t z = (int64_t)g.segs * g.parts;
    if (!fused::make_map(&p.d_k, g.d, g.N, g.M, z, g.pitch_d, g.M * g.pitch_d, kRows) ||
        !fused::make_map(&p.d_mn, g.d, g.N, g.M, z, g.pitch_d, g.M * g.pitch_d, kBK) ||
        !fused::make_map(&p.w, g.w, g.K, g.N, g.segs, g.pitch_k, g.N * g.pitch_k, kBK) ||
        !fused::make_map(&p.a, g.a, g.K, g.M, 1, g.pitch_k, g.M * g.pitch_k, kBK))
        return BDR_ERR_CUDA;
    GradPlan plan = plan_grads(g.M, g.N, g.K, g.segs, g.parts, F32);
    if (!g.da) { plan.da = 0; plan.cut_da = 1; }
    if (!g.dw) { plan.dw = 0; plan.cut_dw = 1; }
    p.tiles_m = (int)((g.M + 255) / 256);
    p.tiles_n = (int)((g.N + 255) / 256);
    p.tiles_k = plan.tiles_k;
    p.bn = plan.bn;
    p.steps_n = (int)((g.N + kBK - 1) / kBK);
    p.steps_m = (int)((g.M + kBK - 1) / kBK);
    p.segs = g.segs; p.parts = g.parts; p.scale = g.scale;
    p.cols = (int)g.K;
    p.items_da_split = plan.da;
    p.items_dw_seg = p.tiles_n * p.tiles_k;
    p.items_dw_split = plan.dw;
    p.da.rows = (int)g.M;
    p.dw.rows = (int)g.N;
    p.da.steps = p.steps_n * g.segs * g.parts;
    p.dw.steps = p.steps_m * g.parts;
    float* sums = g.sums;
    const int64_t pitch = line_pitch(g.K);
    for (int i = 0; i < 2; ++i) {
        Target& t = i ? p.dw : p.da;
        const int64_t rows = i ? g.segs * g.N : g.M;
        t.out = i ? fused::make_rows(g.dw, g.ld_dw, F32) : (g.last ? fused::make_rows(g.da, g.ld_da, F32) : fused::make_rows(g.acc, g.ld_acc, true));
        t.scaled = i || g.last;
        t.targets = !i && g.last ? g.targets : nullptr;
        t.vocab = g.vocab;
        t.read = i || g.first ? nullptr : g.acc;
        t.ld_read = g.ld_acc * 4;
        t.splits = i ? plan.cut_dw : plan.cut_da;
        t.span = i ? plan.span_dw : plan.span_da;
        if (t.splits > 1) {
            t.sums = fused::make_rows(sums, pitch, true);
            sums += t.splits * rows * pitch;
        }
    }
    p.n_items = plan.n_da() + plan.n_dw();
    p.dw_first = plan.dw_first;
    p.n_long = plan.dw_first ? plan.n_dw() : plan.n_da();
    p.extra = plan.extra;
    p.status = device_status_word();
    if (!p.status) return BDR_ERR_CUDA;
    if (p.n_items == 0) return BDR_OK;
    const int rc = fused::launch<GradJob<F32>>(p, st);
    if (rc || (p.da.splits == 1 && p.dw.splits == 1)) return rc;
    const int64_t rows_da = g.M, rows_dw = g.segs * g.N;
    const dim3 grid((unsigned)((g.K + 511) / 512), (unsigned)std::min<int64_t>(2048, std::max(p.da.splits > 1 ? rows_da : 0, p.dw.splits > 1 ? rows_dw : 0)), 2);
    return launch_dependent(grad_join_kernel, grid, dim3(128), st, p.da, p.dw, rows_da, rows_dw, p.cols, p.scale);
}

int launch_grad_products(const GradProducts& g, cudaStream_t st) { return g.f32 ? launch_grads<true>(g, st) : launch_grads<false>(g, st); }

int check_fused_operands(const bdr_config_t* cfg_a, const bdr_planes_t* a, const bdr_config_t* cfg_w, const bdr_planes_t* w, int64_t K) {
    int rc = check_table2_config(cfg_a);
    if (!rc) rc = check_table2_config(cfg_w);
    if (!rc) rc = check_table2_planes(cfg_a, a, K);
    return rc ? rc : check_table2_planes(cfg_w, w, K);
}

}  // namespace bdr
