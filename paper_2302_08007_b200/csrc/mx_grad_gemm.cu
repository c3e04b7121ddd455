// The two gradient products of a layer whose operands are packed along K: with D = dLoss / d(A W^T) in bf16,
//     dA[M, K] = D W        (sum over the layer's outputs)       dW[N, K] = D^T A     (sum over tokens)
// Both reduce over a dimension along which their operands are not contiguous in memory: W and A are decoded once, row by row,
// and D^T is D.  Nothing is transposed for it: the tensor core reads an operand with its rows contiguous just as well (descriptors of
// rows-contiguous chunks, see mx_fused_gemm.cuh), so TMA fetches boxes of 64 columns x 64 K from the matrices as they lie.
// Both products run in one launch: their tiles share the clusters, and a last round that is half empty is paid for once.
#include "bdr_x2.cuh"
#include "mx_fused_gemm.cuh"
#include "mx_frag.cuh"

namespace bdr {
namespace {

using fused::kRows;

struct Target {
    void* out;
    int64_t ld;
    int rows, vec;   // rows of a segment
    float* read;     // fp32 sums to add to, or NULL
    float* keep;     // fp32 sums to store instead of `out`, or NULL
    int64_t ld_acc;
};

template <bool F32>
struct GradJob {
    struct Params {
        CUtensorMap d_k;   // D, boxes of 64 (K) x 128 rows: A operand of dA
        CUtensorMap d_mn;  // D, boxes of 64 (rows of dW) x 64 (K)
        CUtensorMap w, a;  // boxes of 64 columns x 64 K
        Target da, dw;
        int n_items, items_da, items_dw_seg;
        int tiles_m, tiles_n, tiles_k;
        int steps_n, steps_m;  // K steps over one segment's columns of D, over tokens
        int segs, parts;
        const float* scale;
        int cols;              // K
        int* status;
    };
    struct Item {
        int steps, tm, tk, seg;  // seg < 0: dA
    };
    static constexpr bool b_mn = true;
    static constexpr int kSpan = F32 ? 4 : 0;  // 16 instructions in a chain
    static __device__ __forceinline__ bool a_mn(const Item& it) { return it.seg >= 0; }
    static __device__ __forceinline__ Item item(const Params& p, int i) {
        Item it;
        if (i < p.items_da) {
            it.seg = -1;
            it.steps = p.steps_n * p.segs * p.parts;
            gemm_tile_coords(i, p.tiles_m, p.tiles_k, 8, it.tm, it.tk);
        } else {
            i -= p.items_da;
            it.seg = i / p.items_dw_seg;
            it.steps = p.steps_m * p.parts;
            gemm_tile_coords(i - it.seg * p.items_dw_seg, p.tiles_n, p.tiles_k, 8, it.tm, it.tk);
        }
        return it;
    }
    static __device__ __forceinline__ void load(const Params& p, const Item& it, int kk, int rank, uint8_t* dst, uint64_t* bar) {
        const int row = (it.tm * 2 + rank) * kRows, col = (it.tk * 2 + rank) * kRows;
        uint8_t* const b = dst + fused::kOperandBytes;
        constexpr int kChunk = fused::kOperandBytes / 2;
        if (it.seg < 0) {
            const int i = kk / p.steps_n, k = (kk - i * p.steps_n) * kBK;
            const int z = p.segs * p.parts - 1 - i, seg = z % p.segs;  // z = part * segs + segment; the smallest part first
            tma_load_3d(dst, &p.d_k, k, row, z, bar);
            tma_load_3d(b, &p.w, col, k, seg, bar);
            tma_load_3d(b + kChunk, &p.w, col + 64, k, seg, bar);
        } else {
            const int i = kk / p.steps_m, k = (kk - i * p.steps_m) * kBK, z = (p.parts - 1 - i) * p.segs + it.seg;
            tma_load_3d(dst, &p.d_mn, row, k, z, bar);
            tma_load_3d(dst + kChunk, &p.d_mn, row + 64, k, z, bar);
            tma_load_3d(b, &p.a, col, k, 0, bar);
            tma_load_3d(b + kChunk, &p.a, col + 64, k, 0, bar);
        }
    }
    // 32 sums of a row, from column c of the 256
    static __device__ __forceinline__ void put(const Params& p, const Item& it, int r, int c, float (&v)[32]) {
        const Target& t = it.seg < 0 ? p.da : p.dw;
        const int row = it.tm * 256 + r, col = it.tk * 256 + c, n = min(32, p.cols - col);
        if (row >= t.rows || n <= 0) return;
        const int64_t out_row = row + (it.seg > 0 ? (int64_t)it.seg * t.rows : 0);
        if (t.read) {
            float old[32];
            fused::load_run(t.read + out_row * t.ld_acc, col, old, n, true, true);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += old[j];
        }
        if (t.keep) {
            fused::store_run(t.keep + out_row * t.ld_acc, col, v, n, true, true);
        } else {
            if (p.scale) {
                const float s = *p.scale;
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] *= s;
            }
            fused::store_run(static_cast<char*>(t.out) + out_row * t.ld * (F32 ? 4 : 2), col, v, n, F32, t.vec);
        }
    }
    static __device__ __forceinline__ void epilogue(const Params& p, const Item& it, int r, int half, uint32_t tmem) {
#pragma unroll 1
        for (int c = half * 128; c < half * 128 + 128; c += 32) {
            __syncwarp();
            uint32_t u[32];
            tmem_ld32(tmem + (uint32_t)c, u);
            float v[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(u[j]);
            put(p, it, r, c, v);
        }
    }
    static __device__ __forceinline__ void finish(const Params& p, const Item& it, int r, int half, float (&v)[4][32]) {
#pragma unroll
        for (int q = 0; q < 4; ++q) put(p, it, r, half * 128 + 32 * q, v[q]);
    }
};

// One thread decodes 32 elements of a line (two blocks) straight from the planes and writes 64 bytes.
template <int W>
__global__ void __launch_bounds__(256) decode_lines_kernel(bdr_planes_t in, __nv_bfloat16* out, int64_t pitch, int64_t n_items, uint32_t items_per_row, int nb) {
    const int64_t stride = (int64_t)gridDim.x * 256;
    for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < n_items; g += stride) {
        const int64_t row = g / items_per_row;
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
        const uint32_t F0 = Fw & 0xFFu, F1 = Fw >> 8;
        if ((F0 - x2::kMinF <= (uint32_t)(x2::kMaxDecodeF - x2::kMinF)) && (F1 - x2::kMinF <= (uint32_t)(x2::kMaxDecodeF - x2::kMinF))) {
            x2::decode_two_blocks_row<W>(s, F0, F1, mw, yw);
        } else {
            x2::TwoBlocks<W> in2;
#pragma unroll
            for (int k = 0; k < W; ++k) in2.s[k] = s[k];
            const x2::TwoBlocksOut o = x2::decode_two_blocks_slow<W>(in2, F0, F1, mw);
#pragma unroll
            for (int k = 0; k < 16; ++k) yw[k] = o.y[k];
        }
        uint4* dst = reinterpret_cast<uint4*>(out + row * pitch + (int64_t)it * 32);
#pragma unroll
        for (int k = 0; k < 4; ++k) dst[k] = make_uint4(yw[4 * k], yw[4 * k + 1], yw[4 * k + 2], yw[4 * k + 3]);
    }
}

template <int W>
int launch_decode(const bdr_planes_t& in, int64_t rows, int64_t K, __nv_bfloat16* out, int64_t pitch, cudaStream_t st) {
    const int64_t per_row = (K + 31) / 32, n = rows * per_row;
    if (n == 0) return BDR_OK;
    const unsigned grid = (unsigned)std::min<int64_t>((n + 255) / 256, (int64_t)sm_count() * 32);
    decode_lines_kernel<W><<<grid, 256, 0, st>>>(in, out, pitch, n, (uint32_t)per_row, (int)((K + 15) / 16));
    return cudaGetLastError() == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

}  // namespace

int decode_lines(const bdr_planes_t& in, int m, int64_t rows, int64_t K, __nv_bfloat16* out, int64_t pitch, cudaStream_t st) {
    QParams qp;
    qp.k1 = 16; qp.k2 = 2; qp.d2 = 1; qp.m = m; qp.rounding = BDR_ROUND_NEAREST_EVEN; qp.beta = 1; qp.qmax = (1u << m) - 1u;
    const int rc = unpack_rowwise_mx_x2(in, out, rows, K, pitch, qp, st);  // whole runs of 2048 elements: through shared memory
    if (rc != BDR_ERR_UNSUPPORTED) return rc;
    switch (m) {
        case 2: return launch_decode<3>(in, rows, K, out, pitch, st);
        case 4: return launch_decode<5>(in, rows, K, out, pitch, st);
        case 7: return launch_decode<8>(in, rows, K, out, pitch, st);
    }
    return BDR_ERR_UNSUPPORTED;
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
    const int width = F32 ? 4 : 2;
    p.da = {g.da, g.ld_da, (int)g.M, fused::rows_aligned(g.da, g.ld_da, width), g.first ? nullptr : g.acc, g.last ? nullptr : g.acc, g.ld_acc};
    p.dw = {g.dw, g.ld_dw, (int)g.N, fused::rows_aligned(g.dw, g.ld_dw, width), nullptr, nullptr, 0};
    p.tiles_m = (int)((g.M + 255) / 256);
    p.tiles_n = (int)((g.N + 255) / 256);
    p.tiles_k = (int)((g.K + 255) / 256);
    p.steps_n = (int)((g.N + kBK - 1) / kBK);
    p.steps_m = (int)((g.M + kBK - 1) / kBK);
    p.segs = g.segs; p.parts = g.parts; p.scale = g.scale;
    p.cols = (int)g.K;
    p.items_da = g.da ? p.tiles_m * p.tiles_k : 0;
    p.items_dw_seg = p.tiles_n * p.tiles_k;
    p.n_items = p.items_da + (g.dw ? g.segs * p.items_dw_seg : 0);
    p.status = device_status_word();
    if (!p.status) return BDR_ERR_CUDA;
    if (p.n_items == 0) return BDR_OK;
    return fused::launch<GradJob<F32>>(p, st);
}

int launch_grad_products(const GradProducts& g, cudaStream_t st) { return g.f32 ? launch_grads<true>(g, st) : launch_grads<false>(g, st); }

int check_fused_operands(const bdr_config_t* cfg_a, const bdr_planes_t* a, const bdr_config_t* cfg_w, const bdr_planes_t* w, int64_t K) {
    int rc = check_table2_config(cfg_a);
    if (!rc) rc = check_table2_config(cfg_w);
    if (!rc) rc = check_table2_planes(cfg_a, a, K);
    return rc ? rc : check_table2_planes(cfg_w, w, K);
}

}  // namespace bdr
