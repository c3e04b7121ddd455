// Gated feed-forward layer on packed operands: h[M, N] = act(A Wg^T) * (A Wu^T), and its gradients.
//
// Forward.  The two weights are one packed tensor of 2 N lines (gate first).  Both are decoded to bf16 once (exact: at most seven
// magnitude bits), and one persistent kernel computes both products: a cluster's 256-column accumulator holds 128 columns of the gate
// (which the leader CTA loads) and the same 128 columns of the other projection (its peer's), so that a thread of the epilogue has both values
// of an output in its own tensor-memory lane and writes h without either product passing through memory.  For training they are
// stored on the side, rounded to h's type.
// Backward.  dG = dh * u * act'(g), dU = dh * act(g); dA = dG Wg + dU Wu, dWg = dG^T A, dWu = dU^T A.  With the products stored by the
// forward pass the first step is an elementwise kernel; without them they are computed again, in the same kernel as the forward's, whose
// epilogue then reads dh and writes dG and dU.  The gradient products are those of mx_grad_gemm.cu.
//
// Measured: forward of 4096 tokens, 2048 -> 2 x 4096, MX9, both products kept: 80 us = 1711 TFLOP/s, the tensor pipe busy for 86 % of it (the rest: an SM takes in
// a step's 32 KB in 640 clocks where the products need 512); 8192 tokens, 4096 -> 2 x 8192, MX6 on the 8-bit path 374 us = 2940 TFLOP/s, 411 with the re-encoding.
#include <algorithm>

#include "mx_act.cuh"
#include "mx_frag.cuh"
#include "mx_fused_f8.cuh"
#include "mx_fused_gemm.cuh"

namespace bdr {
namespace {

using fused::kRows;
using fused::Rows;

// GRAD: the epilogue writes dG and dU instead of h
template <bool GRAD>
struct GatedJob {
    struct Params {
        CUtensorMap a, w;          // bf16 [M][K]; [2][N][K]
        int n_items, n_long, extra, bn, tiles_m, tiles_n, band_rows, steps, splits, span;
        float* partials;
        int* counters;
        int M, N, act;
        Rows h;                    // h, or dh
        Rows gate_out, up_out;     // where the two products go (NULL: nowhere)
        Rows d;                    // [parts][2][M][pitch]
        int parts;
        fused::F8 f8;              // 8-bit operands, where they are used
        const int* gate;
        int* status;
    };
    struct Item { int steps, tm, tn, tile, split; };
    static constexpr bool b_mn = false;
    static constexpr int kSpan = 0;
    static constexpr bool kCut = true, kBack = false;
    static __device__ __forceinline__ int rows(const Params& p) { return p.M; }
    // half of the accumulator is the gate, whose pieces of 32 columns the two halves of the warps take in turn
    static __device__ __forceinline__ int chunks(int bn, int half) { return 2 * ((bn / 64 + 1 - half) / 2); }
    static __device__ __forceinline__ int chunk(int bn, int half, int i) {
        const int gates = (bn / 64 + 1 - half) / 2;
        return i < gates ? 32 * (half + 2 * i) : bn / 2 + 32 * (half + 2 * (i - gates));
    }
    static __device__ __forceinline__ void prefetch(const Params& p) { prefetch_map(&p.a); prefetch_map(&p.w); }
    static __device__ __forceinline__ bool a_mn(const Item&) { return false; }
    static __device__ __forceinline__ Item item(const Params& p, int i) {
        Item it;
        const int tiles = p.tiles_m * p.tiles_n;
        it.split = i / tiles;
        it.tile = i - it.split * tiles;
        it.steps = min(p.span, p.steps - it.split * p.span);
        gemm_tile_coords(it.tile, p.tiles_m, p.tiles_n, p.band_rows, it.tm, it.tn);
        return it;
    }
    static __device__ __forceinline__ void load(const Params& p, const Item& it, int kk, int rank, uint8_t* dst, uint64_t* bar) {
        kk += it.split * p.span;
        tma_load_3d(dst, &p.a, kk * kBK, (it.tm * 2 + rank) * kRows, 0, bar);
        tma_load_3d(dst + fused::kOperandBytes, &p.w, kk * kBK, it.tn * (p.bn >> 1), rank, bar);
    }
    static __device__ __forceinline__ void load8(const Params& p, const Item& it, int kk, int rank, uint8_t* dst, uint64_t* bar) {
        tma_load_3d(dst, &p.f8.a, kk * fused::kK8, (it.tm * 2 + rank) * kRows, 0, bar);
        tma_load_3d(dst + kRows * fused::kK8, &p.f8.w, kk * fused::kK8, it.tn * kRows, rank, bar);
        uint8_t* const sf = dst + fused::kTiles8;
        const uint8_t* const w = p.f8.sf_w + ((int64_t)kk * p.f8.row_tiles_w + it.tn) * 512;
        bulk_load_g2s(sf, p.f8.sf_a + ((int64_t)kk * p.f8.row_tiles_a + it.tm * 2 + rank) * 512, 512, bar);
        bulk_load_g2s(sf + 512, w, 512, bar);                                            // of the gate
        bulk_load_g2s(sf + 1024, w + (int64_t)(p.f8.row_tiles_w >> 1) * 512, 512, bar);  // of the other projection
    }
    static __device__ __forceinline__ int column(int half, int q) { return (q & 2) * 64 + half * 64 + (q & 1) * 32; }
    static __device__ __forceinline__ void finish(const Params& p, const Item& it, const fused::Epi& e, float (&v)[4][32]) {
        const int64_t row = (int64_t)it.tm * 256 + e.r0;
        const int rows = (int)min((int64_t)32, p.M - row);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int col = it.tn * kRows + column(e.half, q);
            one_tile(p, e, row, col, rows, min(32, p.N - col), v[q], v[q + 2]);
        }
    }
    // a warp's 32 x 32 outputs, whose products are g and u
    static __device__ __forceinline__ void one_tile(const Params& p, const fused::Epi& e, int64_t row, int col, int rows, int n, float (&g)[32], float (&u)[32]) {
        if (rows <= 0 || n <= 0) return;  // (the same for the whole warp)
        if constexpr (!GRAD) {
            if (p.gate_out.p) {
                fused::store_tile(e, p.gate_out, row, col, rows, n, g);
                fused::store_tile(e, p.up_out, row, col, rows, n, u);
            }
            act::with(p.act, [&](auto f) {
#pragma unroll
                for (int j = 0; j < 32; ++j) g[j] = act::of<decltype(f)::value>(g[j]) * u[j];
            });
            fused::store_tile(e, p.h, row, col, rows, n, g);
        } else {
            float dh[32];
            fused::load_tile(e, p.h, row, col, rows, n, dh);
            act::with(p.act, [&](auto f) {
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    float y, slope;
                    act::both<decltype(f)::value>(g[j], y, slope);
                    g[j] = dh[j] * u[j] * slope;
                    u[j] = dh[j] * y;
                }
            });
            fused::store_parts(e, p.d, 2 * (int64_t)p.M, row, col, rows, p.parts, g);
            fused::store_parts(e, p.d, 2 * (int64_t)p.M, p.M + row, col, rows, p.parts, u);
        }
    }
    static __device__ __forceinline__ void epilogue(const Params& p, const Item& it, const fused::Epi& e) {
        const int64_t row = (int64_t)it.tm * 256 + e.r0;
        const int rows = (int)min((int64_t)32, p.M - row), cols = p.bn >> 1;  // half of the accumulator is the gate
#pragma unroll 1
        for (int c = e.half * 32; c < cols; c += 64) {
            uint32_t gu[2][32];
            __syncwarp();
            tmem_ld32_nowait(e.tmem + (uint32_t)c, gu[0]);
            tmem_ld32_nowait(e.tmem + (uint32_t)(cols + c), gu[1]);
            tmem_ld_wait();
            const int col = it.tn * cols + c, n = min(32, p.N - col);
            float g[32], u[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) { g[j] = __uint_as_float(gu[0][j]); u[j] = __uint_as_float(gu[1][j]); }
            one_tile(p, e, row, col, rows, n, g, u);
        }
    }
};

// for 32-bit results, where one chain of additions would lose bits of them
template <bool GRAD>
struct GatedJobInSpans : GatedJob<GRAD> {
    static constexpr int kSpan = fused::kBackSpan;
    static constexpr bool kBack = true;
};

// dG and dU from the stored products.  A thread keeps its eight columns and walks down the rows, two at a time.  Bound by memory (bf16: 6 bytes in, 4 out
// per output): 8192 x 8192 142 us = 4.7 TB/s.
template <bool F32>
__device__ __forceinline__ void read8(const Rows& t, int64_t row, int col, int n, float (&v)[8]) {
    const char* const from = t.at(row, col);
    if constexpr (F32) {
        if (t.align == 16 && n == 8) {
            const float4 a = *reinterpret_cast<const float4*>(from), b = *reinterpret_cast<const float4*>(from + 16);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < n ? reinterpret_cast<const float*>(from)[j] : 0.f;
        }
    } else {
        if (t.align == 16 && n == 8) {
            const uint4 x = *reinterpret_cast<const uint4*>(from);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(w[e] << 16); v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u); }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < n ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(from)[j]) : 0.f;
        }
    }
}
template <bool F32, int ACT>
__global__ void __launch_bounds__(256) gated_grad_kernel(Rows gate, Rows up, Rows dh, int64_t M, int N, Rows d) {
    const int col = ((int)blockIdx.x * (int)blockDim.x + (int)threadIdx.x) * 8, n = min(8, N - col);
    if (n <= 0) return;
    constexpr int kAhead = F32 ? 1 : 2;  // rows in flight
    for (int64_t row0 = (int64_t)blockIdx.y * kAhead; row0 < M; row0 += (int64_t)gridDim.y * kAhead) {
        float g[kAhead][8], u[kAhead][8], e[kAhead][8];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t row = min(row0 + i, M - 1);
            read8<F32>(gate, row, col, n, g[i]);
            read8<F32>(up, row, col, n, u[i]);
            read8<F32>(dh, row, col, n, e[i]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (row0 + i >= M) break;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float y, slope;
                act::both<ACT>(g[i][j], y, slope);
                g[i][j] = e[i][j] * u[i][j] * slope;
                u[i][j] = e[i][j] * y;
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float(&v)[8] = s ? u[i] : g[i];
#pragma unroll
                for (int part = 0; part < (F32 ? fused::kPartsF32 : 1); ++part) {  // (the pitch has room for whole groups)
                    *reinterpret_cast<uint4*>(d.at((2 * part + s) * M + row0 + i, col)) =
                        make_uint4(fused::bf16x2(v[0], v[1]), fused::bf16x2(v[2], v[3]), fused::bf16x2(v[4], v[5]), fused::bf16x2(v[6], v[7]));
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] -= __bfloat162float(__float2bfloat16_rn(v[j]));
                }
            }
        }
    }
}
template <bool F32>
int launch_gated_grad(const Rows& gate, const Rows& up, const Rows& dh, int act, int64_t M, int64_t N, const Rows& d, cudaStream_t st) {
    const int64_t groups = (N + 7) / 8;
    const int threads = groups >= 256 ? 256 : (int)round_up(groups, 32);
    const int64_t x = (groups + threads - 1) / threads, y = std::min<int64_t>(M, std::max<int64_t>(1, (int64_t)sm_count() * 4096 / (x * threads)));
    const dim3 grid((unsigned)x, (unsigned)std::min<int64_t>(y, 65535));
    switch (act) {
        case MX_ACT_SILU: gated_grad_kernel<F32, MX_ACT_SILU><<<grid, threads, 0, st>>>(gate, up, dh, M, (int)N, d); break;
        case MX_ACT_GELU: gated_grad_kernel<F32, MX_ACT_GELU><<<grid, threads, 0, st>>>(gate, up, dh, M, (int)N, d); break;
        case MX_ACT_GELU_TANH: gated_grad_kernel<F32, MX_ACT_GELU_TANH><<<grid, threads, 0, st>>>(gate, up, dh, M, (int)N, d); break;
        default: gated_grad_kernel<F32, MX_ACT_RELU><<<grid, threads, 0, st>>>(gate, up, dh, M, (int)N, d); break;
    }
    return cudaGetLastError() == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

// Workspace: A, W and, for gradients, D.
struct GatedSpace {
    int64_t pitch_k, pitch_d, a, w, d, sums, f8, flag, partials, counters, n_counters, bytes;  // offsets in bytes
    GatedSpace(int64_t M, int64_t N, int64_t K, int parts) {
        pitch_k = line_pitch(K);
        pitch_d = round_up(N, 64);
        a = 0;
        w = a + round_up(M * pitch_k * 2, 256);
        d = w + round_up(2 * N * pitch_k * 2, 256);
        sums = d + (parts ? round_up((int64_t)parts * 2 * M * pitch_d * 2, 256) : 0);
        f8 = sums + (parts ? grad_sums_bytes(M, N, K, 2) : 0);
        // (whether it will be used depends on the formats too; a forward pass keeps the bytes where the bf16 operands would lie)
        flag = parts ? f8 + (fused::takes_f8(4, 4, M, 2 * N, N, K) ? fused::f8_bytes(M, 2 * N, K) : 0) : std::max(f8, fused::f8_bytes(M, 2 * N, K));
        const int64_t tiles_m = (M + 255) / 256;
        const fused::Share share = fused::share_product(tiles_m, N, 2, (K + kBK - 1) / kBK);
        partials = flag + 256;
        counters = partials + round_up(share.partial_bytes(tiles_m), 256);
        n_counters = share.counters(tiles_m);
        bytes = counters + round_up(n_counters * 4, 256);
    }
};

constexpr int64_t kMost = 1ll << 28;  // of every size: no product of two sizes and a few bytes leaves 64 bits

int check_rows(const void* p, int64_t ld, int64_t cols, int width) {
    if (!p) return BDR_ERR_NULL;
    if (ld < cols) return BDR_ERR_SIZE;
    return (uintptr_t)p % width ? BDR_ERR_MISALIGNED : BDR_OK;
}

template <class Params>
int set_products(Params& p, int64_t M, int64_t N, int64_t K, const GatedSpace& s, uint8_t* ws, bool f8) {
    p.tiles_m = (int)((M + 255) / 256);
    p.steps = (int)((K + kBK - 1) / kBK);
    const fused::Share share = fused::share_product(p.tiles_m, N, 2, p.steps, f8);
    p.bn = share.bn;
    p.tiles_n = share.tiles_n;
    p.splits = share.splits;
    p.span = share.span;
    p.partials = reinterpret_cast<float*>(ws + s.partials);
    p.counters = reinterpret_cast<int*>(ws + s.counters);
    if (!fused::make_map(&p.a, ws + s.a, K, M, 1, s.pitch_k, M * s.pitch_k, kRows) ||
        !fused::make_map(&p.w, ws + s.w, K, N, 2, s.pitch_k, N * s.pitch_k, p.bn / 2))
        return BDR_ERR_CUDA;
    p.n_items = p.n_long = p.tiles_m * p.tiles_n * p.splits;
    p.extra = 0;
    p.band_rows = gemm_band_rows((M + 2 * N) * K * 2);
    p.M = (int)M;
    p.N = (int)N;
    p.status = device_status_word();
    return p.status ? BDR_OK : BDR_ERR_CUDA;
}

}  // namespace
}  // namespace bdr

using namespace bdr;

extern "C" {

int64_t mx_gated_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N < 0 || K < 1 || M > kMost || N > kMost || K > kMost) return 0;
    return GatedSpace(M, N, K, 0).bytes;
}

int mx_gated_gemm(const bdr_config_t* cfg_a, const bdr_planes_t* a, const bdr_config_t* cfg_w, const bdr_planes_t* w, int64_t M, int64_t N,
                  int64_t K, int32_t act, void* h, bdr_dtype_t dt, int64_t ldh, void* gate_up, int64_t ld_gate_up, void* workspace,
                  int64_t workspace_bytes, void* stream) {
    if (dt != BDR_F32 && dt != BDR_BF16) return BDR_ERR_UNSUPPORTED;
    if (!act::known(act)) return BDR_ERR_UNSUPPORTED;
    if (M < 0 || N < 0 || K < 0 || M > kMost || N > kMost || K > kMost) return BDR_ERR_SIZE;
    if (K == 0 || ((M + 255) / 256) * ((N + kRows - 1) / kRows) >= (1ll << 30)) return BDR_ERR_UNSUPPORTED;
    int rc = check_table2_config(cfg_a);
    if (!rc) rc = check_table2_config(cfg_w);
    if (rc || M == 0 || N == 0) return rc;
    if ((rc = check_fused_operands(cfg_a, a, cfg_w, w, K))) return rc;
    const int width = dt == BDR_F32 ? 4 : 2;
    if ((rc = check_rows(h, ldh, N, width))) return rc;
    if (gate_up && (rc = check_rows(gate_up, ld_gate_up, 2 * N, width))) return rc;
    const GatedSpace s(M, N, K, 0);
    if (!workspace || workspace_bytes < s.bytes) return BDR_ERR_WORKSPACE;
    if ((uintptr_t)workspace % 256) return BDR_ERR_MISALIGNED;
    cudaStream_t st = (cudaStream_t)stream;
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    if (few_rows(M, 2 * N, K)) {
        __nv_bfloat16* const x = reinterpret_cast<__nv_bfloat16*>(ws + s.a);
        if ((rc = decode_pair(*a, cfg_a->m, M, x, *w, cfg_w->m, 0, nullptr, K, s.pitch_k, st))) return rc;
        return gated_rows(cfg_w, w, N, K, x, s.pitch_k, M, act, h, dt, ldh, gate_up, ld_gate_up, st);
    }
    GatedJob<false>::Params p = {};
    const bool f8 = fused::takes_f8(cfg_a->m, cfg_w->m, M, 2 * N, N, K);
    p.act = act;
    p.h = fused::make_rows(h, ldh, dt == BDR_F32);
    p.gate_out = fused::make_rows(gate_up, ld_gate_up, dt == BDR_F32);
    p.up_out = fused::make_rows(gate_up ? static_cast<char*>(gate_up) + N * width : nullptr, ld_gate_up, dt == BDR_F32);
    if ((rc = set_products(p, M, N, K, s, ws, f8))) return rc;
    if (f8) {  // the bytes lie where the bf16 operands would: those are written only once the 8-bit kernel has found nothing to do
        if ((rc = fused::encode_f8(*a, cfg_a->m, M, *w, cfg_w->m, 2 * N, 2, K, ws, reinterpret_cast<int*>(ws + s.flag), &p.f8, &p.gate, st))) return rc;
        if ((rc = fused::launch_f8<GatedJob<false>>(p, st))) return rc;
    }
    if ((rc = decode_pair(*a, cfg_a->m, M, reinterpret_cast<__nv_bfloat16*>(ws + s.a), *w, cfg_w->m, 2 * N, reinterpret_cast<__nv_bfloat16*>(ws + s.w), K,
                          s.pitch_k, st, p.gate, p.counters, s.n_counters)))
        return rc;
    if (dt == BDR_F32 && !fused::one_chain(cfg_a->m, cfg_w->m, p.span)) return fused::launch<GatedJobInSpans<false>>(p, st);
    return fused::launch<GatedJob<false>>(p, st);
}

int64_t mx_gated_gemm_bwd_workspace_bytes(int64_t M, int64_t N, int64_t K, bdr_dtype_t dt) {
    if (M < 0 || N < 0 || K < 1 || M > kMost || N > kMost || K > kMost) return 0;
    return GatedSpace(M, N, K, dt == BDR_F32 ? fused::kPartsF32 : 1).bytes;
}

int mx_gated_gemm_bwd(const bdr_config_t* cfg_a, const bdr_planes_t* a, const bdr_config_t* cfg_w, const bdr_planes_t* w, int64_t M, int64_t N,
                      int64_t K, int32_t act, const void* dh, bdr_dtype_t dt, int64_t ld_dh, const void* gate_up, int64_t ld_gate_up, void* da,
                      int64_t ld_da, void* dw, int64_t ld_dw, void* workspace, int64_t workspace_bytes, void* stream) {
    if (dt != BDR_F32 && dt != BDR_BF16) return BDR_ERR_UNSUPPORTED;
    if (!act::known(act)) return BDR_ERR_UNSUPPORTED;
    if (M < 0 || N < 0 || K < 0 || M > kMost || N > kMost || K > kMost) return BDR_ERR_SIZE;
    const int64_t tiles_k = (K + 255) / 256;
    if (K == 0 || ((M + 255) / 256) * std::max(tiles_k, (N + kRows - 1) / kRows) >= (1ll << 29) || ((N + 255) / 256) * tiles_k >= (1ll << 29) ||
        (N + kBK - 1) / kBK * 4 >= (1ll << 30))
        return BDR_ERR_UNSUPPORTED;
    int rc = check_table2_config(cfg_a);
    if (!rc) rc = check_table2_config(cfg_w);
    if (rc) return rc;
    const int width = dt == BDR_F32 ? 4 : 2;
    if (da && M > 0 && (rc = check_rows(da, ld_da, K, width))) return rc;
    if (dw && N > 0 && (rc = check_rows(dw, ld_dw, K, width))) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    if (M == 0 || N == 0) {  // sums over nothing
        if (da && M > 0 && cudaMemset2DAsync(da, ld_da * width, 0, K * width, M, st) != cudaSuccess) return BDR_ERR_CUDA;
        if (dw && N > 0 && cudaMemset2DAsync(dw, ld_dw * width, 0, K * width, 2 * N, st) != cudaSuccess) return BDR_ERR_CUDA;
        return BDR_OK;
    }
    if (!da && !dw) return BDR_OK;
    if ((rc = check_fused_operands(cfg_a, a, cfg_w, w, K))) return rc;
    if ((rc = check_rows(dh, ld_dh, N, width))) return rc;
    if (gate_up && (rc = check_rows(gate_up, ld_gate_up, 2 * N, width))) return rc;
    const int parts = dt == BDR_F32 ? fused::kPartsF32 : 1;
    const GatedSpace s(M, N, K, parts);
    if (!workspace || workspace_bytes < s.bytes) return BDR_ERR_WORKSPACE;
    if ((uintptr_t)workspace % 256) return BDR_ERR_MISALIGNED;
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    __nv_bfloat16 *const wa = reinterpret_cast<__nv_bfloat16*>(ws + s.a), *const ww = reinterpret_cast<__nv_bfloat16*>(ws + s.w),
                         *const d = reinterpret_cast<__nv_bfloat16*>(ws + s.d);
    if ((rc = decode_pair(*a, cfg_a->m, M, wa, *w, cfg_w->m, 2 * N, ww, K, s.pitch_k, st, nullptr, reinterpret_cast<int*>(ws + s.counters), s.n_counters)))
        return rc;
    const bool f32 = dt == BDR_F32;
    const Rows dh_rows = fused::make_rows(dh, ld_dh, f32), d_rows = fused::make_rows(d, s.pitch_d, false);
    if (gate_up) {
        const Rows g = fused::make_rows(gate_up, ld_gate_up, f32), u = fused::make_rows(static_cast<const char*>(gate_up) + N * width, ld_gate_up, f32);
        rc = f32 ? launch_gated_grad<true>(g, u, dh_rows, act, M, N, d_rows, st) : launch_gated_grad<false>(g, u, dh_rows, act, M, N, d_rows, st);
        if (rc) return rc;
    } else {
        GatedJob<true>::Params p = {};
        const bool f8 = fused::takes_f8(cfg_a->m, cfg_w->m, M, 2 * N, N, K);
        if ((rc = set_products(p, M, N, K, s, ws, f8))) return rc;
        p.act = act;
        p.h = dh_rows;
        p.d = d_rows;
        p.parts = parts;
        if (f8) {
            if ((rc = fused::encode_f8(*a, cfg_a->m, M, *w, cfg_w->m, 2 * N, 2, K, ws + s.f8, reinterpret_cast<int*>(ws + s.flag), &p.f8, &p.gate, st))) return rc;
            if ((rc = fused::launch_f8<GatedJob<true>>(p, st))) return rc;
        }
        rc = f32 && !fused::one_chain(cfg_a->m, cfg_w->m, p.span) ? fused::launch<GatedJobInSpans<true>>(p, st) : fused::launch<GatedJob<true>>(p, st);
        if (rc) return rc;
    }
    GradProducts g = {};
    g.d = d; g.a = wa; g.w = ww;
    g.M = M; g.N = N; g.K = K; g.pitch_d = s.pitch_d; g.pitch_k = s.pitch_k;
    g.segs = 2; g.parts = parts;
    g.da = da; g.dw = dw; g.ld_da = ld_da; g.ld_dw = ld_dw;
    g.f32 = f32;
    g.sums = reinterpret_cast<float*>(ws + s.sums);
    g.first = g.last = true;
    return launch_grad_products(g, st);
}

}  // extern "C"
