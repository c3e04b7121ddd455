// Few-token product with packed weights: y[T, N] = x[T, K] deq(W)[N, K]^T, the linear layers of token-by-token inference
// (Section V, inferencing: weights are stored in the MX format; the activations stay as they are).
//
// Every packed weight is read once and used for T columns, so the kernel is bound by the bytes of W as long as decoding keeps
// up.  A warp owns 16 rows of W and walks along K in steps of 256 elements: lane (g, c) of the matrix instruction's layout
// takes blocks 4c .. 4c+3 of rows g and g + 8 (64 contiguous elements each: 24, 40 or 64 bytes of codes and one word each of
// exponents and microexponents), decodes them in registers and feeds 16 matrix instructions.  The activations sit in shared
// memory in the order those instructions want them, as bf16; a 32-bit activation is split exactly into three bf16 columns,
// which costs nothing while the eight columns of an instruction are not full.  The warps of a CTA split into rw row tiles
// times kw shares of K; the shares are added in shared memory in a fixed order.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "bdr_host.h"
#include "mx_frag.cuh"

namespace bdr {

constexpr int kGvThreads = 256, kGvWarps = kGvThreads / 32;
constexpr int kGvStep = 256;                 // elements of K per warp step
constexpr int kGvSmem = 72 * 1024;           // most shared memory for activations: three CTAs fit on an SM
constexpr int kGvMaxCols = 64;               // columns (tokens, or thirds of a 32-bit token) of one pass

struct GemvArgs {
    bdr_planes_t w;
    const void* x;
    void* y;
    int64_t ldx, ldy;
    int64_t n, k;
    int tokens, tokens_per_pass;
    int x32, y32;        // 32-bit activations / results (else bf16)
    int xvec;            // activations may be read four at a time
    int rw;              // row tiles of a CTA (a power of two up to 8)
    int phase_steps;     // steps whose activations fit in shared memory at once
};

// four consecutive blocks of one row
template <int W> struct Run {
    uint32_t w[2 * W];
    uint32_t exps, micro;
};

template <int W>
__device__ __forceinline__ void load_run(Run<W>& r, const bdr_planes_t& p, int64_t row, int block, int nb) {
    const uint8_t* codes = p.elems + row * p.ld_elems + (int64_t)block * (2 * W);
    const uint8_t* ex = p.exps + row * p.ld_exps + block;
    const uint8_t* mi = p.micro + row * p.ld_micro + block;
    if (block + 4 <= nb) {
        r.exps = __ldg(reinterpret_cast<const uint32_t*>(ex));
        r.micro = __ldg(reinterpret_cast<const uint32_t*>(mi));
        if constexpr (W == 8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 v = __ldg(reinterpret_cast<const uint4*>(codes) + i);
                r.w[4 * i] = v.x; r.w[4 * i + 1] = v.y; r.w[4 * i + 2] = v.z; r.w[4 * i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const uint2 v = __ldg(reinterpret_cast<const uint2*>(codes) + i);
                r.w[2 * i] = v.x; r.w[2 * i + 1] = v.y;
            }
        }
    } else {  // the end of a line: block by block, absent blocks are zero blocks
        r.exps = r.micro = 0;
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) r.w[i] = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            if (block + b < nb) {
                r.exps |= (uint32_t)__ldg(ex + b) << (8 * b);
                r.micro |= (uint32_t)__ldg(mi + b) << (8 * b);
#pragma unroll
                for (int h = 0; h < W; ++h) {
                    const int o = 2 * W * b + 2 * h;
                    r.w[o >> 2] |= (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(codes + o)) << (8 * (o & 2));
                }
            }
        }
    }
}

// Activations of K steps k0 / 256 .. into shared memory, in the order of the B fragments: a lane's word for two matrix
// instructions holds elements 4h .. 4h+3 of blocks 2p and 2p+1 of its four, alternating.  Word (p, h) of lane column c lies
// at 16 (4 p + h) + 4 c 32-bit words of the step: the eight lanes that a shared-memory request serves at a time (two columns,
// four c) hit different banks (column pitch 64 bytes off a multiple of 128).
template <bool X32>
__device__ __forceinline__ void stage_x(const GemvArgs& a, uint16_t* xs, int64_t pitch, int t0, int nt, int64_t k0, int span) {
    const int per = span / 8;
    for (int i = threadIdx.x; i < nt * per; i += kGvThreads) {
        const int t = i / per, v = i - t * per;
        const int s = v >> 5, c = (v >> 3) & 3, p = (v >> 2) & 1, h = v & 3;
        const int64_t k = k0 + (int64_t)s * kGvStep + 64 * c + 32 * p + 4 * h;
        const int64_t at = (int64_t)s * kGvStep + (4 * p + h) * 32 + c * 8;
        if constexpr (X32) {
            const float* x = static_cast<const float*>(a.x) + (int64_t)(t0 + t) * a.ldx + k;
            float f[8];
            if (a.xvec && k + 20 <= a.k) {
                const float4 u = __ldg(reinterpret_cast<const float4*>(x)), w = __ldg(reinterpret_cast<const float4*>(x) + 4);
                f[0] = u.x; f[1] = w.x; f[2] = u.y; f[3] = w.y; f[4] = u.z; f[5] = w.z; f[6] = u.w; f[7] = w.w;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int o = (e >> 1) + 16 * (e & 1);
                    f[e] = k + o < a.k ? __ldg(x + o) : 0.f;
                }
            }
            uint16_t q[8][3];
#pragma unroll
            for (int e = 0; e < 8; ++e) frag::split3(f[e], q[e]);
#pragma unroll
            for (int part = 0; part < 3; ++part)
                *reinterpret_cast<uint4*>(xs + (3 * t + part) * pitch + at) =
                    make_uint4(frag::pack2(q[0][part], q[1][part]), frag::pack2(q[2][part], q[3][part]),
                               frag::pack2(q[4][part], q[5][part]), frag::pack2(q[6][part], q[7][part]));
        } else {
            const uint16_t* x = static_cast<const uint16_t*>(a.x) + (int64_t)(t0 + t) * a.ldx + k;
            uint2 u, w;
            if (a.xvec && k + 20 <= a.k) {
                u = __ldg(reinterpret_cast<const uint2*>(x));
                w = __ldg(reinterpret_cast<const uint2*>(x) + 4);
            } else {
                uint16_t q[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int o = (e & 3) + 16 * (e >> 2);
                    q[e] = k + o < a.k ? __ldg(x + o) : (uint16_t)0;
                }
                u = make_uint2(frag::pack2(q[0], q[1]), frag::pack2(q[2], q[3]));
                w = make_uint2(frag::pack2(q[4], q[5]), frag::pack2(q[6], q[7]));
            }
            *reinterpret_cast<uint4*>(xs + t * pitch + at) =
                make_uint4(__byte_perm(u.x, w.x, 0x5410), __byte_perm(u.x, w.x, 0x7632), __byte_perm(u.y, w.y, 0x5410), __byte_perm(u.y, w.y, 0x7632));
        }
    }
}

// One step of a warp.  The tensor core's fp32 additions are cut off rather than rounded, so a step's products are summed from
// zero and then added to the totals with a rounded addition: 16 instructions in a chain instead of K / 16.
template <int W, int NT>
__device__ __forceinline__ void run_step(const Run<W>& r0, const Run<W>& r1, const uint16_t* xs, int64_t pitch, int cols, int lane,
                                         float (&acc)[NT][4]) {
    const int g = lane >> 2, c = lane & 3;
    float part[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[n][i] = 0.f;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const frag::Scales s0 = frag::make_scales(frag::spread_bytes(r0.exps >> (16 * p)), frag::spread_bytes(r0.micro >> (16 * p)));
        const frag::Scales s1 = frag::make_scales(frag::spread_bytes(r1.exps >> (16 * p)), frag::spread_bytes(r1.micro >> (16 * p)));
        const int a0 = 32 * W * p, b0 = a0 + 16 * W;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            uint32_t y0[4], y1[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y0[e] = frag::decode_word<W>(r0.w, a0, r0.w, b0, 4 * h + e, frag::scale_word(s0, 2 * h + (e >> 1)));
                y1[e] = frag::decode_word<W>(r1.w, a0, r1.w, b0, 4 * h + e, frag::scale_word(s1, 2 * h + (e >> 1)));
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                // a column beyond the last repeats it: what it gives is not looked at
                const uint4 x = *reinterpret_cast<const uint4*>(xs + min(8 * n + g, cols - 1) * pitch + (4 * p + h) * 32 + c * 8);
                frag::mma_bf16(part[n], y0[0], y1[0], y0[1], y1[1], x.x, x.y);
                frag::mma_bf16(part[n], y0[2], y1[2], y0[3], y1[3], x.z, x.w);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] += part[n][i];
}

template <int W, int NT, bool X32>
__global__ void __launch_bounds__(kGvThreads, NT <= 2 ? 3 : 2) mx_gemv_kernel(const GemvArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    uint16_t* xs = reinterpret_cast<uint16_t*>(smem);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int rw = a.rw, kw = kGvWarps / rw, my_r = warp & (rw - 1), my_k = warp / rw;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * rw);
    const int t0 = blockIdx.y * a.tokens_per_pass, nt = min(a.tokens_per_pass, a.tokens - t0), cols = X32 ? 3 * nt : nt;
    const int nb = (int)((a.k + 15) / 16), steps = (nb + 15) / 16;
    const int64_t row0 = min(n0 + 16 * my_r + g, a.n - 1), row1 = min(n0 + 16 * my_r + g + 8, a.n - 1);
    const int64_t pitch = (int64_t)min(a.phase_steps, steps) * kGvStep + 32;
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.f;

    // The next step's words are fetched once the present one is decoded; the SM's other warps cover the wait.
    Run<W> run[2];
    auto fetch = [&](int s) {
        load_run<W>(run[0], a.w, row0, 16 * s + 4 * c, nb);
        load_run<W>(run[1], a.w, row1, 16 * s + 4 * c, nb);
    };
    int s = my_k;
    if (s < steps) fetch(s);
    for (int p0 = 0; p0 < steps; p0 += a.phase_steps) {
        const int p1 = min(p0 + a.phase_steps, steps);
        if (p0) __syncthreads();  // everyone is done with the phase before
        stage_x<X32>(a, xs, pitch, t0, nt, (int64_t)p0 * kGvStep, (p1 - p0) * kGvStep);
        __syncthreads();
        for (; s < p1; s += kw) {
            run_step<W, NT>(run[0], run[1], xs + (int64_t)(s - p0) * kGvStep, pitch, cols, lane, acc);
            if (s + kw < steps) fetch(s + kw);
        }
    }
    // the shares of K, added in order; each row tile's results are [column][16 rows]
    __syncthreads();
    float* red = reinterpret_cast<float*>(smem);
    const int tile = 8 * NT * 16;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[(my_k * rw + my_r) * tile + (8 * n + 2 * c + (i & 1)) * 16 + g + 8 * (i >> 1)] = acc[n][i];
    __syncthreads();
    for (int i = threadIdx.x; i < nt * 16 * rw; i += kGvThreads) {
        const int t = i / (16 * rw), r = i - t * (16 * rw);
        if (n0 + r >= a.n) continue;
        float v = 0.f;
        for (int part = 0; part < (X32 ? 3 : 1); ++part) {
            const int col = X32 ? 3 * t + (2 - part) : t;  // smallest part first
            for (int q = 0; q < kw; ++q) v += red[(q * rw + (r >> 4)) * tile + col * 16 + (r & 15)];
        }
        v *= 2.f;  // the operand was decoded halved
        const int64_t at = (int64_t)(t0 + t) * a.ldy + n0 + r;
        if (a.y32) static_cast<float*>(a.y)[at] = v;
        else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
    }
}

template <int W, int NT, bool X32>
static int launch_gemv(GemvArgs a, cudaStream_t st) {
    static PerDevice once;
    if (kernel_setup(once, mx_gemv_kernel<W, NT, X32>, kGvThreads, kGvSmem) < 1) return BDR_ERR_CUDA;
    const int cols = (X32 ? 3 : 1) * std::min(a.tokens, a.tokens_per_pass);
    const int steps = (int)((a.k + kGvStep - 1) / kGvStep);
    // as many row tiles per CTA as there are groups of eight columns: the activations are fetched once per CTA, and a CTA's
    // weights should outweigh them
    a.rw = NT >= 4 ? 4 : NT;
    const int kw = kGvWarps / a.rw;
    a.phase_steps = (int)((kGvSmem / cols - 64) / (2 * kGvStep)) / kw * kw;
    const size_t smem = std::max<size_t>((size_t)cols * (std::min(a.phase_steps, steps) * kGvStep * 2 + 64),
                                         (size_t)kGvWarps * 8 * NT * 16 * 4);
    const dim3 grid((unsigned)((a.n + 16 * a.rw - 1) / (16 * a.rw)), (unsigned)((a.tokens + a.tokens_per_pass - 1) / a.tokens_per_pass));
    mx_gemv_kernel<W, NT, X32><<<grid, kGvThreads, smem, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

template <int W, bool X32>
static int pick_columns(GemvArgs a, cudaStream_t st) {
    a.tokens_per_pass = X32 ? kGvMaxCols / 3 : kGvMaxCols;
    const int cols = (X32 ? 3 : 1) * std::min(a.tokens, a.tokens_per_pass);
    if (cols <= 8) return launch_gemv<W, 1, X32>(a, st);
    if (cols <= 16) return launch_gemv<W, 2, X32>(a, st);
    if (cols <= 32) return launch_gemv<W, 4, X32>(a, st);
    return launch_gemv<W, 8, X32>(a, st);
}

}  // namespace bdr

using namespace bdr;

extern "C" int mx_gemv(const bdr_config_t* cfg_w, const bdr_planes_t* w, int64_t N, int64_t K, const void* x, bdr_dtype_t x_dt,
                       int64_t ldx, int64_t T, void* y, bdr_dtype_t y_dt, int64_t ldy, void* stream) {
    int rc = check_table2_config(cfg_w);
    if (rc) return rc;
    for (int dt : {(int)x_dt, (int)y_dt})
        if (dt != BDR_F32 && dt != BDR_BF16) return BDR_ERR_UNSUPPORTED;
    if (N < 0 || K < 0 || T < 0 || ldx < K || ldy < N || K > (1ll << 30) || N > (1ll << 34) || T > (1ll << 20)) return BDR_ERR_SIZE;
    if (T == 0 || N == 0) return BDR_OK;
    if (!y) return BDR_ERR_NULL;
    if ((uintptr_t)y % (y_dt == BDR_F32 ? 4 : 2)) return BDR_ERR_MISALIGNED;
    GemvArgs a = {};
    if (K > 0) {  // a sum over nothing is zero
        if (!x) return BDR_ERR_NULL;
        if ((uintptr_t)x % (x_dt == BDR_F32 ? 4 : 2)) return BDR_ERR_MISALIGNED;
        if ((rc = check_table2_planes(cfg_w, w, K))) return rc;
        a.w = *w;
    }
    a.x = x; a.y = y; a.ldx = ldx; a.ldy = ldy; a.n = N; a.k = K; a.tokens = (int)T;
    a.x32 = x_dt == BDR_F32; a.y32 = y_dt == BDR_F32;
    const int64_t xb = a.x32 ? 4 : 2;
    a.xvec = (uintptr_t)x % (4 * xb) == 0 && (T == 1 || ldx % 4 == 0);
    cudaStream_t st = (cudaStream_t)stream;
    switch (cfg_w->m) {
        case 2: return a.x32 ? pick_columns<3, true>(a, st) : pick_columns<3, false>(a, st);
        case 4: return a.x32 ? pick_columns<5, true>(a, st) : pick_columns<5, false>(a, st);
        case 7: return a.x32 ? pick_columns<8, true>(a, st) : pick_columns<8, false>(a, st);
    }
    return BDR_ERR_UNSUPPORTED;
}
