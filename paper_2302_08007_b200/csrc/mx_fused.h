// Host-side declarations shared by the operators that fuse work to a product of packed operands (gated feed-forward layer,
// cross entropy): decoding into a workspace, and the two gradient products.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "bdr.h"

namespace bdr {

int* device_status_word();

constexpr int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Pitch (elements) of lines of K decoded elements: whole items of the decode kernel.
constexpr int64_t line_pitch(int64_t K) { return round_up(K, 32); }

// Whether a row counts: its target is a column of the vocabulary.
__host__ __device__ constexpr bool row_counts(int64_t target, int64_t V) { return target >= 0 && target < V; }
// The largest |dloss| of the rows that count, by which a gradient is divided before it is rounded to bf16 and the results are
// multiplied in fp32; 1 where there is none, or an infinity.
struct Largest {
    const float* dloss;
    const int64_t* targets;
    int64_t M, V;
    float* out;
};
// Packed lines of K elements (Table II formats, m magnitude bits) of two operands -> bf16 [rows, pitch]; what lies behind K in a row is
// unspecified.  gate: NULL, or device flag without which nothing is decoded.  n_zero words at `zero` are cleared on the side.
// beside: the kernel in front in the stream is a product that does not read the output: it is decoded on what that product leaves free of the
// SMs, and is complete when both are.  largest: NULL, or what a block of its own computes on the side; blocks of a without values (exponent
// byte 0xFF) in rows that do not count are then zeros instead of NaN, which would stay NaN in a product with the row's zero gradient.
int decode_pair(const bdr_planes_t& a, int m_a, int64_t rows_a, __nv_bfloat16* out_a, const bdr_planes_t& w, int m_w, int64_t rows_w, __nv_bfloat16* out_w,
                int64_t K, int64_t pitch, cudaStream_t st, const int* gate = nullptr, int* zero = nullptr, int64_t n_zero = 0, bool beside = false, const Largest* largest = nullptr);

// Launches a kernel without shared memory behind another in the stream so that it is set up while that one drains; the kernel waits for it
// (griddepcontrol.wait) before it touches memory.
template <typename... P, typename... A>
int launch_dependent(void (*kern)(P...), dim3 grid, dim3 block, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, P(args)...);
    return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

// The gradient products.  D is bf16 [parts * segs][M][pitch_d] of which N columns count: D = sum over parts, segment s belongs to
// the weight lines w + s * N * pitch_k.  dA[M, K] (+)= sum_s D_s W_s, dW[s * N + n, K] = D_s^T A.  W is bf16 [segs * N, pitch_k],
// A bf16 [M, pitch_k].
struct GradProducts {
    const __nv_bfloat16 *d, *a, *w;
    int64_t M, N, K, pitch_d, pitch_k;
    int segs, parts;
    void *da, *dw;          // either may be NULL: not computed
    int64_t ld_da, ld_dw;   // elements
    bool f32;               // type of da and dw (else bf16)
    float* acc;             // fp32 [M, ld_acc] running sum of dA over several calls; NULL: this call is the only one
    int64_t ld_acc;
    float* sums;            // grad_sums_bytes(M, N, K, segs) bytes
    const float* scale;     // device: factor of both gradients; NULL: 1
    const int64_t* targets; // device, NULL or [M]: rows of dA that do not count are zeros, whatever W holds
    int64_t vocab;
    bool first, last;       // of those calls: the first does not read acc, the last writes da
};
int64_t grad_sums_bytes(int64_t M, int64_t N, int64_t K, int segs);
int launch_grad_products(const GradProducts& g, cudaStream_t st);

// The gated layer of a few rows of bf16 x (mx_gated_gemv), with both products stored where `products` is not NULL.
int gated_rows(const bdr_config_t* cfg_w, const bdr_planes_t* w, int64_t N, int64_t K, const __nv_bfloat16* x, int64_t ldx, int64_t T, int act, void* h,
               bdr_dtype_t dt, int64_t ldh, void* products, int64_t ld_products, cudaStream_t st);

// Few rows are left to the few-token kernel, which reads the packed weights, instead of decoding them for the tensor-core kernel, which would
// multiply 256 rows all the same.  Measured (gated layer, MX9, few-token and tensor-core kernel): 8000 lines of 1024, 24 rows 17.4 and 21.4 us, 32 rows 19.5 and
// 21.4, 48 rows 21.5 and 21.4; 2000 lines of 8192, 24 rows 33.8 and 35.8, 32 rows 37.9 and 33.9; 32000 lines of 4096, 16 rows 54 and 140, 48 rows 114 and
// 140; 1000 lines of 256 alike up to 16 rows, where the cross entropy, which needs two launches more for the few-token kernel's logits, takes 19.5 and 15.4.
constexpr int64_t kMostFewRows = 48;
inline bool few_rows(int64_t M, int64_t lines, int64_t K) { return lines * K >= 1ll << 21 && M <= (lines * K >= 1ll << 25 ? kMostFewRows : 24); }

// Host checks of the shares that the operators' launches follow, over sizes from one to the largest (bdr_selftest_host).
bool entropy_pieces_hold();

// What the operators accept of two packed operands A [M, K] and W [lines, K] (host).
int check_fused_operands(const bdr_config_t* cfg_a, const bdr_planes_t* a, const bdr_config_t* cfg_w, const bdr_planes_t* w, int64_t K);

}  // namespace bdr
