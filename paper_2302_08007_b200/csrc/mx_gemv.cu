// Few-token product with packed weights: y[T, N] = x[T, K] deq(W)[N, K]^T, the linear layers of token-by-token inference.  The weights
// are kept in the MX format (Section V, inferencing).  That the activations stay as they are is this library's choice: the section
// quantizes them on the way to the product, which pays where the product itself is computed on the format.
//
// Every packed weight is read once and used for T columns, so the kernel is bound by the bytes of W as long as decoding keeps
// up.  A warp owns 16 rows of W and walks along K in steps of 256 elements: lane (g, c) of the matrix instruction's layout
// takes four blocks of rows g and g + 8 (24, 40 or 64 bytes of codes each), decodes them in registers and feeds 16 matrix
// instructions.  The bytes come through a ring of the warp's own in shared memory, filled by 16-byte asynchronous copies one or
// two steps ahead: a lane's own bytes are strided in memory, and loads of them straight into registers kept the L1 busy with
// four times as many lines per request and the compiler moving them down to where they were needed (16384 x 4096 MX9, the same
// weights again and again: 18.5 us, with the ring 15.8).  The activations sit in shared memory in the order those instructions want them, as bf16; a 32-bit
// activation is split exactly into three bf16 columns, which costs nothing while the eight columns of an instruction are not full.
// One CTA per SM stays for the whole call and its warps form groups of kw that share a tile's K; a group's sums are added in
// shared memory in a fixed order.  The host picks kw so that the longest group's walk is shortest: few large groups balance few
// rows, many small ones need fewer joins.  Activations that do not fit beside the rings come in phases, each copied while the
// one before is computed (loaded, ordered and stored between two phases instead, they took as long as the products: 16 tokens of
// 16384 x 8192 MX9 67.8 us, now 45).
//
// Measured (bf16 activations, the weights not in the L2): one token, 16384 x 4096 MX9 17.9 us = 4.2 TB/s, 16384 x 16384 MX9 57 us =
// 5.3 TB/s, MX6 68 us = 3.0 TB/s, MX4 58 us = 2.3 TB/s, 16384 x 4096 MX6 20 us = 2.5 TB/s, 4096 x 4096 MX4 7.4 us; 16 tokens,
// 16384 x 8192 MX9 45.6 us = 3.3 TB/s, MX6 50.5 us; 32 and 64 tokens, 16384 x 4096 MX9 34.5 and 63.6 us (16: 26.0).  MX9 is near the
// memory's rate for one token; MX6 and MX4 are bound by decoding (the integer/logic pipe, and latency: no pipe is more than two thirds
// busy); sixteen tokens by decoding on half the warps, which is what the registers of two column groups allow.  Small products are
// a launch and one trip to memory.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "bdr_device.cuh"
#include "bdr_host.h"
#include "mx_frag.cuh"

namespace bdr {

constexpr int kGvStep = 256;                 // elements of K per warp step
constexpr int kGvSmem = 227 * 1024;
constexpr int kGvMaxCols = 64;               // columns (tokens, or thirds of a 32-bit token) of one pass

// Warps of a CTA: 16 of up to 128 registers when there are few columns, 8 (and shared memory left for the activations) when there are
// more.  Two groups of columns run with 16 warps for 3-bit codes, whose rings are small; with 5-bit codes the activations of K = 4096 would
// no longer fit beside the rings (16 of 4096 x 4096: 13.5 us, with eight 11.5).  For 3-bit codes the choice is made per call.  Where the
// activations fit beside either's rings, or beside neither's, 16 warps are 3 to 17 % faster (16 tokens of 4096 x 4096: 10.0 us, with eight
// 11.3).  Where they fit beside those of eight only, eight win as long as an SM has at most two row tiles, whose phases nothing hides (16
// tokens of 2048 x 4352: 9.5 us, with sixteen 10.4; of 4096 x 5120 13.3, 13.8; 9 of 1024 x 8960 12.7, 15.1); from three tiles on sixteen are
// ahead (16 tokens of 5120 x 5120: 16.3 us, with eight 17.0; of 16384 x 5120 28.3, 30.0; 9 of 16384 x 8960 42.5, 45.7; of 8192 x 4352 they
// lose by 4 %).
__host__ __device__ constexpr int gemv_warps(int w, int nt) { return nt == 1 || (nt == 2 && w == 3) ? 16 : 8; }

template <int W, int NT, int WARPS> struct GemvShape {
    static constexpr int kWarps = WARPS, kThreads = 32 * kWarps;
    static constexpr int kRed = kWarps * 8 * NT * 16 * 4;  // bytes of all warps' sums of a tile
    static constexpr int kPitch = 32 * W;                  // bytes of codes of a row and step
    static constexpr int kAtX = 16 * kPitch, kStage = kAtX + 2 * 256;  // 16 rows of codes, of exponents, of microexponents
    static constexpr int kStages = W != 8 && (NT == 1 || (NT == 2 && W == 5)) ? 3 : 2;  // steps in a warp's ring
    static constexpr int kReds = NT < 4 ? 2 : 1;                       // buffers of sums
    static constexpr int kXs = kReds * kRed + kWarps * kStages * kStage;  // where the activations start
    // steps whose activations fit beside the rings, for a number of columns
    static int fit(int cols) { return ((kGvSmem - kXs) / cols - 64) / (2 * kGvStep); }
};

struct GemvArgs {
    bdr_planes_t w;
    const void* x;
    void* y;
    int64_t ldx, ldy;
    int64_t n, k;
    int tokens, tokens_per_pass;
    int x32, y32;        // 32-bit activations / results (else bf16)
    int xalign;          // rows of activations start on boundaries of 16, 4 or 2 bytes
    int kw, kw_log;      // warps that share a tile's K (a power of two, at most the steps there are)
    int rounds;          // of the groups over all tiles, rounded down; the first `rest` CTAs have one more
    unsigned rest;
    int phase_steps;     // steps whose activations are in shared memory at once: all, or a multiple of kw in each of two buffers
};

// Four blocks of one row.  3- and 5-bit codes: blocks 4c .. 4c + 3 of a step, 24 or 40 contiguous bytes of the ring, which eight
// lanes (two rows, four c) read from different banks as they lie.  8-bit codes: blocks c, c + 4, c + 8, c + 12, so that the four
// lanes of a row read 64 contiguous bytes at a time (the upper and lower half of a row's 128 bytes change places in odd rows);
// of the scales they read the row's whole word of sixteen and pick theirs.
template <int W> struct Run {
    uint32_t w[2 * W];
    uint32_t exps[2], micro[2];  // of blocks 2p and 2p + 1 of the run, one per half (8-bit codes: bits 8 .. 15 of micro are leftovers)
};
template <int W>
__device__ __forceinline__ constexpr int run_block(int c, int i) { return W == 8 ? c + 4 * i : 4 * c + i; }

template <int W>
__device__ __forceinline__ void read_run(Run<W>& r, const uint8_t* stage, int row, int c) {
    constexpr int kPitch = 32 * W, kAtX = 16 * kPitch;
    const uint8_t* codes = stage + row * kPitch;
    const uint8_t* scales = stage + kAtX + row * 16;
    if constexpr (W == 8) {
        const uint4 e = *reinterpret_cast<const uint4*>(scales), m = *reinterpret_cast<const uint4*>(scales + 256);
        const uint32_t pick = 0x4400u + 0x1111u * c;  // byte c of one word in the low half, of the other in the high half
        r.exps[0] = __byte_perm(e.x, e.y, pick) & 0x00FF00FFu;
        r.exps[1] = __byte_perm(e.z, e.w, pick) & 0x00FF00FFu;
        r.micro[0] = __byte_perm(m.x, m.y, pick);
        r.micro[1] = __byte_perm(m.z, m.w, pick);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 v = *reinterpret_cast<const uint4*>(codes + 16 * ((c + 4 * i) ^ (4 * (row & 1))));
            r.w[4 * i] = v.x; r.w[4 * i + 1] = v.y; r.w[4 * i + 2] = v.z; r.w[4 * i + 3] = v.w;
        }
    } else {
        const uint32_t e = *reinterpret_cast<const uint32_t*>(scales + 4 * c), m = *reinterpret_cast<const uint32_t*>(scales + 256 + 4 * c);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            r.exps[p] = frag::spread_bytes(e >> (16 * p));
            r.micro[p] = frag::spread_bytes(m >> (16 * p));
        }
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const uint2 v = reinterpret_cast<const uint2*>(codes + 8 * W * c)[i];
            r.w[2 * i] = v.x; r.w[2 * i + 1] = v.y;
        }
    }
}

// s * bytes + p in one instruction of the multiply-add pipe
__device__ __forceinline__ const uint8_t* step_from(const uint8_t* p, int s, uint32_t bytes) {
    const uint8_t* q;
    asm("mad.wide.u32 %0, %1, %2, %3;" : "=l"(q) : "r"((uint32_t)s), "r"(bytes), "l"(p));
    return q;
}

// A warp's copies of a step of a row tile, with their sources kept as pointers into the tile's rows.
template <int W>
struct StepCopies {
    static constexpr int kPieces = 2 * W, kCount = 16 * kPieces / 32;  // 16-byte pieces of a row; copies per lane
    static constexpr int kPitch = 32 * W, kAtX = 16 * kPitch;
    const uint8_t *code[kCount], *scale;
    __device__ __forceinline__ void point(const bdr_planes_t& p, int64_t tile, int64_t n, int lane) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int at = lane + 32 * i, row = at / kPieces;
            code[i] = p.elems + min(16 * tile + row, n - 1) * p.ld_elems + 16 * (at - row * kPieces);
        }
        const int64_t row = min(16 * tile + (lane & 15), n - 1);
        scale = lane < 16 ? p.exps + row * p.ld_exps : p.micro + row * p.ld_micro;
    }
    // TAIL: the step may pass the end of the rows; what lies beyond a row's pitch is left out
    template <bool TAIL>
    __device__ __forceinline__ void queue(uint8_t* stage, const bdr_planes_t& p, int s, int lane) const {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int at = lane + 32 * i, row = at / kPieces, piece = at - row * kPieces;
            const int unit = W == 8 ? piece ^ (4 * (row & 1)) : piece;
            if (!TAIL || (int64_t)s * kPitch + 16 * piece < p.ld_elems) cp_async16(stage + row * kPitch + 16 * unit, step_from(code[i], s, kPitch));
        }
        if (!TAIL || (int64_t)s * 16 < (lane < 16 ? p.ld_exps : p.ld_micro)) cp_async16(stage + kAtX + lane * 16, step_from(scale, s, 16));
    }
};

// Activations of some K steps in shared memory, in the order of the B fragments: a lane's 16 bytes for two matrix instructions hold
// elements 4h .. 4h+3 of blocks 2p and 2p+1 of its four, alternating.  Where they lie in a column's step of 512 bytes, in units of 16:
// the eight lanes that a shared-memory request serves at a time (two columns, 64 bytes off a multiple of 128 apart, and four c) hit
// different banks, and so do those that put the activations in order (below).
// That order costs the reader more address arithmetic, so up to eight columns, which are put in order quickly, do without.
template <int W, int NT>
__device__ __forceinline__ int x_slot(int c, int p, int h) { return W == 8 || NT == 1 ? 4 * (4 * p + h) + c : 8 * c + ((4 * p + h) ^ c); }

// They come as they are, by asynchronous copies that run while the phase before is computed, and are put in order in place by the warp
// that copied them.  A warp's share is a step of two tokens (32-bit ones: of one token, in the first two of its three columns).
template <int W, int NT, bool X32>
struct StageX {
    int t, s, dt, ds, steps;
    __device__ __forceinline__ StageX(int n_steps) {  // not zero
        const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5;
        steps = n_steps;
        t = dt = 0; s = warp; ds = warps;
        if (warps > n_steps) {
            t = warp / n_steps; s = warp - t * n_steps;
            dt = warps / n_steps; ds = warps - dt * n_steps;
            if constexpr (!X32) { t *= 2; dt *= 2; }
        }
    }
    __device__ __forceinline__ void next() {
        t += dt; s += ds;
        if (s >= steps) { s -= steps; t += X32 ? 1 : 2; }
    }
    // the 16 bytes of a row at x, of which `left` elements exist, zeros behind them
    template <typename T>
    __device__ static __forceinline__ void piece(uint16_t* to, const T* x, const T* row, int64_t left, int align) {
        constexpr int kN = X32 ? 4 : 8;
        if (align == 16 && left >= kN) {
            cp_async16(to, x);
        } else if (align >= 4) {
            const int bytes = (int)max((int64_t)0, min((int64_t)kN, left)) * (int)sizeof(T);
            if (bytes == 0) x = row;
            if (align == 16) cp_async16_part(to, x, bytes);
            else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    cp_async4_part(to + 2 * i, bytes > 4 * i ? reinterpret_cast<const char*>(x) + 4 * i : reinterpret_cast<const char*>(x), max(0, min(4, bytes - 4 * i)));
            }
        } else {
            T q[kN];
#pragma unroll
            for (int e = 0; e < kN; ++e) q[e] = e < left ? __ldg(x + e) : (T)0;
            *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(q);
        }
    }
    // starts the copies of steps s0 .. s0 + n_steps - 1 of nt tokens
    __device__ static __forceinline__ void copy(const GemvArgs& a, uint16_t* xs, int64_t pitch, int t0, int nt, int s0, int n_steps) {
        using T = typename std::conditional<X32, float, uint16_t>::type;
        const int lane = threadIdx.x & 31;
        const int align = a.xalign;
        for (StageX m(n_steps); m.t < nt; m.next()) {
            const T* const row = static_cast<const T*>(a.x) + (t0 + m.t) * a.ldx;
            uint16_t* const to = xs + (X32 ? 3 : 1) * m.t * pitch + m.s * kGvStep + 8 * lane;
            const int64_t k = (int64_t)(s0 + m.s) * kGvStep + (X32 ? 4 : 8) * lane, left = a.k - k;
            piece<T>(to, row + k, row, left, align);
            if constexpr (X32) piece<T>(to + pitch, row + k + kGvStep / 2, row, left - kGvStep / 2, align);
            else if (m.t + 1 < nt) piece<T>(to + pitch, row + a.ldx + k, row, left, align);
        }
    }
    // puts them in order, once the warp's copies are there
    __device__ static __forceinline__ void arrange(uint16_t* xs, int64_t pitch, int nt, int n_steps) {
        const int lane = threadIdx.x & 31;
        __syncwarp();
        for (StageX m(n_steps); m.t < nt; m.next()) {
            uint16_t* const at = xs + (X32 ? 3 : 1) * m.t * pitch + m.s * kGvStep;
            if constexpr (X32) {
                const int h = lane & 3, c = W == 8 ? (lane >> 2) & 3 : lane >> 3, p = W == 8 ? lane >> 4 : (lane >> 2) & 1;
                auto from = [&](int i) {  // elements 4h .. of block 2p + i
                    const int piece = 4 * run_block<W>(c, 2 * p + i) + h;
                    return reinterpret_cast<const float4*>(at + (piece >> 5) * pitch + 8 * (piece & 31));
                };
                const float4 u = *from(0), w = *from(1);
                __syncwarp();
                const float f[8] = {u.x, w.x, u.y, w.y, u.z, w.z, u.w, w.w};
                uint16_t q[8][3];
#pragma unroll
                for (int e = 0; e < 8; ++e) frag::split3(f[e], q[e]);
#pragma unroll
                for (int part = 0; part < 3; ++part)
                    *reinterpret_cast<uint4*>(at + part * pitch + 8 * x_slot<W, NT>(c, p, h)) =
                        make_uint4(frag::pack2(q[0][part], q[1][part]), frag::pack2(q[2][part], q[3][part]),
                                   frag::pack2(q[4][part], q[5][part]), frag::pack2(q[6][part], q[7][part]));
            } else {
                // elements 8 half .. of blocks 2p and 2p + 1.  To hit all banks, lanes of odd c (3 and 5 bits) read the second block first,
                // and lanes of the upper half (8 bits) write the second 16 bytes first.
                const int half = lane & 1, c = W == 8 ? (lane >> 1) & 3 : (lane >> 2) & 3, p = W == 8 ? (lane >> 3) & 1 : (lane >> 1) & 1;
                const bool there = m.t + (lane >> 4) < nt;
                uint16_t* const mine = at + (lane >> 4) * pitch;
                const int swap = W == 8 ? 0 : c & 1;
                uint4 u = make_uint4(0, 0, 0, 0), w = u;
                if (there) {
                    u = *reinterpret_cast<const uint4*>(mine + 8 * (2 * run_block<W>(c, 2 * p + swap) + half));
                    w = *reinterpret_cast<const uint4*>(mine + 8 * (2 * run_block<W>(c, 2 * p + 1 - swap) + half));
                }
                __syncwarp();
                const uint32_t low = swap ? 0x1054u : 0x5410u, high = swap ? 0x3276u : 0x7632u;
                uint4 a0 = make_uint4(__byte_perm(u.x, w.x, low), __byte_perm(u.x, w.x, high), __byte_perm(u.y, w.y, low), __byte_perm(u.y, w.y, high));
                uint4 a1 = make_uint4(__byte_perm(u.z, w.z, low), __byte_perm(u.z, w.z, high), __byte_perm(u.w, w.w, low), __byte_perm(u.w, w.w, high));
                const int first = W == 8 ? half : 0;
                if (W == 8 && first) { const uint4 x = a0; a0 = a1; a1 = x; }
                if (there) {
                    *reinterpret_cast<uint4*>(mine + 8 * x_slot<W, NT>(c, p, 2 * half + first)) = a0;
                    *reinterpret_cast<uint4*>(mine + 8 * x_slot<W, NT>(c, p, 2 * half + 1 - first)) = a1;
                }
            }
        }
    }
};

// One step of a warp.  The tensor core's fp32 additions are cut off rather than rounded, so a step's products are summed from
// zero and then added to the totals with a rounded addition: 16 instructions in a chain instead of K / 16.
template <int W, int NT, bool FAST>
__device__ __forceinline__ void run_step_as(const Run<W>& r0, const Run<W>& r1, const uint16_t* xs, int64_t pitch, int cols, int lane,
                                            float (&acc)[NT][4]) {
    const int g = lane >> 2, c = lane & 3;
    float part[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[n][i] = 0.f;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const frag::Scales s0 = frag::make_scales<FAST>(r0.exps[p], r0.micro[p]);
        const frag::Scales s1 = frag::make_scales<FAST>(r1.exps[p], r1.micro[p]);
        const int a0 = 32 * W * p, b0 = a0 + 16 * W;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            uint32_t y0[4], y1[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y0[e] = frag::decode_word<W, FAST>(r0.w, a0, r0.w, b0, 4 * h + e, frag::scale_word(s0, 2 * h + (e >> 1)));
                y1[e] = frag::decode_word<W, FAST>(r1.w, a0, r1.w, b0, 4 * h + e, frag::scale_word(s1, 2 * h + (e >> 1)));
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                // a column beyond the last repeats it: what it gives is not looked at
                const uint4 x = *reinterpret_cast<const uint4*>(xs + min(8 * n + g, cols - 1) * pitch + 8 * x_slot<W, NT>(c, p, h));
                frag::mma_bf16(part[n], y0[0], y1[0], y0[1], y1[1], x.x, x.y);
                frag::mma_bf16(part[n], y0[2], y1[2], y0[3], y1[3], x.z, x.w);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = FAST ? fmaf(part[n][i], frag::kFastFactor, acc[n][i]) : acc[n][i] + part[n][i];
}
template <int W, int NT>
__device__ __forceinline__ void run_step(const Run<W>& r0, const Run<W>& r1, const uint16_t* xs, int64_t pitch, int cols, int lane,
                                         float (&acc)[NT][4]) {
    if (__all_sync(0xFFFFFFFFu, frag::all_fast(r0.exps[0] + (r0.exps[1] << 8)) && frag::all_fast(r1.exps[0] + (r1.exps[1] << 8)))) run_step_as<W, NT, true>(r0, r1, xs, pitch, cols, lane, acc);
    else run_step_as<W, NT, false>(r0, r1, xs, pitch, cols, lane, acc);
}

template <int W, int NT, bool X32, int WARPS>
__global__ void __launch_bounds__((GemvShape<W, NT, WARPS>::kThreads), 1) mx_gemv_kernel(const GemvArgs a) {
    using S = GemvShape<W, NT, WARPS>;
    constexpr int kWarps = S::kWarps, D = S::kStages;
    extern __shared__ __align__(16) uint8_t smem[];
    float* const red = reinterpret_cast<float*>(smem);
    uint16_t* const xs = reinterpret_cast<uint16_t*>(smem + S::kXs);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    uint8_t* const ring = smem + S::kReds * S::kRed + warp * (D * S::kStage);
    const int kw = a.kw, my_k = warp & (kw - 1), group = warp >> a.kw_log, groups = kWarps >> a.kw_log;
    const int t0 = blockIdx.y * a.tokens_per_pass, nt = min(a.tokens_per_pass, a.tokens - t0), cols = X32 ? 3 * nt : nt;
    const int nb = (int)((a.k + 15) / 16), steps = (nb + 15) / 16;
    // tiles go to the CTAs in turn, then to a CTA's groups: every SM has the same number to within one
    const int64_t tiles = (a.n + 15) / 16, stride = (int64_t)gridDim.x * groups;
    const int rounds = a.rounds + (blockIdx.x < a.rest ? 1 : 0);  // of the CTA's first group; the others may have one fewer
    const int64_t pitch = (int64_t)min(a.phase_steps, steps) * kGvStep + 32;
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.f;

    int64_t tile = blockIdx.x + (int64_t)group * gridDim.x;
    // the copies run ahead of the computation, across the ends of tiles
    StepCopies<W> copies;
    int64_t ahead_tile = tile;
    int ahead = my_k, to = 0, at = 0;
    if (ahead_tile < tiles) copies.point(a.w, ahead_tile, a.n, lane);
    auto queue_next = [&] {
        if (ahead_tile < tiles && ahead < steps) {
            if (16 * ahead + 16 <= nb) copies.template queue<false>(ring + to, a.w, ahead, lane);
            else copies.template queue<true>(ring + to, a.w, ahead, lane);
            ahead += kw;
            if (ahead >= steps) {
                ahead = my_k;
                ahead_tile += stride;
                if (ahead_tile < tiles) copies.point(a.w, ahead_tile, a.n, lane);
            }
        }
        cp_async_commit();
        to = to + S::kStage == D * S::kStage ? 0 : to + S::kStage;
    };
    // Activations: the first phase now, each other one while the phase before it is computed.  With few columns and a ring of three
    // steps, the first step of weights goes ahead of them (16384 x 4096 MX6: 18.7 us, else 19.0; with two steps MX9 16.5, else 16.2).
    constexpr bool kWeightsFirst = NT == 1 && D == 3;
    constexpr int kBehind = kWeightsFirst ? D - 2 : D - 1;  // steps of weights behind the activations
    using X = StageX<W, NT, X32>;
    if (kWeightsFirst) queue_next();
    if (steps > 0) X::copy(a, xs, pitch, t0, nt, 0, min(a.phase_steps, steps));
    cp_async_commit();
#pragma unroll
    for (int i = 0; i < kBehind; ++i) queue_next();
    cp_async_wait<kBehind>();
    if (steps > 0) X::arrange(xs, pitch, nt, min(a.phase_steps, steps));
    __syncthreads();
    int64_t buffer = 0, other = cols * pitch;  // where the phase's activations are, and the next one's
    int queued = 0;                            // groups of copies since those of the next phase's activations began
    bool first = true;
    int s = my_k, round = 0;
    for (; round < rounds; ++round, tile += stride) {
        const bool active = tile < tiles;
        for (int p0 = 0; p0 < steps; p0 += a.phase_steps) {
            const int p1 = min(p0 + a.phase_steps, steps);
            if (a.phase_steps < steps) {
                if (!first) {
                    // the group with this phase's activations is the first of `queued`; with D or more it has been waited for
                    if (queued == 0) cp_async_commit();
                    if (queued < 2) cp_async_wait<0>();
                    else if (D == 3 && queued == 2) cp_async_wait<1>();
                    X::arrange(xs + other, pitch, nt, p1 - p0);
                    __syncthreads();  // in order for everyone, and everyone is done with the phase before
                    const int64_t was = buffer;
                    buffer = other;
                    other = was;
                }
                first = false;
                queued = 0;
                if (p1 < steps) X::copy(a, xs + other, pitch, t0, nt, p1, min(a.phase_steps, steps - p1));
                else if (round + 1 < rounds) X::copy(a, xs + other, pitch, t0, nt, 0, a.phase_steps);
            }
            if (!active) continue;
            const uint16_t* const xp = xs + buffer - (int64_t)p0 * kGvStep;
            for (; s < p1; s += kw) {
                queue_next();
                ++queued;
                cp_async_wait<D - 1>();
                __syncwarp();  // every lane's pieces of the step are in place
                Run<W> run[2];
                read_run<W>(run[0], ring + at, g, c);
                read_run<W>(run[1], ring + at, g + 8, c);
                if (16 * s + 16 > nb) {  // the end of a line: an ordinary exponent for the blocks that are not there (their activations are zero)
#pragma unroll
                    for (int b = 0; b < 4; ++b)
                        if (16 * s + run_block<W>(c, b) >= nb) {
                            const uint32_t mask = 0xFFu << (16 * (b & 1));
                            run[0].exps[b >> 1] = (run[0].exps[b >> 1] & ~mask) | (0x007F007Fu & mask);
                            run[1].exps[b >> 1] = (run[1].exps[b >> 1] & ~mask) | (0x007F007Fu & mask);
                        }
                }
                at = at + S::kStage == D * S::kStage ? 0 : at + S::kStage;
                run_step<W, NT>(run[0], run[1], xp + (int64_t)s * kGvStep, pitch, cols, lane, acc);
                __syncwarp();  // the next copies may overwrite the step
            }
        }
        if (!active) continue;
        s = my_k;
        // the shares of K, added in order; a warp's sums are [column][16 rows].  Two buffers: the sums of a tile are read before
        // anyone passes the barrier of the next, and only then overwritten.
        float* const mine = red + (S::kReds == 2 ? round & 1 : 0) * (S::kRed / 4) + warp * (8 * NT * 16);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                mine[(8 * n + 2 * c + (i & 1)) * 16 + g + 8 * (i >> 1)] = acc[n][i];
                acc[n][i] = 0.f;
            }
        if (kw == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(32 * kw) : "memory");
        const float* const from = mine - my_k * (8 * NT * 16);
        for (int i = my_k * 32 + lane; i < nt * 16; i += kw * 32) {
            const int t = i >> 4, r = i & 15;
            if (16 * tile + r >= a.n) continue;
            float v = 0.f;
#pragma unroll
            for (int part = 0; part < (X32 ? 3 : 1); ++part) {
                const int col = X32 ? 3 * t + (2 - part) : t;  // smallest part first
                for (int q = 0; q < kw; ++q) v += from[q * (8 * NT * 16) + col * 16 + r];
            }
            v *= 2.f;  // the operand was decoded halved
            const int64_t at = (int64_t)(t0 + t) * a.ldy + 16 * tile + r;
            if (a.y32) static_cast<float*>(a.y)[at] = v;
            else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
        }
        if (kw == 1) __syncwarp();
        else if (S::kReds == 1) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(32 * kw) : "memory");
    }
    cp_async_wait<0>();
}

template <int W, int NT, bool X32, int WARPS = gemv_warps(W, NT)>
static int launch_gemv(GemvArgs a, cudaStream_t st) {
    using S = GemvShape<W, NT, WARPS>;
    static PerDevice once;
    if (kernel_setup(once, mx_gemv_kernel<W, NT, X32, WARPS>, S::kThreads, kGvSmem) < 1) return BDR_ERR_CUDA;
    const int cols = (X32 ? 3 : 1) * std::min(a.tokens, a.tokens_per_pass);
    const int steps = (int)((a.k + kGvStep - 1) / kGvStep), sms = sm_count();
    const int64_t tiles = (a.n + 15) / 16;
    // the longest walk in steps, where a tile's join counts as a third of one and, if the activations come in phases, so does each phase's
    // barrier; putting a column's step in order, again for every round, takes about 1/500
    double best = 0;
    // steps whose activations fit, and of which two sets fit: one at least
    const int room = (kGvSmem - S::kXs) / cols, fit = S::fit(cols), half = (room / 2 - 64) / (2 * kGvStep);
    for (int kw = 1; kw <= S::kWarps && kw <= std::max(1, steps) && (steps <= fit || kw <= half); kw *= 2) {
        const int64_t rounds = ((tiles + sms - 1) / sms + S::kWarps / kw - 1) / (S::kWarps / kw);
        const double walk = (double)rounds * ((steps + kw - 1) / kw + 0.33 + (steps > fit ? 0.3 * steps / (half / kw * kw) + cols * steps / 500.0 : 0));
        if (kw == 1 || walk < best) { best = walk; a.kw = kw; }
    }
    a.phase_steps = std::max(1, steps);
    if (steps > fit) {  // phases of about the same length
        const int most = half / a.kw * a.kw, phases = (steps + most - 1) / most;
        a.phase_steps = ((steps + phases - 1) / phases + a.kw - 1) / a.kw * a.kw;
    }
    const size_t smem = S::kXs + (size_t)(steps > fit ? 2 : 1) * cols * (a.phase_steps * kGvStep * 2 + 64);
    const int64_t ctas = std::min<int64_t>(sms, tiles), stride = ctas * (S::kWarps / a.kw);
    while (1 << a.kw_log < a.kw) ++a.kw_log;
    a.rounds = (int)(tiles / stride);
    a.rest = (unsigned)std::min<int64_t>(tiles % stride, ctas);
    const dim3 grid((unsigned)ctas, (unsigned)((a.tokens + a.tokens_per_pass - 1) / a.tokens_per_pass));
    mx_gemv_kernel<W, NT, X32, WARPS><<<grid, S::kThreads, smem, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

template <int W, bool X32>
static int pick_columns(GemvArgs a, cudaStream_t st) {
    a.tokens_per_pass = X32 ? kGvMaxCols / 3 : kGvMaxCols;
    const int cols = (X32 ? 3 : 1) * std::min(a.tokens, a.tokens_per_pass);
    if (cols <= 8) return launch_gemv<W, 1, X32>(a, st);
    if (cols <= 16) {
        if constexpr (W == 3) {  // see gemv_warps
            const int64_t steps = (a.k + kGvStep - 1) / kGvStep;
            if (steps > GemvShape<3, 2, 16>::fit(cols) && steps <= GemvShape<3, 2, 8>::fit(cols) && (a.n + 15) / 16 <= 2 * sm_count())
                return launch_gemv<W, 2, X32, 8>(a, st);
        }
        return launch_gemv<W, 2, X32>(a, st);
    }
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
    const uintptr_t at = (uintptr_t)x | (T == 1 ? 0 : (uintptr_t)(ldx * xb));
    a.xalign = at % 16 == 0 ? 16 : (at % 4 == 0 ? 4 : 2);
    cudaStream_t st = (cudaStream_t)stream;
    switch (cfg_w->m) {
        case 2: return a.x32 ? pick_columns<3, true>(a, st) : pick_columns<3, false>(a, st);
        case 4: return a.x32 ? pick_columns<5, true>(a, st) : pick_columns<5, false>(a, st);
        case 7: return a.x32 ? pick_columns<8, true>(a, st) : pick_columns<8, false>(a, st);
    }
    return BDR_ERR_UNSUPPORTED;
}
