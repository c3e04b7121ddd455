// Packed MX blocks -> bf16 register fragments of the warp-level matrix instruction (m16n8k16), for the kernels whose
// operand is read once from memory and used for a few columns only (few-token products, attention of one new token).
//
// Those kernels are bound by the memory that holds the packed operand and by the instructions that decode it, not by the
// tensor core: a tcgen05 product would need the decoded operand in shared memory (a store and a load per value, and a
// 128-row tile of which a few columns are used), while a fragment of mma.sync takes the decoded pairs from the registers
// they were decoded in.  The reduction index of a product may be permuted freely as long as both operands agree, so a lane
// is given whole 16-element blocks (contiguous bytes of the packed line) instead of the scattered pairs of the
// instruction's own order.
//
// Decoding: an element is (-1)^s q 2^(F-127-tau-(m-1)), two neighbouring elements share tau.  With f = q / 2^m (q moved to
// the top of the seven bf16 mantissa bits, so 1 + f is 0x3F80 | bits) and S = 2^(F-127-tau), whose bf16 pattern is simply
// (F - tau) << 7,
//     fma(1 + f, S, -S) = f S = value / 2       exactly (f S is a multiple of 2^-133, a bf16 number for every F - tau >= 1),
// for every finite block without a special case at either end of the exponent range: nothing overflows because the value is
// halved, F = 255 makes S infinite and the result NaN, and F = 0 (zeros, and values below 2^-126, which count as zero here)
// makes S zero.  The kernels double their results once, in fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "bdr.h"

namespace bdr {
namespace frag {

// d += a b, a 16x16 (row), b 16x8 (column), bf16 operands, fp32 accumulators
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// the transpose of an 8x8 matrix of 16-bit values held as one row pair per lane
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}

// 32-bit words that hold one block of W-bit codes, and the words a reader of a block at a two-byte boundary fetches: the
// aligned words around it (16 or 10 or 6 bytes; never beyond the next four-byte boundary after the block)
template <int W> struct Block {
    static constexpr int kBytes = 2 * W;
    static constexpr int kWords = (kBytes + 3) / 4;
    uint32_t w[kWords];
};

template <int W>
__device__ __forceinline__ Block<W> load_block(const uint8_t* p) {
    Block<W> b;
    if constexpr (W == 8) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
        b.w[0] = v.x; b.w[1] = v.y; b.w[2] = v.z; b.w[3] = v.w;
    } else {
        const uint32_t* q = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)3);
#pragma unroll
        for (int i = 0; i < Block<W>::kWords; ++i) b.w[i] = __ldg(q + i);
    }
    return b;
}

// moves the stream of a block that was fetched from a two-byte boundary (off = its byte offset, or only the offset's low
// bits) down to bit 0
template <int W>
__device__ __forceinline__ void align_block(Block<W>& b, uint32_t off) {
    if constexpr (W != 8) {
        const uint32_t sh = (off & 2u) * 8u;
#pragma unroll
        for (int i = 0; i < Block<W>::kWords; ++i)
            b.w[i] = __funnelshift_r(b.w[i], i + 1 < Block<W>::kWords ? b.w[i + 1] : 0u, sh);
    }
}

// Pair j (elements 2j, 2j+1) of a stream of W-bit codes: the magnitudes at the top of the seven mantissa bits of each half,
// the sign bits where sign_of() expects them; other bits hold leftovers.
template <int W, int NW>
__device__ __forceinline__ uint32_t code_pair(const uint32_t (&s)[NW], int j) {
    if constexpr (W == 8) {
        return __byte_perm(s[j >> 1], 0u, (j & 1) ? 0x3322 : 0x1100);  // each code in both bytes of its half
    } else {
        const int bit = 2 * W * j, wi = bit >> 5, sh = bit & 31;
        uint32_t f = sh == 0 ? s[wi] : (sh + 2 * W > 32 ? __funnelshift_r(s[wi], s[wi + 1], sh) : s[wi] >> sh);
        f &= (1u << (2 * W)) - 1u;
        return f * ((1u << (8 - W)) + (1u << (24 - 2 * W)));  // the two copies do not overlap: 2 W <= 16 - W + W
    }
}

template <int W> struct PairMask {  // magnitude bits of a half: W - 1 bits ending at bit 6
    static constexpr uint32_t kMag = (0x7Fu & ~((1u << (8 - W)) - 1u)) * 0x00010001u;
};

// The eight pairs of a block as bf16x2 words, halved (see above).  `s` holds the stream from word/bit 0 of pair `first`.
template <int W, int NW>
__device__ __forceinline__ void decode_block(const uint32_t (&s)[NW], int first, uint32_t F, uint32_t micro, uint32_t (&y)[8]) {
    const uint32_t S0 = F * 0x00800080u;
    // zero and Inf/NaN blocks keep their scale whatever their microexponents say
    const uint32_t mb = (F - 1u) < 254u ? micro : 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t c = code_pair<W, NW>(s, first + j);
        const uint32_t S = S0 - (mb & (1u << j)) * (0x00800080u >> j);  // minus tau in both exponent fields
        uint32_t d;
        asm("{.reg .b32 n; neg.bf16x2 n, %2; fma.rn.bf16x2 %0, %1, %2, n;}" : "=r"(d) : "r"((c & PairMask<W>::kMag) | 0x3F803F80u), "r"(S));
        const uint32_t sign = W == 8 ? c : c << 8;
        y[j] = d ^ (sign & 0x80008000u);
    }
}

// A 24-bit fp32 value as the sum of three bf16 values (truncated eight bits at a time, so the sum is exact; parts below the
// bf16 range are dropped).  An infinity stays in the first part, a NaN becomes the quiet NaN.
__device__ __forceinline__ void split3(float x, uint16_t (&p)[3]) {
    const uint32_t u = __float_as_uint(x);
    if ((u & 0x7F800000u) == 0x7F800000u) {
        p[0] = (u & 0x007FFFFFu) ? 0x7FC0 : (uint16_t)(u >> 16);
        p[1] = p[2] = 0;
        return;
    }
    const float r1 = x - __uint_as_float(u & 0xFFFF0000u);
    const uint32_t u1 = __float_as_uint(r1);
    const float r2 = r1 - __uint_as_float(u1 & 0xFFFF0000u);
    p[0] = (uint16_t)(u >> 16);
    p[1] = (uint16_t)(u1 >> 16);
    p[2] = (uint16_t)(__float_as_uint(r2) >> 16);
}

__device__ __forceinline__ uint32_t pack2(uint16_t lo, uint16_t hi) { return (uint32_t)lo | ((uint32_t)hi << 16); }

}  // namespace frag

// What the kernels over packed lines accept of a configuration: the formats of Table II with ties to even (host).
inline int check_table2_config(const bdr_config_t* c) {
    if (!c) return BDR_ERR_NULL;
    if (c->scale_kind < 0 || c->scale_kind > BDR_SCALE_FP32_VSQ) return BDR_ERR_BAD_CONFIG;
    if (c->scale_kind != BDR_SCALE_POW2) return BDR_ERR_UNSUPPORTED;
    if (c->rounding != BDR_ROUND_NEAREST_EVEN && c->rounding != BDR_ROUND_NEAREST_AWAY) return BDR_ERR_BAD_CONFIG;
    if (c->d1 != 8 || c->k1 < 1 || c->k2 < 1 || c->k1 % c->k2 != 0 || c->d2 < 0 || c->d2 > 3 || c->m < 1 || c->m > 8)
        return BDR_ERR_BAD_CONFIG;
    if (c->k1 != 16 || c->k2 != 2 || c->d2 != 1 || (c->m != 2 && c->m != 4 && c->m != 7)) return BDR_ERR_UNSUPPORTED;
    return BDR_OK;
}

// Planes of lines of `len` elements in such a format (host).
inline int check_table2_planes(const bdr_config_t* c, const bdr_planes_t* p, int64_t len) {
    if (!p || !p->exps || !p->micro || !p->elems) return BDR_ERR_NULL;
    const int64_t nb = (len + 15) / 16;
    if (p->ld_exps < nb || p->ld_micro < nb || p->ld_elems < nb * 2 * (c->m + 1)) return BDR_ERR_SIZE;
    if (((uintptr_t)p->exps | (uintptr_t)p->micro | (uintptr_t)p->elems) % 16) return BDR_ERR_MISALIGNED;
    if ((p->ld_exps | p->ld_micro | p->ld_elems) % 16) return BDR_ERR_MISALIGNED;
    return BDR_OK;
}

}  // namespace bdr
