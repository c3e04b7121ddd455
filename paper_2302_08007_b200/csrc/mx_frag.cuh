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
// Decoding.  An element is (-1)^s q 2^(F-127-tau-(m-1)); two neighbouring elements share tau.  With f = q / 2^m, q at the top
// of the seven mantissa bits of a bf16 number, and S = 2^(F-127-tau), whose bf16 pattern is simply (F - tau) << 7, value / 2 is
// f S.  Two ways to it, both exact:
//   blocks with 96 <= F <= 159 (largest element between 2^-31 and 2^33): the mantissa bits alone, under the code's sign and a zero
//     exponent, are the subnormal +-f 2^-126; one multiplication by 2^(F-tau-33), a normal number, gives value / 2 * 2^-32
//     (the kernels put the factor 2^33 back in fp32);
//   any block: fma(1 + f, S, -S) = f S (1 + f is 0x3F80 | bits), then the sign.  Nothing overflows because the value is halved,
//     F = 255 makes S infinite and the result NaN, and F = 0 (zeros, and values below 2^-126, which count as zero here) makes
//     S zero.
// A warp takes the first way when all of its blocks allow it.
//
// The two halves of a decoded word are the same element of TWO blocks (two blocks of a line, or one block of two lines),
// not two neighbours: a sub-block's two elements then use the same scale word, which halves the work on microexponents, and
// a product over lines gets its pairs of lines without a transposition.  Codes of 3 and 5 bits are first spread to bytes with
// the sign in bit 7 (four codes at a time: 2 or 3 shifts and as many selections); a byte permutation then puts one code into
// both bytes of each half, where the sign is the half's sign bit and the magnitude is in the mantissa.  The integer/logic
// pipe, which issues at half the rate of the FMA pipe, is what decoding keeps busy: per word 2.5 of its instructions for
// MX9, 3.9 for MX6, 3.4 for MX4, of 4.0, 6.5 and 6.0 in all on the first way.
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

// 32-bit words that hold one block of W-bit codes.  A reader of a block at a two-byte boundary fetches the aligned words around
// it (16 or 10 or 6 bytes; never beyond the next four-byte boundary after the block).
template <int W> struct Block {
    static constexpr int kBytes = 2 * W;
    static constexpr int kWords = (kBytes + 3) / 4;
    uint32_t w[kWords];
};

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

// One three-input logic instruction.  Written out where it matters: the compiler splits (a & b) | c with two constants in two.
template <int TABLE>
__device__ __forceinline__ uint32_t lop3(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, %4;" : "=r"(d) : "r"(a), "r"(b), "r"(c), "n"(TABLE));
    return d;
}
constexpr int kAndOr = 0xEA, kXorAnd = 0x78, kSelect = 0xD8;  // (a & b) | c,  a ^ (b & c),  c ? b : a

// The exponents and microexponents of the two blocks of a word: S0 holds the scale of an unshifted sub-block per half, micro
// the eight shifts of each block in the low byte of its half.
struct Scales {
    uint32_t S0, micro;
};
constexpr float kFastFactor = 4294967296.f;  // 2^32: what the first way leaves out
// F2, micro2: one byte per half.
template <bool FAST>
__device__ __forceinline__ Scales make_scales(uint32_t F2, uint32_t micro2) {
    if constexpr (FAST) return {F2 * 0x80u + (94u << 7) * 0x00010001u, micro2};
    // zero blocks and Inf/NaN blocks (F = 0, 255) keep their scale whatever their microexponents say
    uint32_t one;
    asm("min.u16x2 %0, %1, %2;" : "=r"(one) : "r"((F2 + 0x00010001u) & 0x00FE00FEu), "r"(0x00010001u));
    return {F2 * 0x80u, micro2 & (one * 0xFFu)};
}
template <bool FAST>
__device__ __forceinline__ Scales make_scales(uint32_t Fa, uint32_t Fb, uint32_t ma, uint32_t mb) {
    return make_scales<FAST>(Fa + (Fb << 16), ma + (mb << 16));
}
// bytes 0 and 1 of a word, one per half
__device__ __forceinline__ uint32_t spread_bytes(uint32_t w) { return __byte_perm(w, 0u, 0x4140); }
// whether all four bytes of F4 are exponents of the first way: their top three bits are 011 or 100
__device__ __forceinline__ bool all_fast(uint32_t F4) { return (lop3<0x18>(F4, F4 << 1, F4 << 2) & 0x80808080u) == 0x80808080u; }

// The scale word of sub-block j: tau off the exponent field of each half.  Written as the multiply-add it is meant to be: a
// compiler would shift and subtract, on the pipe that is busy.
__device__ __forceinline__ uint32_t scale_word(const Scales& s, int j) {
    uint32_t S;
    asm("mad.lo.u32 %0, %1, %2, %3;" : "=r"(S) : "r"(s.micro & (0x00010001u << j)), "r"(0u - (0x80u >> j)), "r"(s.S0));
    return S;
}

// bits [bit, bit + 32) of a stream (a constant offset once loops are unrolled); bits beyond its words are zero or leftovers
template <int NW>
__device__ __forceinline__ uint32_t stream_bits(const uint32_t (&s)[NW], int bit) {
    const int wi = bit >> 5, sh = bit & 31;
    if (sh == 0) return s[wi];
    return wi + 1 < NW ? __funnelshift_r(s[wi], s[wi + 1 < NW ? wi + 1 : wi], sh) : s[wi] >> sh;
}

// Four codes of the block whose stream of W-bit codes starts at bit `at`, one per byte, the sign in bit 7 and the magnitude below it
// (other bits hold leftovers).  Word u of the four of a block: codes 4u .. 4u + 3; for 3-bit codes the even (u even) or odd (u odd)
// ones of codes 8 (u / 2) .. + 7.
template <int W, int NW>
__device__ __forceinline__ uint32_t code_bytes(const uint32_t (&s)[NW], int at, int u) {
    if constexpr (W == 8) {
        return s[(at >> 5) + u];
    } else if constexpr (W == 5) {
        const int bit = at + 20 * u;  // the first code goes to bits 3 .. 7
        const uint32_t v = bit % 32 < 3 ? stream_bits(s, bit) << 3 : stream_bits(s, bit - 3);
        const uint32_t w = lop3<kSelect>(v, v << 6, 0xFFFF0000u);
        return lop3<kSelect>(w, w << 3, 0xFF00FF00u);
    } else {
        static_assert(W == 3, "code widths of Table II");
        const int bit = at + 24 * (u >> 1);  // the first code goes to bits 1 .. 3
        const uint32_t v = bit % 32 < 1 ? stream_bits(s, bit) << 1 : stream_bits(s, bit - 1);
        const uint32_t w = lop3<kSelect>(v, v << 4, 0xFFFF0000u);
        const uint32_t x = lop3<kSelect>(w, w << 2, 0xFF00FF00u);
        const uint32_t y = lop3<kSelect>(x, x << 1, 0xF0F0F0F0u);
        return u & 1 ? y : y << 4;
    }
}

// Elements e of two blocks whose streams of W-bit codes start at bits a0 of `a` and b0 of `b`, halved (see above), with the
// scale word S of the element's sub-block.
template <int W, bool FAST, int NA, int NB>
__device__ __forceinline__ uint32_t decode_word(const uint32_t (&a)[NA], int a0, const uint32_t (&b)[NB], int b0, int e, uint32_t S) {
    constexpr uint32_t kMag = (0x7Fu & ~((1u << (8 - W)) - 1u)) * 0x00010001u;
    const int u = W == 3 ? 2 * (e >> 3) + (e & 1) : e >> 2, x = W == 3 ? (e >> 1) & 3 : e & 3;
    // the code in both bytes of its half
    const uint32_t c = __byte_perm(code_bytes<W>(a, a0, u), code_bytes<W>(b, b0, u), ((4 + x) << 12) | ((4 + x) << 8) | (x << 4) | x);
    uint32_t d;
    if constexpr (FAST) {
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(c & (kMag | 0x80008000u)), "r"(S));
        return d;
    }
    asm("{.reg .b32 n; neg.bf16x2 n, %2; fma.rn.bf16x2 %0, %1, %2, n;}" : "=r"(d) : "r"(lop3<kAndOr>(c, kMag, 0x3F803F80u)), "r"(S));
    return lop3<kXorAnd>(d, c, 0x80008000u);
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
