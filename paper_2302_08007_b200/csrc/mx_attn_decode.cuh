// Attention of one new token per sequence over a paged key-value cache in MX format (see mx_attn_decode in bdr.h).
//
// The cache is read once and every element of it is used for the few query heads that share it, so the bounds are the bytes
// of the cache and the instructions that decode them.  A warp owns one "unit", a key-value head with its query heads (small heads
// are merged until a unit fills 128 elements), and walks over tiles of 16 tokens.  It copies its tiles' packed bytes into a ring of
// its own in shared memory with asynchronous 16- and 8-byte copies, a lane per piece, a tile or two ahead: no registers are
// tied up by bytes in flight, fetching costs 45 instructions a tile (and 65 for the slots) where loads into registers cost 230,
// and nothing but the warp itself has to be waited for.  (One bulk copy per token and plane by a producer warp, tried instead, was twice
// as slow as loads into registers: the pieces, 64 to 640 bytes, are too small for the bulk-copy unit.)
//   scores    S^T[16 tokens, 8 columns] = K[16, d] Q^T: the key blocks are decoded straight into the A fragment (lane (g, c)
//             decodes whole blocks of tokens g and g + 8); Q waits in shared memory in the order of the B fragment;
//   softmax   with a running reference per column instead of the running maximum: it is raised only when a score passes it
//             by kAtSlack (in powers of two), so most tiles need a vote and no reduction over lanes;
//   output    O^T[d, 8 columns] += V^T P^T: V is decoded like K (lane (g, c): block g of four tokens, two tokens to a word as the A
//             fragment wants them), and P^T is the 8x8 transpose of the score fragment.
//
// Work is split over the length of the cache: the tiles of all sequences form one long line that is cut into equal parts,
// one per worker CTA, whatever the individual lengths are (each worker finds its part from `lengths`).  Where a group has
// fewer units than the CTA has warps, several sets of warps take turns with the tiles and are joined in shared memory.  A part
// that covers a sequence's whole range writes the result; other parts leave their sums and references in the workspace, where
// a second kernel joins them in order.
//
// Measured (32 query heads on 8 key-value heads of 128 elements, bf16, both kernels, the cache not in the L2): 64 sequences of 2048 to
// 8192 tokens, MX6, 190 us = 2.65 TB/s of cache; 16 sequences of 500 to 4096, MX9, 34.3 us = 2.5 TB/s; one of 777, MX9, 12 us; 64 query
// heads, one sequence of 131072, MX4, 78 us = 1.7 TB/s.  With 32-bit queries 64 sequences of 2048 to 8096, MX6, take 247 us.  A tile of
// 16 x 128 keys and values takes 790 instructions in MX6, 730 in MX4 and 670 in MX9, 60 % of them the decoding; the integer/logic pipe
// is busy 62 to 65 % of the time and the issue slots 68 to 70 % (MX9: 49 %, waiting for copies as well).  Short calls are two
// launches and a chain of dependent reads: lengths, page, bytes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "bdr_device.cuh"
#include "bdr_host.h"
#include "mx_frag.cuh"

namespace bdr {

constexpr int kAtSmemBytes = 227 * 1024;
constexpr float kAtLift = 32.f;      // weights carry the factor 2^32 that the first way of decoding the values leaves out
constexpr float kAtSlack = 8.f;      // a weight stays below 2^8 times that
constexpr float kAtNone = -3.0e38f;  // the reference before the first score: below every finite score, and finite itself

struct AttnArgs {
    bdr_planes_t k, v;
    const void* q;
    void* out;
    float* lse;
    const int32_t *table, *lengths;
    float* part_o;          // [worker][2][n_q][d]
    float2* part_ml;        // [worker][2][n_q]: reference (base 2) and sum of weights
    int64_t ldq, ldo, ld_table;
    int n_seqs, n_q, n_kv, group, d, nb;   // group: query heads per key-value head; nb: blocks per head
    int merge, per_pass, passes, n_units;  // key-value heads of a unit, query heads per pass of each, passes, units
    int hw, tw, workers;                   // units of a group (one per warp), sets of warps, worker CTAs per group
    int n_pages, max_pages, cap, window;   // cap = max_pages * page_size
    int q_vec, o_vec;                      // two query elements may be read at once; results may be written 16 bytes at a time
    FastDiv page, by_workers;
    int hw_log, inv_pass;                  // log2 of hw; 65536 / per_pass rounded up
    float scale2, scale2_fast;             // 2 scale log2(e): the keys are decoded halved (and on the first way scaled)
    int* status;
};

// Tiles of 16 tokens that sequence b's positions touch.
struct SeqRange {
    int start, end, first, count;
};
__device__ __forceinline__ SeqRange seq_range(const AttnArgs& a, int b) {
    SeqRange r;
    const int len = min(__ldg(a.lengths + b), a.cap + 1);  // a position beyond the table's pages poisons the result
    r.end = max(len, 0);
    r.start = a.window > 0 ? max(0, r.end - a.window) : 0;
    r.first = r.start / 16;
    r.count = r.end > r.start ? (r.end + 15) / 16 - r.first : 0;
    return r;
}

// Tiles of all sequences together, and of those before sequence `b` (called by whole warps).  Up to 32 sequences, a lane each,
// take one round of loads.
struct TileCounts {
    int64_t total, prefix;
};
__device__ __forceinline__ int64_t inclusive_scan(int64_t n, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xFFFFFFFFu, n, o);
        if (lane >= o) n += v;
    }
    return n;
}
__device__ __forceinline__ TileCounts count_tiles(const AttnArgs& a, int lane, int b) {
    TileCounts c = {0, 0};
    for (int i = lane; i < a.n_seqs; i += 32) {
        const int n = seq_range(a, i).count;
        c.total += n;
        if (i < b) c.prefix += n;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        c.total += __shfl_xor_sync(0xFFFFFFFFu, c.total, o);
        c.prefix += __shfl_xor_sync(0xFFFFFFFFu, c.prefix, o);
    }
    return c;
}

// The line of all tiles in equal parts, one per worker: the first `more` have one tile more than the others' `each`.
struct Split {
    int64_t each, more;
    __device__ __forceinline__ Split(const AttnArgs& a, int64_t total) {
        each = total < (1ll << 31) ? (int64_t)fastdiv((uint32_t)total, a.by_workers) : total / a.workers;
        more = total - each * a.workers;
    }
    __device__ __forceinline__ int64_t begin(int w) const { return each * w + min((int64_t)w, more); }
    // the worker that has a tile of the line
    __device__ __forceinline__ int holder(int64_t tile) const {
        const int64_t bound = more * (each + 1), at = tile < bound ? tile : tile - bound, n = tile < bound ? each + 1 : each;
        const int64_t w = at < (1ll << 31) && n < (1ll << 31) ? (int64_t)((uint32_t)at / (uint32_t)n) : at / n;
        return (int)(tile < bound ? w : more + w);
    }
};

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

// MAXB: blocks of a unit (8 or 16); NT: groups of eight columns (query heads); F32: 32-bit queries and results; FULL: every
// unit has all MAXB blocks, so a lane's key blocks are whole aligned words.
template <int MAXB, int NT, bool F32>
struct AttnShape {
    // As many as the registers allow: at 128 a thread (16 warps) most kernels spill a little, 8 to 52 bytes with bf16 queries and 20 to 92
    // with 32-bit ones.
    static constexpr int kWarps = MAXB == 8 && NT == 1 ? 16 : 8;
    static constexpr int kThreads = 32 * kWarps;
    static constexpr int kKeyBlocks = MAXB / 4, kValBlocks = MAXB / 8;  // per lane and token
    static constexpr int kParts = F32 ? 3 : 1;
    // bf16 parts of a softmax weight.  One, rounded to eight bits, took the error of a bf16 result from 1.7e-3 (the result's own rounding)
    // to 2.3e-3 over long sequences; the second costs 1 to 4 % (64 sequences of 2048 to 8096, MX6: 187 us, with one 184).
    static constexpr int kWeightParts = F32 ? 3 : 2;
    static constexpr int kMaxUnits = F32 ? 4 : 8;  // units of a group: their queries share the memory with the rings
    static constexpr int kQBytes = kParts * MAXB * NT * 32 * 8;          // per unit
    static constexpr int kSums = kValBlocks * 8 * NT * 4 + NT * 4;       // a lane's sums, references and weights
    static constexpr int kJoinBytes = kSums * 32 * 4;                    // what a warp hands over (in its own ring)
};

// A tile in shared memory: 16 rows of key codes, 16 of value codes, 16 of scales (key exponents, key microexponents, value
// exponents, value microexponents).  Pitches are odd multiples of 16 bytes, so that eight rows at one offset start in eight
// different groups of banks.  Where units do not start at multiples of the copies' sizes, rows hold the words around them.
template <int WK, int WV, int MAXB, bool FULL>
struct AttnTile {
    static constexpr int code_pitch(int w) {
        const int len = FULL || w == 8 ? MAXB * 2 * w : ((MAXB - 1) * 2 * w + 14 + 15) / 16 * 16;
        return len % 32 == 16 ? len : len + 16;
    }
    static constexpr int kPitchK = code_pitch(WK), kPitchV = code_pitch(WV);
    static constexpr int kScale = FULL ? MAXB : MAXB == 8 ? 16 : 24;  // bytes of a plane's scales in a row
    static constexpr int kPitchX = 4 * kScale % 32 == 16 ? 4 * kScale : 4 * kScale + 16;
    static constexpr int kAtV = 16 * kPitchK, kAtX = kAtV + 16 * kPitchV, kBytes = kAtX + 16 * kPitchX;
    // tiles in a warp's ring: what 227 KB hold, two at least, three at most
    static constexpr int kStages = MAXB == 8 && 16 * 3 * kBytes + 4 * AttnShape<8, 1, true>::kQBytes <= kAtSmemBytes ? 3 : 2;
};

// a warp's part of shared memory: its ring, or the sums it hands over
template <int WK, int WV, int MAXB, int NT, bool F32, bool FULL>
__host__ __device__ constexpr int attn_ring_bytes() {
    using L = AttnTile<WK, WV, MAXB, FULL>;
    return L::kStages * L::kBytes > AttnShape<MAXB, NT, F32>::kJoinBytes ? L::kStages * L::kBytes : AttnShape<MAXB, NT, F32>::kJoinBytes;
}

// The bytes of a token's line that a unit needs, rounded out to aligned pieces.
struct RowSpan {
    int from, len, skew;  // first byte, bytes, where the unit's first block lies in them
};
template <int ALIGN>
__device__ __forceinline__ RowSpan row_span(int block0, int blocks, int block_bytes) {
    const int at = block0 * block_bytes;
    RowSpan s;
    s.from = at & ~(ALIGN - 1);
    s.skew = at - s.from;
    s.len = (s.skew + blocks * block_bytes + ALIGN - 1) & ~(ALIGN - 1);
    return s;
}

// one block of W-bit codes from shared memory, at any two-byte boundary
template <int W>
__device__ __forceinline__ frag::Block<W> shared_block(const uint8_t* base, int off) {
    frag::Block<W> b;
    if constexpr (W == 8) {
        const uint4 v = *reinterpret_cast<const uint4*>(base + off);
        b.w[0] = v.x; b.w[1] = v.y; b.w[2] = v.z; b.w[3] = v.w;
    } else {
        const uint32_t* q = reinterpret_cast<const uint32_t*>(base + (off & ~3));
#pragma unroll
        for (int i = 0; i < frag::Block<W>::kWords; ++i) b.w[i] = q[i];
    }
    return b;
}

// A worker's part of the line of tiles, sequence by sequence.
struct Segments {
    int64_t u, u_end, prefix;
    int b;
    SeqRange r;
    int t0, t1;
    bool known;  // r is sequence b's
    // finds the part of worker w (called by whole warps)
    __device__ __forceinline__ void begin(const AttnArgs& a, int w, int lane) {
        if (a.n_seqs <= 32) {
            r = {0, 0, 0, 0};
            if (lane < a.n_seqs) r = seq_range(a, lane);
            const int64_t incl = inclusive_scan(r.count, lane), total = __shfl_sync(0xFFFFFFFFu, incl, 31);
            const Split split(a, total);
            u = split.begin(w);
            u_end = split.begin(w + 1);
            const unsigned hit = __ballot_sync(0xFFFFFFFFu, incl > u);
            b = hit ? __ffs(hit) - 1 : 0;
            prefix = __shfl_sync(0xFFFFFFFFu, incl - r.count, b);
            r.start = __shfl_sync(0xFFFFFFFFu, r.start, b);
            r.end = __shfl_sync(0xFFFFFFFFu, r.end, b);
            r.first = __shfl_sync(0xFFFFFFFFu, r.first, b);
            r.count = __shfl_sync(0xFFFFFFFFu, r.count, b);
            known = true;
            return;
        }
        const Split split(a, count_tiles(a, lane, 0).total);
        u = split.begin(w);
        u_end = split.begin(w + 1);
        known = false;
        prefix = 0;
        if (u >= u_end) return;
        for (b = 0;; b += 32) {  // 32 sequences at a time up to the one that holds tile u
            const int64_t n = b + lane < a.n_seqs ? seq_range(a, b + lane).count : 0, incl = inclusive_scan(n, lane);
            const unsigned hit = __ballot_sync(0xFFFFFFFFu, prefix + incl > u);
            if (hit) {
                const int at = __ffs(hit) - 1;
                prefix += __shfl_sync(0xFFFFFFFFu, incl - n, at);
                b += at;
                return;
            }
            prefix += __shfl_sync(0xFFFFFFFFu, incl, 31);
        }
    }
    // false when the part is done; else tiles t0 .. t1 of sequence b (counted from the first that its range touches)
    __device__ __forceinline__ bool next(const AttnArgs& a) {
        if (u >= u_end) return false;
        if (!known) r = seq_range(a, b);
        while (r.count == 0) r = seq_range(a, ++b);
        known = true;
        t0 = (int)(u - prefix);
        t1 = (int)min((int64_t)r.count, u_end - prefix);
        return true;
    }
    __device__ __forceinline__ void advance() {
        u = prefix + t1;
        if (t1 == r.count) { prefix += r.count; ++b; known = false; }
    }
};

template <int WK, int WV, int MAXB, int NT, bool F32, bool FULL>
__global__ void __launch_bounds__((AttnShape<MAXB, NT, F32>::kThreads), 1) mx_attn_decode_kernel(const AttnArgs a) {
    cudaTriggerProgrammaticLaunchCompletion();  // the joining kernel may take its place as soon as there is room
    using S = AttnShape<MAXB, NT, F32>;
    using L = AttnTile<WK, WV, MAXB, FULL>;
    using T = typename std::conditional<F32, float, __nv_bfloat16>::type;
    constexpr int KB = S::kKeyBlocks, VB = S::kValBlocks, PARTS = S::kParts, WPARTS = S::kWeightParts, D = L::kStages;
    // The weights' factor 2^32 is part of the exponent's argument, which costs its last bits; 32-bit queries have it multiplied to the
    // weights instead (with the partial sums of scores, below, that took their error from 9e-7 to 2.4e-7 of the result).
    constexpr float kLift = F32 ? 0.f : kAtLift;
    constexpr int kRing = attn_ring_bytes<WK, WV, MAXB, NT, F32, FULL>();
    extern __shared__ __align__(128) uint8_t smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Segments seg;
    seg.begin(a, blockIdx.x, lane);
    if (seg.u >= seg.u_end) return;  // uniform for the CTA

    const int g = lane >> 2, c = lane & 3, hw = warp & (a.hw - 1), tw = warp >> a.hw_log;
    const int unit = blockIdx.y * a.hw + hw, mk = unit / a.passes, pass = unit - mk * a.passes, kv0 = mk * a.merge;
    const int kv_n = min(a.merge, a.n_kv - kv0), blocks = kv_n * a.nb, block0 = kv0 * a.nb;
    uint4* const qs = reinterpret_cast<uint4*>(smem + hw * S::kQBytes);
    uint8_t* const rings = smem + a.hw * S::kQBytes;
    uint8_t* const ring = rings + warp * kRing;
    // the bytes of a token's line that the unit needs, rounded out to the pieces that are copied
    const RowSpan span_k = row_span<16>(block0, blocks, 2 * WK), span_v = row_span<16>(block0, blocks, 2 * WV), span_x = row_span<8>(block0, blocks, 1);
    // byte offsets of this lane's rows within a tile; a block that the unit does not have is read as its first and ignored
    const int off_k = g * L::kPitchK + (FULL ? c * KB * (2 * WK) : span_k.skew);
    const int off_kx = L::kAtX + g * L::kPitchX + (FULL ? c * KB : span_x.skew);
    const int val_block = FULL || g * VB < blocks ? g * VB : 0;
    const int off_v = L::kAtV + 2 * c * L::kPitchV + span_v.skew + val_block * (2 * WV);
    const int off_vx = L::kAtX + 2 * c * L::kPitchX + 2 * L::kScale + span_x.skew + val_block;

    // Where this lane's pieces come from: piece `lane % pieces` of every row's codes, and the exponents (lanes 0 .. 15) or
    // microexponents (lanes 16 .. 31) of token lane % 16.  Kept in registers: the compiler would rather rebuild them per tile.
    constexpr int kPiecesK = WK * MAXB / 8, kPiecesV = WV * MAXB / 8;  // 16-byte pieces of a full unit's row
    const bool micro = lane >= 16;
    const uint8_t* src_k = a.k.elems + span_k.from + (FULL ? lane % kPiecesK * 16 : 0);
    const uint8_t* src_v = a.v.elems + span_v.from + (FULL ? lane % kPiecesV * 16 : 0);
    const uint8_t* src_kx = (micro ? a.k.micro : a.k.exps) + span_x.from;
    const uint8_t* src_vx = (micro ? a.v.micro : a.v.exps) + span_x.from;
    uint32_t ld_kx = (uint32_t)(micro ? a.k.ld_micro : a.k.ld_exps), ld_vx = (uint32_t)(micro ? a.v.ld_micro : a.v.ld_exps);
    asm volatile("" : "+l"(src_k), "+l"(src_v), "+l"(src_kx), "+l"(src_vx), "+r"(ld_kx), "+r"(ld_vx));
    // Queues the copies of a tile whose token i has the slot that lane i (and i + 16) holds; ALL: every token is there, else
    // tokens with negative slots are left out.
    auto fetch = [&](uint8_t* to, int slot, auto all) {
        constexpr bool ALL = decltype(all)::value;
        auto rows = [&](auto pieces_, const uint8_t* src, uint32_t ld, int len, uint8_t* dst, auto pitch_) {
            constexpr int kPitch = decltype(pitch_)::value;
            if constexpr (FULL) {
                constexpr int kPieces = decltype(pieces_)::value, kRows = 32 / kPieces;  // rows to an instruction
                const int r0 = lane / kPieces;
                uint8_t* const d = dst + r0 * kPitch + 16 * (lane - r0 * kPieces);
#pragma unroll
                for (int r = 0; r < 16; r += kRows) {
                    const int from = __shfl_sync(0xFFFFFFFFu, slot, (r + r0) & 15);
                    if ((32 % kPieces == 0 || r0 < kRows) && (r + kRows <= 16 || r + r0 < 16) && (ALL || from >= 0))
                        cp_async16(d + r * kPitch, src + (uint64_t)(uint32_t)from * ld);
                }
            } else {
                const int pieces = len / 16, inv = 65536 / pieces + 1;
                for (int i = lane; i < (16 * pieces + 31) / 32 * 32; i += 32) {
                    const int r = (i * inv) >> 16, piece = i - r * pieces;
                    const int from = __shfl_sync(0xFFFFFFFFu, slot, r & 15);
                    if (r < 16 && (ALL || from >= 0)) cp_async16(dst + r * kPitch + 16 * piece, src + (uint64_t)(uint32_t)from * ld + 16 * piece);
                }
            }
        };
        rows(std::integral_constant<int, kPiecesK>{}, src_k, (uint32_t)a.k.ld_elems, span_k.len, to, std::integral_constant<int, L::kPitchK>{});
        rows(std::integral_constant<int, kPiecesV>{}, src_v, (uint32_t)a.v.ld_elems, span_v.len, to + L::kAtV, std::integral_constant<int, L::kPitchV>{});
        if (ALL || slot >= 0) {
            const uint8_t* k = src_kx + (uint64_t)(uint32_t)slot * ld_kx;
            const uint8_t* v = src_vx + (uint64_t)(uint32_t)slot * ld_vx;
            uint8_t* x = to + L::kAtX + (lane & 15) * L::kPitchX + (micro ? L::kScale : 0);
#pragma unroll
            for (int i = 0; i < L::kScale; i += 8)
                if (FULL || i < span_x.len) {
                    cp_async8(x + i, k + i);
                    cp_async8(x + 2 * L::kScale + i, v + i);
                }
        }
    };

    // query head of a column, or -1; the key-value head of the unit that it belongs to (below 16 columns the product is exact)
    auto kv_of = [&](int col) { return (col * a.inv_pass) >> 16; };
    auto head_of = [&](int col) {
        const int f = kv_of(col), i = pass * a.per_pass + (col - f * a.per_pass);
        return f < kv_n && i < a.group ? (kv0 + f) * a.group + i : -1;
    };
    auto sync_all = [&] {  // where one set of warps works alone there is nobody to wait for but the queries' loader, the warp itself
        if (a.tw > 1) __syncthreads();
        else __syncwarp();
    };

    bool first_segment = true;
    for (; seg.next(a); seg.advance(), first_segment = false) {
        const int b = seg.b;
        // ---- queries into shared memory: [part][pair of steps][column group][lane].  Step 8 x + j of a lane holds elements 2j and 2j + 1 of
        // blocks 2x and 2x + 1 of its own: {2x: 2j, 2x+1: 2j}, {2x: 2j+1, 2x+1: 2j+1}.
        {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int col = 8 * n + g, head = head_of(col), f = kv_of(col);
                const T* q = static_cast<const T*>(a.q) + (int64_t)b * a.ldq + (int64_t)max(head, 0) * a.d;
#pragma unroll
                for (int x = 0; x < KB / 2; ++x) {
                    const int at0 = (c * KB + 2 * x) * 16 - f * a.d, at1 = at0 + 16;  // elements of the head
                    const bool in0 = head >= 0 && at0 >= 0 && at0 < a.d, in1 = head >= 0 && at1 >= 0 && at1 < a.d;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if ((j & (a.tw - 1)) != tw) continue;  // the unit's sets of warps share the work
                        uint16_t p[4][3];
                        if constexpr (F32) {
                            float2 u = make_float2(0.f, 0.f), v = u;
                            if (in0) u = a.q_vec ? __ldg(reinterpret_cast<const float2*>(q + at0 + 2 * j)) : make_float2(q[at0 + 2 * j], q[at0 + 2 * j + 1]);
                            if (in1) v = a.q_vec ? __ldg(reinterpret_cast<const float2*>(q + at1 + 2 * j)) : make_float2(q[at1 + 2 * j], q[at1 + 2 * j + 1]);
                            frag::split3(u.x, p[0]);
                            frag::split3(v.x, p[1]);
                            frag::split3(u.y, p[2]);
                            frag::split3(v.y, p[3]);
                        } else {
                            const uint16_t* h = reinterpret_cast<const uint16_t*>(q);
                            uint32_t u = 0, v = 0;
                            if (in0) u = a.q_vec ? __ldg(reinterpret_cast<const uint32_t*>(h + at0 + 2 * j)) : frag::pack2(h[at0 + 2 * j], h[at0 + 2 * j + 1]);
                            if (in1) v = a.q_vec ? __ldg(reinterpret_cast<const uint32_t*>(h + at1 + 2 * j)) : frag::pack2(h[at1 + 2 * j], h[at1 + 2 * j + 1]);
                            p[0][0] = (uint16_t)u; p[1][0] = (uint16_t)v; p[2][0] = (uint16_t)(u >> 16); p[3][0] = (uint16_t)(v >> 16);
                        }
#pragma unroll
                        for (int part = 0; part < PARTS; ++part)
                            reinterpret_cast<uint2*>(qs + ((part * MAXB / 2 + 4 * x + j / 2) * NT + n) * 32 + lane)[j & 1] =
                                make_uint2(frag::pack2(p[0][part], p[1][part]), frag::pack2(p[2][part], p[3][part]));
                    }
                }
            }
        }
        sync_all();

        float o[VB * 8][NT][4], ref[NT][2], sum[NT][2];
#pragma unroll
        for (int i = 0; i < VB * 8; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][n][e] = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) { ref[n][0] = ref[n][1] = kAtNone; sum[n][0] = sum[n][1] = 0.f; }

        // slot of token 16 tile + lane % 16: -1 outside the range, -2 for a page that does not exist
        const int tile_end = seg.r.first + seg.t1;
        const int32_t* const table = a.table + (int64_t)b * a.ld_table;
        auto slot_of = [&](int t) {
            const int tok = 16 * t + (lane & 15);
            const int pg = (int)fastdiv((uint32_t)tok, a.page), known = min(pg, max(a.max_pages - 1, 0));
            const int id = __ldg(table + known);
            int slot = id * (int)a.page.d + (tok - pg * (int)a.page.d);
            slot = pg < a.max_pages && (uint32_t)id < (uint32_t)a.n_pages ? slot : -2;
            slot = t < tile_end && tok >= seg.r.start && tok < seg.r.end ? slot : -1;
            return slot;
        };
        // tokens present (bits 0 .. 15) and tokens of bad pages (16 .. 31)
        auto marks = [&](int slot) {
            const uint32_t present = __ballot_sync(0xFFFFFFFFu, slot >= 0) & 0xFFFFu;
            return present | (present == 0xFFFFu ? 0u : __ballot_sync(0xFFFFFFFFu, slot == -2) << 16);
        };
        int tile = seg.r.first + seg.t0 + tw, slot = slot_of(tile), to = 0;
        uint32_t held[D];  // marks of the tiles in the ring, the present one first
#pragma unroll
        for (int i = 0; i + 1 < D; ++i) {
            fetch(ring + to, slot, std::false_type{});
            cp_async_commit();
            held[i] = marks(slot);
            slot = slot_of(tile + (i + 1) * a.tw);
            to += L::kBytes;
        }
        int at = 0;
        for (; tile < tile_end; tile += a.tw) {
            held[D - 1] = marks(slot);
            if (held[D - 1] == 0xFFFFu) fetch(ring + to, slot, std::true_type{});
            else if (tile + (D - 1) * a.tw < tile_end) fetch(ring + to, slot, std::false_type{});
            cp_async_commit();
            slot = slot_of(tile + D * a.tw);
            to = to + L::kBytes == D * L::kBytes ? 0 : to + L::kBytes;
            cp_async_wait<D - 1>();
            __syncwarp();  // every lane's pieces of the tile are in place
            const uint8_t* const st = ring + at;
            const uint32_t here = held[0];
            at = at + L::kBytes == D * L::kBytes ? 0 : at + L::kBytes;
#pragma unroll
            for (int i = 0; i + 1 < D; ++i) held[i] = held[i + 1];
            // ---- scores
            float s[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
            constexpr int BW = frag::Block<WK>::kWords;
            uint32_t kr[2][FULL ? KB * WK / 2 : KB * BW], kf[2], km[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint8_t* e = st + off_k + 8 * i * L::kPitchK;
                const uint8_t* x = st + off_kx + 8 * i * L::kPitchX;
                if constexpr (FULL) {
                    if constexpr (KB == 2) { kf[i] = *reinterpret_cast<const uint16_t*>(x); km[i] = *reinterpret_cast<const uint16_t*>(x + L::kScale); }
                    else { kf[i] = *reinterpret_cast<const uint32_t*>(x); km[i] = *reinterpret_cast<const uint32_t*>(x + L::kScale); }
                    if constexpr (WK == 8) {
#pragma unroll
                        for (int w = 0; w < KB; ++w) {
                            const uint4 v = reinterpret_cast<const uint4*>(e)[w];
                            kr[i][4 * w] = v.x; kr[i][4 * w + 1] = v.y; kr[i][4 * w + 2] = v.z; kr[i][4 * w + 3] = v.w;
                        }
                    } else {
#pragma unroll
                        for (int w = 0; w < KB * WK / 2; ++w) kr[i][w] = reinterpret_cast<const uint32_t*>(e)[w];
                    }
                } else {
                    kf[i] = 0x7F7F7F7Fu;  // absent blocks: an ordinary exponent, zero queries
                    km[i] = 0;
#pragma unroll
                    for (int y = 0; y < KB; ++y) {
                        const int blk = c * KB + y < blocks ? c * KB + y : 0;
                        const int off = off_k + 8 * i * L::kPitchK + blk * (2 * WK);
                        frag::Block<WK> v = shared_block<WK>(st, off);
                        frag::align_block(v, (uint32_t)off);
#pragma unroll
                        for (int w = 0; w < BW; ++w) kr[i][y * BW + w] = v.w[w];
                        if (c * KB + y < blocks) {
                            kf[i] ^= (uint32_t)(0x7F ^ x[blk]) << (8 * y);
                            km[i] |= (uint32_t)x[blk + L::kScale] << (8 * y);
                        }
                    }
                }
            }
            uint32_t vf[4], vm[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = (i & 1) + 8 * (i >> 1);  // token 2c + r
                const uint8_t* x = st + off_vx + r * L::kPitchX;
                if constexpr (FULL && VB == 1) {
                    vf[i] = x[0];
                    vm[i] = x[L::kScale];
                } else {
                    vf[i] = VB == 1 ? 0x7Fu : 0x7F7Fu;
                    vm[i] = 0;
#pragma unroll
                    for (int y = 0; y < VB; ++y)
                        if (FULL || g * VB + y < blocks) {
                            vf[i] ^= (uint32_t)(0x7F ^ x[y]) << (8 * y);
                            vm[i] |= (uint32_t)x[y + L::kScale] << (8 * y);
                        }
                }
            }
            bool ordinary;
            if constexpr (VB == 1) ordinary = frag::all_fast((kf[0] & 0xFFFFu) + (kf[1] << 16)) && frag::all_fast(vf[0] + (vf[1] << 8) + (vf[2] << 16) + (vf[3] << 24));
            else ordinary = frag::all_fast(kf[0]) && frag::all_fast(kf[1]) && frag::all_fast(vf[0] + (vf[1] << 16)) && frag::all_fast(vf[2] + (vf[3] << 16));
            const bool fast = __all_sync(0xFFFFFFFFu, ordinary);
            auto scores = [&](auto way) {
                constexpr bool FAST = decltype(way)::value;
#pragma unroll
                for (int x = 0; x < KB / 2; ++x) {
                    frag::Scales sc[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        sc[i] = frag::make_scales<FAST>(frag::spread_bytes(kf[i] >> (16 * x)), frag::spread_bytes(km[i] >> (16 * x)));
                    constexpr int kBits = FULL ? 16 * WK : 32 * BW;  // from one block's stream to the next's
                    const int b0 = 2 * x * kBits, b1 = b0 + kBits;
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        uint32_t y[2][4];  // rows g and g + 8, elements 2j .. 2j + 3
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                y[i][e] = frag::decode_word<WK, FAST>(kr[i], b0, kr[i], b1, 2 * j + e, frag::scale_word(sc[i], j + (e >> 1)));
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            float d[4] = {0.f, 0.f, 0.f, 0.f};  // 32-bit queries: short sums in the tensor core, as for the output below
#pragma unroll
                            for (int part = PARTS - 1; part >= 0; --part) {
                                const uint4 qv = qs[((part * MAXB / 2 + 4 * x + j / 2) * NT + n) * 32 + lane];
                                frag::mma_bf16(F32 ? d : s[n], y[0][0], y[1][0], y[0][1], y[1][1], qv.x, qv.y);
                                frag::mma_bf16(F32 ? d : s[n], y[0][2], y[1][2], y[0][3], y[1][3], qv.z, qv.w);
                            }
                            if constexpr (F32) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) s[n][e] += d[e];
                            }
                        }
                    }
                }
            };
            if (fast) {
                scores(std::true_type{});
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[n][e] *= a.scale2_fast;
            } else {
                // Merged heads share the reduction: a NaN block of one head must not reach the others' columns through their zero
                // queries, so it is decoded as zeros and its head's scores are made NaN below.
                uint32_t spoilt[2] = {0, 0};  // per row: the unit's heads with such a block
                if (a.merge > 1) {
                    bool any = false;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int x = 0; x < KB; ++x) any |= ((kf[i] >> (8 * x)) & 0xFFu) == 255u;
                    if (__any_sync(0xFFFFFFFFu, any)) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
#pragma unroll
                            for (int x = 0; x < KB; ++x)
                                if (((kf[i] >> (8 * x)) & 0xFFu) == 255u) {
                                    spoilt[i] |= 1u << ((c * KB + x) / a.nb);
                                    kf[i] &= ~(0xFFu << (8 * x));
                                }
                            spoilt[i] |= __shfl_xor_sync(0xFFFFFFFFu, spoilt[i], 1);
                            spoilt[i] |= __shfl_xor_sync(0xFFFFFFFFu, spoilt[i], 2);
                        }
                    }
                }
                scores(std::false_type{});
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[n][e] *= a.scale2;
                if (spoilt[0] | spoilt[1]) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (spoilt[e >> 1] >> kv_of(8 * n + 2 * c + (e & 1)) & 1u) s[n][e] = __uint_as_float(0x7FC00000u);
                }
            }
            // ---- the tile's values
            frag::Block<WV> vb[4][VB];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int y = 0; y < VB; ++y) {
                    const int off = off_v + ((i & 1) + 8 * (i >> 1)) * L::kPitchV + (FULL || g * VB + y < blocks ? y : 0) * (2 * WV);
                    vb[i][y] = shared_block<WV>(st, off);
                    frag::align_block(vb[i][y], (uint32_t)off);
                }
            if (here != 0xFFFFu) {  // a tile at an end of the range, or with a page that does not exist
                if (here >> 16 && lane == 0) atomicCAS(a.status, 0, (int)BDR_ERR_SIZE);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int tok = g + 8 * i;
                    const bool bad = here >> (16 + tok) & 1u;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 2 * i; e < 2 * i + 2; ++e)
                            if (!(here >> tok & 1u)) s[n][e] = bad ? __uint_as_float(0x7FC00000u) : -INFINITY;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)  // finite values: a weight of zero times an infinity that may lie there would not do
                    if (!(here >> (2 * c + (i & 1) + 8 * (i >> 1)) & 1u)) vf[i] = 0x7F7Fu;
            }
            // ---- softmax weights relative to the running references, t = log2 of a weight (lifted by kLift)
            float t[NT][4], high = 0.f;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    t[n][e] = s[n][e] - ref[n][e & 1];
                    high = fmaxf(high, t[n][e]);
                }
            if (__any_sync(0xFFFFFFFFu, high > kLift + kAtSlack)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = fmaxf(s[n][e], s[n][e + 2]);
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
                        top = fmaxf(top - kLift, ref[n][e]);
                        const float f = exp2_approx(ref[n][e] - top);
                        ref[n][e] = top;
                        sum[n][e] *= f;
                        t[n][e] = s[n][e] - top;
                        t[n][e + 2] = s[n][e + 2] - top;
#pragma unroll
                        for (int i = 0; i < VB * 8; ++i) { o[i][n][e] *= f; o[i][n][e + 2] *= f; }
                    }
            }
            float p[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[n][e] = exp2_approx(t[n][e]);
                    if constexpr (F32) p[n][e] *= frag::kFastFactor;
                    sum[n][e & 1] += p[n][e];
                }
            // ---- output
            auto output = [&](auto way) {
                constexpr bool FAST = decltype(way)::value;
                uint32_t pb[NT][WPARTS][2];  // P^T fragments
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        constexpr float kLower = FAST ? 1.f : 1.f / frag::kFastFactor;
                        float lo = p[n][2 * h] * kLower, hi = p[n][2 * h + 1] * kLower;
#pragma unroll
                        for (int part = 0; part < WPARTS; ++part) {
                            const uint32_t w = pack_bf16x2(lo, hi);
                            pb[n][part][h] = frag::transpose8x8(w);
                            lo -= __uint_as_float(w << 16);
                            hi -= __uint_as_float(w & 0xFFFF0000u);
                        }
                    }
#pragma unroll
                for (int x = 0; x < VB; ++x) {
                    const frag::Scales s0 = frag::make_scales<FAST>((vf[0] >> (8 * x)) & 0xFFu, (vf[1] >> (8 * x)) & 0xFFu, (vm[0] >> (8 * x)) & 0xFFu, (vm[1] >> (8 * x)) & 0xFFu);
                    const frag::Scales s1 = frag::make_scales<FAST>((vf[2] >> (8 * x)) & 0xFFu, (vf[3] >> (8 * x)) & 0xFFu, (vm[2] >> (8 * x)) & 0xFFu, (vm[3] >> (8 * x)) & 0xFFu);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t w0 = frag::scale_word(s0, j), w1 = frag::scale_word(s1, j);
                        const uint32_t a0 = frag::decode_word<WV, FAST>(vb[0][x].w, 0, vb[1][x].w, 0, 2 * j, w0), a1 = frag::decode_word<WV, FAST>(vb[0][x].w, 0, vb[1][x].w, 0, 2 * j + 1, w0);
                        const uint32_t a2 = frag::decode_word<WV, FAST>(vb[2][x].w, 0, vb[3][x].w, 0, 2 * j, w1), a3 = frag::decode_word<WV, FAST>(vb[2][x].w, 0, vb[3][x].w, 0, 2 * j + 1, w1);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            // A long sum in the tensor core is cut off rather than rounded, up to 2^-23 of it per tile.  32-bit queries have a tile's
                            // products added with fp32 additions; a bf16 result, rounded by 2^-9 itself, would gain nothing from the 1 to 4 % that costs.
                            if constexpr (F32) {
                                float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                                for (int part = WPARTS - 1; part >= 0; --part) frag::mma_bf16(d, a0, a1, a2, a3, pb[n][part][0], pb[n][part][1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[8 * x + j][n][e] += d[e];
                            } else {
#pragma unroll
                                for (int part = WPARTS - 1; part >= 0; --part) frag::mma_bf16(o[8 * x + j][n], a0, a1, a2, a3, pb[n][part][0], pb[n][part][1]);
                            }
                        }
                    }
                }
            };
            if (fast) output(std::true_type{});
            else output(std::false_type{});
            __syncwarp();  // the next copies may overwrite the tile
        }
        cp_async_wait<0>();

        // ---- join the sets of warps: in each round the upper half hands its sums to the lower half
        for (int half = a.tw / 2; half >= 1; half >>= 1) {
            if (tw >= half && tw < 2 * half) {
                float* to = reinterpret_cast<float*>(ring) + lane;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) { to[64 * (2 * n + e)] = ref[n][e]; to[64 * (2 * n + e) + 32] = sum[n][e]; }
#pragma unroll
                for (int i = 0; i < VB * 8; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) to[128 * NT + 32 * ((i * NT + n) * 4 + e)] = o[i][n][e];
            }
            sync_all();
            if (tw < half) {
                const float* from = reinterpret_cast<const float*>(rings + (warp + half * a.hw) * kRing) + lane;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float other = from[64 * (2 * n + e)], top = fmaxf(ref[n][e], other);
                        const float f0 = exp2_approx(ref[n][e] - top), f1 = exp2_approx(other - top);
                        ref[n][e] = top;
                        sum[n][e] = sum[n][e] * f0 + from[64 * (2 * n + e) + 32] * f1;
#pragma unroll
                        for (int i = 0; i < VB * 8; ++i)
#pragma unroll
                            for (int h = e; h < 4; h += 2) o[i][n][h] = o[i][n][h] * f0 + from[128 * NT + 32 * ((i * NT + n) * 4 + h)] * f1;
                    }
            }
        }

        // ---- the segment's result: lane (g, c) holds elements 16 (g VB + x) .. + 15 of columns 2c and 2c + 1
        const bool whole = seg.t0 == 0 && seg.t1 == seg.r.count;
        if (tw == 0) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float l = sum[n][e];
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, x);
                    const int col = 8 * n + 2 * c + e, head = head_of(col), f = kv_of(col);
                    if (head < 0) continue;
                    l *= 1.f / frag::kFastFactor;  // the weights' factor; the values' own is in the sums
                    const float norm = whole ? (l == 0.f ? 0.f : 2.f / l) : 2.f;  // the values were decoded halved
                    const int64_t part = ((int64_t)blockIdx.x * 2 + (first_segment ? 0 : 1)) * a.n_q + head;
#pragma unroll
                    for (int x = 0; x < VB; ++x) {
                        const int blk = g * VB + x - f * a.nb;
                        if (blk < 0 || blk >= a.nb) continue;
                        uint32_t v[16];
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            v[2 * j] = __float_as_uint(o[8 * x + j][n][e] * norm);
                            v[2 * j + 1] = __float_as_uint(o[8 * x + j][n][e + 2] * norm);
                        }
                        if (!whole) {
                            store_slice_vec(a.part_o + part * a.d + 16 * blk, v);
                        } else {
                            T* out = static_cast<T*>(a.out) + (int64_t)b * a.ldo + (int64_t)head * a.d + 16 * blk;
                            if constexpr (!F32) {
#pragma unroll
                                for (int j = 0; j < 16; ++j)
                                    v[j] = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(__uint_as_float(v[j]))) << 16;
                            }
                            if (a.o_vec) store_slice_vec(out, v);
                            else store_slice_guarded(out, 1, kSlice, v);
                        }
                    }
                    if (g == 0) {
                        if (!whole) a.part_ml[part] = make_float2(ref[n][e] + kLift, l);
                        else if (a.lse) a.lse[(int64_t)b * a.n_q + head] = (ref[n][e] + kLift + log2f(l)) * 0.69314718055994531f;
                    }
                }
        }
        sync_all();  // nobody overwrites the queries or the handed-over sums while others still read them
    }
}

// host side of one key format; the files that include this instantiate it
template <int WK>
int launch_attn(const AttnArgs& a, int wv, int maxb, int nt, bool f32, bool full, int groups, cudaStream_t st);

template <int WK, int WV, int MAXB, int NT, bool F32, bool FULL>
int launch_attn_one(const AttnArgs& a, int groups, cudaStream_t st) {
    using S = AttnShape<MAXB, NT, F32>;
    constexpr int kRing = attn_ring_bytes<WK, WV, MAXB, NT, F32, FULL>();
    static_assert(S::kMaxUnits * S::kQBytes + S::kWarps * kRing <= kAtSmemBytes, "queries and rings have to fit");
    static PerDevice once;
    if (kernel_setup(once, mx_attn_decode_kernel<WK, WV, MAXB, NT, F32, FULL>, S::kThreads, kAtSmemBytes) < 1) return BDR_ERR_CUDA;
    const size_t smem = a.hw * S::kQBytes + S::kWarps * kRing;
    mx_attn_decode_kernel<WK, WV, MAXB, NT, F32, FULL><<<dim3(a.workers, groups), S::kThreads, smem, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

template <int WK, int WV, bool FULL>
int launch_attn_shape(const AttnArgs& a, int maxb, int nt, bool f32, int groups, cudaStream_t st) {
    if (maxb == 8) {
        if (f32) return launch_attn_one<WK, WV, 8, 1, true, FULL>(a, groups, st);
        return nt == 1 ? launch_attn_one<WK, WV, 8, 1, false, FULL>(a, groups, st) : launch_attn_one<WK, WV, 8, 2, false, FULL>(a, groups, st);
    }
    return f32 ? launch_attn_one<WK, WV, 16, 1, true, FULL>(a, groups, st) : launch_attn_one<WK, WV, 16, 1, false, FULL>(a, groups, st);
}

#define BDR_ATTN_KEY_FORMAT(WK)                                                                                                        \
    template <>                                                                                                                        \
    int launch_attn<WK>(const AttnArgs& a, int wv, int maxb, int nt, bool f32, bool full, int groups, cudaStream_t st) {              \
        switch (wv) {                                                                                                                  \
            case 3: return full ? launch_attn_shape<WK, 3, true>(a, maxb, nt, f32, groups, st) : launch_attn_shape<WK, 3, false>(a, maxb, nt, f32, groups, st); \
            case 5: return full ? launch_attn_shape<WK, 5, true>(a, maxb, nt, f32, groups, st) : launch_attn_shape<WK, 5, false>(a, maxb, nt, f32, groups, st); \
            default: return full ? launch_attn_shape<WK, 8, true>(a, maxb, nt, f32, groups, st) : launch_attn_shape<WK, 8, false>(a, maxb, nt, f32, groups, st); \
        }                                                                                                                              \
    }

}  // namespace bdr
