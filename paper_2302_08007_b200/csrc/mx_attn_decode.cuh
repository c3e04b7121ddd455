// Attention of one new token per sequence over a paged key-value cache in MX format (see mx_attn_decode in bdr.h).
//
// The cache is read once and every element of it is used for the few query heads that share it, so the bounds are the bytes
// of the cache and the instructions that decode them.  A warp owns one "unit", a key-value head with its query heads (small
// heads are merged until a unit fills 128 elements), and walks over tiles of 16 tokens:
//   scores    S^T[16 tokens, 8 columns] = K[16, d] Q^T: the key blocks are decoded straight into the A fragment (lane (g, c)
//             decodes whole blocks of tokens g and g + 8); Q waits in shared memory in the order of the B fragment;
//   softmax   with a running reference per column instead of the running maximum: it is raised only when a score passes it
//             by kSlack (in powers of two), so most tiles need a vote and no reduction over lanes;
//   output    O^T[d, 8 columns] += V^T P^T: V is decoded like K (lane (g, c): block g of four tokens, two tokens to a word as the A
//             fragment wants them), and P^T is the 8x8 transpose of the score fragment.
// The packed bytes of the next tile are fetched while the present one is computed: keys as soon as the scores are done,
// values as soon as the output is.
//
// Work is split over the length of the cache: the tiles of all sequences form one long line that is cut into equal parts,
// one per worker CTA, whatever the individual lengths are (each worker finds its part from `lengths`).  A part that covers a
// sequence's whole range writes the result; other parts leave their sums and references in the workspace, where a second
// kernel joins them in order.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "bdr_device.cuh"
#include "bdr_host.h"
#include "mx_frag.cuh"

namespace bdr {

constexpr int kAtThreads = 256, kAtWarps = kAtThreads / 32;
constexpr float kAtSlack = 8.f;     // a softmax weight relative to the running reference stays below 2^8
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
    int hw, tw, workers;                   // warps over units, warps over tokens, worker CTAs per group of units
    int n_pages, max_pages, cap, window;   // cap = max_pages * page_size
    int q_vec;                             // two query elements may be read at once
    FastDiv page;
    float scale2;                          // 2 scale log2(e): the keys are decoded halved
    int* status;
};

// Tiles of 16 tw tokens that sequence b's positions touch.
struct SeqRange {
    int start, end, first, count;
};
__device__ __forceinline__ SeqRange seq_range(const AttnArgs& a, int b) {
    SeqRange r;
    const int len = min(__ldg(a.lengths + b), a.cap + 1);  // a position beyond the table's pages poisons the result
    r.end = max(len, 0);
    r.start = a.window > 0 ? max(0, r.end - a.window) : 0;
    const int mt = 16 * a.tw;
    r.first = r.start / mt;
    r.count = r.end > r.start ? (r.end + mt - 1) / mt - r.first : 0;
    return r;
}

// Tiles of all sequences together (called by whole warps).
__device__ __forceinline__ int64_t total_tiles(const AttnArgs& a, int lane) {
    int64_t n = 0;
    for (int b = lane; b < a.n_seqs; b += 32) n += seq_range(a, b).count;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xFFFFFFFFu, n, o);
    return n;
}

// Tiles of the sequences before `limit`, stopping early before the sequence that holds tile `u` (u < 0: no such stop).
// Returns the prefix and leaves the sequence in b.
__device__ __forceinline__ int64_t walk_tiles(const AttnArgs& a, int lane, int limit, int64_t u, int& b) {
    int64_t p = 0;
    for (int base = 0;; base += 32) {
        const int mine = base + lane;
        int64_t n = mine < limit ? seq_range(a, mine).count : 0;
        int64_t incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += v;
        }
        const int64_t all = __shfl_sync(0xFFFFFFFFu, incl, 31);
        if (base + 32 >= limit || (u >= 0 && p + all > u)) {
            if (u < 0) { b = limit; return p + all; }
            const unsigned hit = __ballot_sync(0xFFFFFFFFu, p + incl > u);
            const int at = hit ? __ffs(hit) - 1 : 31;
            b = base + at;
            return p + __shfl_sync(0xFFFFFFFFu, incl - n, at);
        }
        p += all;
    }
}

__device__ __forceinline__ int64_t worker_begin(int64_t total, int w, int workers) { return total * w / workers; }

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
template <int WK, int WV, int MAXB, int NT, bool F32>
struct AttnShape {
    static constexpr int kKeyBlocks = MAXB / 4, kValBlocks = MAXB / 8;  // per lane and token
    static constexpr int kParts = F32 ? 3 : 1;
    static constexpr int kD = 16 * MAXB;
    static constexpr size_t kQBytes = (size_t)kParts * MAXB * NT * 32 * 8;          // per warp
    static constexpr int kOPitch = kD + 4;
    static constexpr size_t kOBytes = (size_t)8 * NT * kOPitch * 4 + 8 * NT * 8;    // per warp: sums, references and weights
    static constexpr size_t kSmem = kAtWarps * (kQBytes + kOBytes);
};

template <int WK, int WV, int MAXB, int NT, bool F32, bool FULL>
__global__ void __launch_bounds__(kAtThreads, MAXB == 8 && NT == 1 ? 2 : 1) mx_attn_decode_kernel(const AttnArgs a) {
    cudaTriggerProgrammaticLaunchCompletion();  // the joining kernel may take its place as soon as there is room
    using S = AttnShape<WK, WV, MAXB, NT, F32>;
    using T = typename std::conditional<F32, float, __nv_bfloat16>::type;
    constexpr int KB = S::kKeyBlocks, VB = S::kValBlocks, PARTS = S::kParts;
    extern __shared__ __align__(16) uint8_t smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    uint4* qs = reinterpret_cast<uint4*>(smem + warp * S::kQBytes);
    float* os_all = reinterpret_cast<float*>(smem + kAtWarps * S::kQBytes);
    constexpr int kOFloats = (int)(S::kOBytes / 4);
    float* os = os_all + warp * kOFloats;
    const int hw = warp % a.hw, tw = warp / a.hw;
    const int unit = blockIdx.y * a.hw + hw;
    const bool live = unit < a.n_units && tw < a.tw;
    const int mk = unit / a.passes, pass = unit - mk * a.passes, kv0 = mk * a.merge;
    const int kv_n = live ? min(a.merge, a.n_kv - kv0) : 0, blocks = kv_n * a.nb, block0 = kv0 * a.nb;

    const int64_t total = total_tiles(a, lane);
    int64_t u = worker_begin(total, blockIdx.x, a.workers);
    const int64_t u_end = worker_begin(total, blockIdx.x + 1, a.workers);
    if (u >= u_end) return;  // uniform for the CTA
    int b = 0;
    int64_t prefix = walk_tiles(a, lane, a.n_seqs, u, b);
    bool first_segment = true;

    // query head of a column, or -1
    auto head_of = [&](int col) {
        const int f = col / a.per_pass, i = pass * a.per_pass + (col - f * a.per_pass);
        return f < kv_n && i < a.group ? (kv0 + f) * a.group + i : -1;
    };

    while (u < u_end) {
        const SeqRange r = seq_range(a, b);
        if (r.count == 0) { ++b; continue; }
        const int t0 = (int)(u - prefix), t1 = (int)min((int64_t)r.count, u_end - prefix);

        // ---- queries into shared memory: [part][pair of steps][column group][lane].  Step 8 x + j of a lane holds elements 2j and 2j + 1 of
        // blocks 2x and 2x + 1 of its own: {2x: 2j, 2x+1: 2j}, {2x: 2j+1, 2x+1: 2j+1}.
        if (live) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int col = 8 * n + g, head = head_of(col), f = col / a.per_pass;
                const T* q = static_cast<const T*>(a.q) + (int64_t)b * a.ldq + (int64_t)max(head, 0) * a.d;
#pragma unroll
                for (int x = 0; x < KB / 2; ++x) {
                    const int at0 = (c * KB + 2 * x) * 16 - f * a.d, at1 = at0 + 16;  // elements of the head
                    const bool in0 = head >= 0 && at0 >= 0 && at0 < a.d, in1 = head >= 0 && at1 >= 0 && at1 < a.d;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
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
        __syncwarp();

        float o[VB * 8][NT][4], ref[NT][2], sum[NT][2];
#pragma unroll
        for (int i = 0; i < VB * 8; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][n][e] = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) { ref[n][0] = ref[n][1] = kAtNone; sum[n][0] = sum[n][1] = 0.f; }

        int tile = (r.first + t0) * a.tw + tw;
        int tile_end = live ? min((r.first + t1) * a.tw, (r.end + 15) / 16) : 0;
        while (tile < tile_end && tile * 16 + 16 <= r.start) tile += a.tw;

        // slot of token 16 tile + lane (lanes 0 .. 15): -1 outside the range, -2 for a page that does not exist
        auto slot_of = [&](int t) {
            const int tok = 16 * t + (lane & 15);
            int slot = -1;
            if (t < tile_end && tok >= r.start && tok < r.end) {
                const int pg = (int)fastdiv((uint32_t)tok, a.page);
                const int id = pg < a.max_pages ? __ldg(a.table + (int64_t)b * a.ld_table + pg) : -1;
                const bool ok = id >= 0 && id < a.n_pages;
                slot = ok ? id * (int)a.page.d + (tok - pg * (int)a.page.d) : -2;
                if (!ok) atomicCAS(a.status, 0, (int)BDR_ERR_SIZE);
            }
            return slot;
        };
        // the fetched bytes: keys of tokens g and g + 8, values of tokens 2c, 2c + 1, 2c + 8 and 2c + 9; exponents and
        // microexponents of a lane's blocks in the bytes of one word
        uint32_t kr[2][FULL ? KB * WK / 2 : KB * frag::Block<WK>::kWords];
        uint32_t kf[2], km[2], vf[4], vm[4];
        frag::Block<WV> vb[4][VB];
        const uint8_t* const ke = a.k.elems + (block0 + c * KB) * (2 * WK);
        const uint8_t* const kx = a.k.exps + block0 + c * KB;
        const uint8_t* const ki = a.k.micro + block0 + c * KB;
        const uint8_t* const ve = a.v.elems + (block0 + g * VB) * (2 * WV);
        const uint8_t* const vx = a.v.exps + block0 + g * VB;
        const uint8_t* const vi = a.v.micro + block0 + g * VB;
        // A token outside the range reads slot 0; what it gives is replaced below.
        auto load_keys = [&](int slots) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t at = (uint32_t)max(__shfl_sync(0xFFFFFFFFu, slots, g + 8 * i), 0);
                const uint8_t* e = ke + (uint64_t)at * (uint32_t)a.k.ld_elems;
                const uint8_t* x = kx + (uint64_t)at * (uint32_t)a.k.ld_exps;
                const uint8_t* m = ki + (uint64_t)at * (uint32_t)a.k.ld_micro;
                if constexpr (FULL) {  // neighbouring blocks, all present: whole aligned words
                    if constexpr (KB == 2) { kf[i] = __ldg(reinterpret_cast<const uint16_t*>(x)); km[i] = __ldg(reinterpret_cast<const uint16_t*>(m)); }
                    else { kf[i] = __ldg(reinterpret_cast<const uint32_t*>(x)); km[i] = __ldg(reinterpret_cast<const uint32_t*>(m)); }
                    if constexpr (WK == 8) {
#pragma unroll
                        for (int w = 0; w < KB; ++w) {
                            const uint4 v = __ldg(reinterpret_cast<const uint4*>(e) + w);
                            kr[i][4 * w] = v.x; kr[i][4 * w + 1] = v.y; kr[i][4 * w + 2] = v.z; kr[i][4 * w + 3] = v.w;
                        }
                    } else {
#pragma unroll
                        for (int w = 0; w < KB * WK / 2; ++w) kr[i][w] = __ldg(reinterpret_cast<const uint32_t*>(e) + w);
                    }
                } else {
                    kf[i] = km[i] = 0;
#pragma unroll
                    for (int y = 0; y < KB; ++y) {
                        if (c * KB + y < blocks) {
                            constexpr int BW = frag::Block<WK>::kWords;
                            const frag::Block<WK> blk = frag::load_block<WK>(e + y * (2 * WK));
#pragma unroll
                            for (int w = 0; w < BW; ++w) kr[i][y * BW + w] = blk.w[w];
                            kf[i] |= (uint32_t)__ldg(x + y) << (8 * y);
                            km[i] |= (uint32_t)__ldg(m + y) << (8 * y);
                        }
                    }
                }
            }
        };
        auto load_values = [&](int slots) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t at = (uint32_t)max(__shfl_sync(0xFFFFFFFFu, slots, 2 * c + (i & 1) + 8 * (i >> 1)), 0);
                const uint8_t* e = ve + (uint64_t)at * (uint32_t)a.v.ld_elems;
                const uint8_t* x = vx + (uint64_t)at * (uint32_t)a.v.ld_exps;
                const uint8_t* m = vi + (uint64_t)at * (uint32_t)a.v.ld_micro;
                if constexpr (!FULL) vf[i] = vm[i] = 0;
#pragma unroll
                for (int y = 0; y < VB; ++y) {
                    if (FULL || g * VB + y < blocks) {
                        vb[i][y] = frag::load_block<WV>(e + y * (2 * WV));
                        const uint32_t f = __ldg(x + y), u = __ldg(m + y);
                        if (FULL && y == 0) { vf[i] = f; vm[i] = u; }
                        else { vf[i] |= f << (8 * y); vm[i] |= u << (8 * y); }
                    }
                }
            }
        };

        int next = slot_of(tile), now = next;
        if (tile < tile_end) {
            load_keys(next);
            load_values(next);
            next = slot_of(tile + a.tw);
        }
        for (; tile < tile_end; tile += a.tw) {
            // ---- scores
            float s[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
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
#pragma unroll
            for (int x = 0; x < KB / 2; ++x) {
                frag::Scales sc[2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    sc[i] = frag::make_scales(frag::spread_bytes(kf[i] >> (16 * x)), frag::spread_bytes(km[i] >> (16 * x)));
                if constexpr (!FULL) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int y = 2 * x; y < 2 * x + 2; ++y) {
                            constexpr int BW = frag::Block<WK>::kWords;
                            frag::Block<WK> blk;
#pragma unroll
                            for (int w = 0; w < BW; ++w) blk.w[w] = kr[i][y * BW + w];
                            frag::align_block(blk, (uint32_t)((block0 + c * KB + y) * (2 * WK)));
#pragma unroll
                            for (int w = 0; w < BW; ++w) kr[i][y * BW + w] = blk.w[w];
                        }
                }
                constexpr int kBits = FULL ? 16 * WK : 32 * frag::Block<WK>::kWords;  // from one block's stream to the next's
                const int b0 = 2 * x * kBits, b1 = b0 + kBits;
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    uint32_t y[2][4];  // rows g and g + 8, elements 2j .. 2j + 3
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            y[i][e] = frag::decode_word<WK>(kr[i], b0, kr[i], b1, 2 * j + e, frag::scale_word(sc[i], j + (e >> 1)));
#pragma unroll
                    for (int part = PARTS - 1; part >= 0; --part)
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const uint4 qv = qs[((part * MAXB / 2 + 4 * x + j / 2) * NT + n) * 32 + lane];
                            frag::mma_bf16(s[n], y[0][0], y[1][0], y[0][1], y[1][1], qv.x, qv.y);
                            frag::mma_bf16(s[n], y[0][2], y[1][2], y[0][3], y[1][3], qv.z, qv.w);
                        }
                }
            }
            if (spoilt[0] | spoilt[1]) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (spoilt[e >> 1] >> ((8 * n + 2 * c + (e & 1)) / a.per_pass) & 1u) s[n][e] = __uint_as_float(0x7FC00000u);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][e] *= a.scale2;
            if (!__all_sync(0xFFFFFFFFu, now >= 0)) {  // a tile at an end of the range, or with a page that does not exist
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int slot = __shfl_sync(0xFFFFFFFFu, now, g + 8 * i);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 2 * i; e < 2 * i + 2; ++e)
                            if (slot < 0) s[n][e] = slot == -1 ? -INFINITY : __uint_as_float(0x7FC00000u);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)  // zero blocks: a weight of zero times anything that a slot may hold would not do
                    if (__shfl_sync(0xFFFFFFFFu, now, 2 * c + (i & 1) + 8 * (i >> 1)) < 0) vf[i] = 0;
            }
            const bool more = tile + a.tw < tile_end;
            if (more) load_keys(next);
            // ---- softmax weights relative to the running references, t = log2 of a weight
            float t[NT][4], high = 0.f;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    t[n][e] = s[n][e] - ref[n][e & 1];
                    high = fmaxf(high, t[n][e]);
                }
            if (__any_sync(0xFFFFFFFFu, high > kAtSlack)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = fmaxf(s[n][e], s[n][e + 2]);
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
                        top = fmaxf(top, ref[n][e]);
                        const float f = exp2_approx(ref[n][e] - top);
                        ref[n][e] = top;
                        sum[n][e] *= f;
                        t[n][e] = s[n][e] - top;
                        t[n][e + 2] = s[n][e + 2] - top;
#pragma unroll
                        for (int i = 0; i < VB * 8; ++i) { o[i][n][e] *= f; o[i][n][e + 2] *= f; }
                    }
            }
            uint32_t pb[NT][PARTS][2];  // P^T fragments (32-bit: three parts of eight bits)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = exp2_approx(t[n][e]);
                    sum[n][e & 1] += p[e];
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float lo = p[2 * h], hi = p[2 * h + 1];
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) {
                        const uint32_t w = pack_bf16x2(lo, hi);
                        pb[n][part][h] = frag::transpose8x8(w);
                        lo -= __uint_as_float(w << 16);
                        hi -= __uint_as_float(w & 0xFFFF0000u);
                    }
                }
            }
            // ---- output
#pragma unroll
            for (int x = 0; x < VB; ++x) {
#pragma unroll
                for (int i = 0; i < 4; ++i) frag::align_block(vb[i][x], (uint32_t)((block0 + g * VB + x) * (2 * WV)));
                const frag::Scales s0 = frag::make_scales((vf[0] >> (8 * x)) & 0xFFu, (vf[1] >> (8 * x)) & 0xFFu, (vm[0] >> (8 * x)) & 0xFFu, (vm[1] >> (8 * x)) & 0xFFu);
                const frag::Scales s1 = frag::make_scales((vf[2] >> (8 * x)) & 0xFFu, (vf[3] >> (8 * x)) & 0xFFu, (vm[2] >> (8 * x)) & 0xFFu, (vm[3] >> (8 * x)) & 0xFFu);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t w0 = frag::scale_word(s0, j), w1 = frag::scale_word(s1, j);
                    const uint32_t a0 = frag::decode_word<WV>(vb[0][x].w, 0, vb[1][x].w, 0, 2 * j, w0), a1 = frag::decode_word<WV>(vb[0][x].w, 0, vb[1][x].w, 0, 2 * j + 1, w0);
                    const uint32_t a2 = frag::decode_word<WV>(vb[2][x].w, 0, vb[3][x].w, 0, 2 * j, w1), a3 = frag::decode_word<WV>(vb[2][x].w, 0, vb[3][x].w, 0, 2 * j + 1, w1);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int part = PARTS - 1; part >= 0; --part) frag::mma_bf16(o[8 * x + j][n], a0, a1, a2, a3, pb[n][part][0], pb[n][part][1]);
                }
            }
            if (more) {
                load_values(next);
                now = next;
                next = slot_of(tile + 2 * a.tw);
            }
        }

        // ---- the segment's result: every warp's sums into shared memory, then joined over the token warps
        float2* ml = reinterpret_cast<float2*>(os + 8 * NT * S::kOPitch);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float l = sum[n][e];
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, x);
                const int col = 8 * n + 2 * c + e;
                if (g == 0) ml[col] = make_float2(ref[n][e], l);
#pragma unroll
                for (int x = 0; x < VB; ++x)
#pragma unroll
                    for (int j = 0; j < 8; j += 2)
                        *reinterpret_cast<float4*>(os + col * S::kOPitch + (g * VB + x) * 16 + 2 * j) =
                            make_float4(o[8 * x + j][n][e], o[8 * x + j][n][e + 2], o[8 * x + j + 1][n][e], o[8 * x + j + 1][n][e + 2]);
            }
        if (a.tw > 1) __syncthreads();
        else __syncwarp();
        const bool whole = t0 == 0 && t1 == r.count;
        if (live) {
            for (int col = tw; col < 8 * NT; col += a.tw) {
                const int head = head_of(col);
                if (head < 0) continue;
                const int f = col / a.per_pass;
                float m = kAtNone, l = 0.f;
                for (int w = 0; w < a.tw; ++w)
                    m = fmaxf(m, reinterpret_cast<float2*>(os_all + (hw + w * a.hw) * kOFloats + 8 * NT * S::kOPitch)[col].x);
                for (int w = 0; w < a.tw; ++w) {
                    const float2 x = reinterpret_cast<float2*>(os_all + (hw + w * a.hw) * kOFloats + 8 * NT * S::kOPitch)[col];
                    l += x.y * exp2_approx(x.x - m);
                }
                const float norm = whole ? (l == 0.f ? 0.f : 2.f / l) : 2.f;  // the values were decoded halved
                const int64_t part = ((int64_t)blockIdx.x * 2 + (first_segment ? 0 : 1)) * a.n_q + head;
                for (int e = lane; e < a.d; e += 32) {
                    float v = 0.f;
                    for (int w = 0; w < a.tw; ++w) {
                        const float* ow = os_all + (hw + w * a.hw) * kOFloats;
                        const float mw = reinterpret_cast<const float2*>(ow + 8 * NT * S::kOPitch)[col].x;
                        const float x = ow[col * S::kOPitch + f * a.d + e];
                        v += x * exp2_approx(mw - m);
                    }
                    v *= norm;
                    if (whole) {
                        T* out = static_cast<T*>(a.out) + (int64_t)b * a.ldo + (int64_t)head * a.d + e;
                        if constexpr (F32) *out = v;
                        else *out = __float2bfloat16_rn(v);
                    } else {
                        a.part_o[part * a.d + e] = v;
                    }
                }
                if (lane == 0) {
                    if (!whole) a.part_ml[part] = make_float2(m, l);
                    else if (a.lse) a.lse[(int64_t)b * a.n_q + head] = (m + log2f(l)) * 0.69314718055994531f;
                }
            }
        }
        if (a.tw > 1) __syncthreads();
        else __syncwarp();
        first_segment = false;
        u = prefix + t1;
        if (t1 == r.count) { prefix += r.count; ++b; }
    }
}

// host side of one key format; the files that include this instantiate it
template <int WK>
int launch_attn(const AttnArgs& a, int wv, int maxb, int nt, bool f32, bool full, int groups, cudaStream_t st);

template <int WK, int WV, int MAXB, int NT, bool F32, bool FULL>
int launch_attn_one(const AttnArgs& a, int groups, cudaStream_t st) {
    using S = AttnShape<WK, WV, MAXB, NT, F32>;
    static PerDevice once;
    if (kernel_setup(once, mx_attn_decode_kernel<WK, WV, MAXB, NT, F32, FULL>, kAtThreads, S::kSmem) < 1) return BDR_ERR_CUDA;
    mx_attn_decode_kernel<WK, WV, MAXB, NT, F32, FULL><<<dim3(a.workers, groups), kAtThreads, S::kSmem, st>>>(a);
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
