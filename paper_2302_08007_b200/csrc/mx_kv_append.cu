// New keys and values into an MX-packed paged cache, with the position rotation applied on the way:
//     (a, b) -> (a cos - b sin, b cos + a sin)    for the pairs of the first rot_dim elements of every query and key head,
// then Q(.) of the keys and values along the head dimension (blocks of 16 elements, so a head's blocks are its own), and the
// three packed planes of each into the cache line of the token's slot.
//
// The rotated key goes from its fp32 sum into the quantizer without a rounding to the tensor's type in between; products and
// sums are rounded to fp32 one by one (no contraction), so the result does not depend on how a compiler fuses them.
// Streaming: a lane owns one 16-element block of a head and walks over heads of the same token, which keeps the block's
// cosines and sines in registers; its partner elements (rot_dim / 2 away) come from the same run of heads, which the warp copies
// into shared memory three iterations ahead (144 -> 106 us at the size below).  A CTA's warps share tokens when there are few of
// them.  Results leave in 32-byte stores.
//
// Measured (32 query and 2 x 8 key-value heads of 128 elements, bf16, MX9, rotated queries and quantized values written too): 16384
// tokens 86.6 us = 5.2 TB/s, one token 3.9 us; 1003 tokens of 20 + 2 x 4 heads of 80, fp32, MX6 and MX4, 7.9 us (6.2 from the L2).  Long calls are
// bound by instructions as much as by memory (3570 per warp and token, issue slots about 60 % busy, integer/logic pipe half
// busy); a version whose warps stay and run their copies on into the next token needed more registers than there are (129 us).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "bdr_device.cuh"
#include "bdr_host.h"
#include "mx_frag.cuh"

namespace bdr {

int* device_status_word();

constexpr int kApThreads = 256, kApWarps = kApThreads / 32;
constexpr int kApStages = 4;  // iterations in a warp's ring

struct AppendArgs {
    bdr_planes_t plane[2];       // keys, values
    int m[2];
    const void* src[3];          // q, k, v
    void* dst[3];                // rotated q, quantized k, quantized v (the last two contiguous; NULL = not wanted)
    int64_t ld_src[3], ld_q;
    bool wide[3];                // of dst: blocks start on 32-byte boundaries
    int heads[3], iters[3];      // heads of each, and warp iterations over them
    const int64_t *slots, *positions;
    const float *cosv, *sinv;
    int64_t ld_rot, n_pos, n_slots, n_tokens;
    int rot_dim, nb, warps_per_token, wpt_log;  // (a power of two)
    bool pad[2];                 // lines with bytes between their natural length and the pitch
    int* status;
};

// U elements at p (U = 8, 4 or 1) as fp32 bit patterns
template <typename T, int U>
__device__ __forceinline__ void load_units(const T* p, uint32_t* u) {
    if constexpr (sizeof(T) == 2 && U == 8) {
        const uint4 w = __ldg(reinterpret_cast<const uint4*>(p));
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) { u[2 * k] = ws[k] << 16; u[2 * k + 1] = ws[k] & 0xFFFF0000u; }
    } else if constexpr (sizeof(T) == 2 && U == 4) {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(p));
        u[0] = w.x << 16; u[1] = w.x & 0xFFFF0000u; u[2] = w.y << 16; u[3] = w.y & 0xFFFF0000u;
    } else if constexpr (sizeof(T) == 4 && U >= 4) {
#pragma unroll
        for (int k = 0; k < U / 4; ++k) {
            const uint4 w = __ldg(reinterpret_cast<const uint4*>(p) + k);
            u[4 * k] = w.x; u[4 * k + 1] = w.y; u[4 * k + 2] = w.z; u[4 * k + 3] = w.w;
        }
    } else {
#pragma unroll
        for (int k = 0; k < U; ++k) u[k] = Elem<T>::load_bits(p + k);
    }
}

// eight elements in shared memory as fp32 bit patterns
__device__ __forceinline__ void shared_units(const __nv_bfloat16* p, uint32_t* u) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { u[2 * k] = ws[k] << 16; u[2 * k + 1] = ws[k] & 0xFFFF0000u; }
}
__device__ __forceinline__ void shared_units(const float* p, uint32_t* u) {
    const uint4 w = reinterpret_cast<const uint4*>(p)[0], v = reinterpret_cast<const uint4*>(p)[1];
    u[0] = w.x; u[1] = w.y; u[2] = w.z; u[3] = w.w;
    u[4] = v.x; u[5] = v.y; u[6] = v.z; u[7] = v.w;
}

// A lane's 16 results at p; WIDE: p is on a 32-byte boundary, so that every store fills whole sectors.
__device__ __forceinline__ void store_eight(void* p, const uint32_t (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                 "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}
__device__ __forceinline__ void store_block(__nv_bfloat16* p, const uint32_t (&w)[8], bool wide) {  // already two to a word
    if (wide) {
        store_eight(p, w);
    } else {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}
__device__ __forceinline__ void store_block(float* p, const uint32_t (&u)[kSlice], bool wide) {
    if (wide) {
        const uint32_t a[8] = {u[0], u[1], u[2], u[3], u[4], u[5], u[6], u[7]}, b[8] = {u[8], u[9], u[10], u[11], u[12], u[13], u[14], u[15]};
        store_eight(p, a);
        store_eight(p + 8, b);
    } else {
        store_slice_vec(p, u);
    }
}
// quantized values of 7 mantissa bits at most: the upper half of each word
__device__ __forceinline__ void store_values(__nv_bfloat16* p, const uint32_t (&u)[kSlice], bool wide) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __byte_perm(u[2 * i], u[2 * i + 1], 0x7632);
    store_block(p, w, wide);
}
__device__ __forceinline__ void store_values(float* p, const uint32_t (&u)[kSlice], bool wide) { store_block(p, u, wide); }

template <int W>
__device__ __forceinline__ void store_codes(uint8_t* p, const uint32_t (&u)[kSlice], const uint32_t (&rq)[kSlice],
                                            const uint32_t (&cb)[kSlice / 2]) {
    uint32_t words[(kSlice * W + 31) / 32];
    if constexpr (W == 8) {
        // a word's four magnitudes by multiply-adds, its four signs from the top bytes of the values
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t q = rq[4 * i] + rq[4 * i + 1] * 0x100u + (rq[4 * i + 2] + rq[4 * i + 3] * 0x100u) * 0x10000u -
                               (cb[2 * i] + cb[2 * i + 1] * 0x10000u) * 0x101u;
            const uint32_t s = __byte_perm(__byte_perm(u[4 * i], u[4 * i + 1], 0x0073), __byte_perm(u[4 * i + 2], u[4 * i + 3], 0x0073), 0x5410);
            words[i] = frag::lop3<frag::kAndOr>(s, 0x80808080u, q);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(words[0], words[1], words[2], words[3]);
    } else {  // 10 or 6 bytes at a two-byte boundary
        pack_words<W, kSlice, 2>(u, rq, cb, words);
#pragma unroll
        for (int h = 0; h < W; ++h) *reinterpret_cast<uint16_t*>(p + 2 * h) = (uint16_t)(words[h >> 1] >> (16 * (h & 1)));
    }
}

// maxima that keep a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Q(.) of a finite block of a Table II format, the fast formulation of quantize_slice for exactly this shape: u holds the fp32
// bits, pm the larger magnitude of each pair; yb the quantized values' bits; rq, cb the raw magnitudes and their offsets for
// pack_words; returns the microexponents.
template <int W>
__device__ __forceinline__ uint32_t quantize_table2(const uint32_t (&u)[kSlice], const float (&pm)[kSlice / 2], uint32_t F23,
                                                    uint32_t (&yb)[kSlice], uint32_t (&rq)[kSlice], uint32_t (&cb)[kSlice / 2]) {
    constexpr uint32_t kBase = ((uint32_t)(127 + 23 - (W - 2)) << 23) | 0x400000u, kMax = (1u << (W - 1)) - 1u;
    const float K = __uint_as_float(max(0x7F000000u - F23, 0x00400000u)), Kinv = __uint_as_float(max(F23, 0x00400000u));  // 2^(127-F), 2^(F-127)
    uint32_t micro = 0;
#pragma unroll
    for (int j = 0; j < kSlice / 2; ++j) {
        const bool low = pm[j] < __uint_as_float(F23);  // tau: both below 2^(F-127)
        cb[j] = low ? kBase - 0x00800000u : kBase;
        if (low) micro |= 1u << j;
        const float C = __uint_as_float(cb[j]), Cmax = __uint_as_float(cb[j] + kMax);
#pragma unroll
        for (int k = 2 * j; k < 2 * j + 2; ++k) {
            // the scaling is exact, so the one rounding of the multiply-add is the one to the format's grid
            const float r = fminf(fmaf(fabsf(__uint_as_float(u[k])), K, C), Cmax);
            rq[k] = __float_as_uint(r);
            yb[k] = __float_as_uint(__fmul_rn(__fsub_rn(r, C), Kinv)) | (u[k] & 0x80000000u);
        }
    }
    return micro;
}

// One block of 16 values (fp32 bits u) of the key (which = 0) or value line of a slot.
template <int W>
__device__ __forceinline__ void pack_block_as(const bdr_planes_t& p, int64_t slot, int block, uint32_t (&u)[kSlice], uint32_t (&yb)[kSlice], bool store) {
    float pm[kSlice / 2];  // a NaN stays one
#pragma unroll
    for (int j = 0; j < kSlice / 2; ++j) pm[j] = max_nan(fabsf(__uint_as_float(u[2 * j])), fabsf(__uint_as_float(u[2 * j + 1])));
    const float top = max_nan(max_nan(max_nan(pm[0], pm[1], pm[2]), pm[3], pm[4]), max_nan(pm[5], pm[6], pm[7]));
    const uint32_t F23 = __float_as_uint(top) & kExpMask;
    uint32_t rq[kSlice], cb[kSlice / 2], micro;
    if (F23 != kExpMask) {
        micro = quantize_table2<W>(u, pm, F23, yb, rq, cb);
    } else {  // an infinity or a NaN: codes and microexponents zero, values NaN
        micro = 0;
#pragma unroll
        for (int k = 0; k < kSlice; ++k) {
            yb[k] = 0x7FC00000u;
            u[k] = rq[k] = cb[k / 2] = 0;
        }
    }
    if (!store) return;
    p.exps[slot * p.ld_exps + block] = (uint8_t)(F23 >> 23);
    p.micro[slot * p.ld_micro + block] = (uint8_t)micro;
    store_codes<W>(p.elems + slot * p.ld_elems + block * (2 * W), u, rq, cb);
}
__device__ __forceinline__ void pack_block_to(const AppendArgs& a, int which, int64_t slot, int block, uint32_t (&u)[kSlice],
                                              uint32_t (&yb)[kSlice], bool store) {
    switch (a.m[which]) {
        case 2: pack_block_as<3>(a.plane[which], slot, block, u, yb, store); break;
        case 4: pack_block_as<5>(a.plane[which], slot, block, u, yb, store); break;
        default: pack_block_as<8>(a.plane[which], slot, block, u, yb, store); break;
    }
}

// zeroes the bytes of a slot's lines between their natural length and the pitch, as bdr_pack does
__device__ __forceinline__ void pad_lines(const AppendArgs& a, int which, int64_t slot, int lane) {
    const bdr_planes_t& p = a.plane[which];
    const int64_t nb = (int64_t)a.heads[1] * a.nb;
    for (int64_t i = nb + lane; i < p.ld_exps; i += 32) p.exps[slot * p.ld_exps + i] = 0;
    for (int64_t i = nb + lane; i < p.ld_micro; i += 32) p.micro[slot * p.ld_micro + i] = 0;
    for (int64_t i = nb * 2 * (a.m[which] + 1) + lane; i < p.ld_elems; i += 32) p.elems[slot * p.ld_elems + i] = 0;
}

// U: how many elements may be loaded at once at multiples of U elements of a head, at rot_dim / 2 and in the tables
template <typename T, int U, bool INTERLEAVED>
__global__ void __launch_bounds__(kApThreads, 2) mx_kv_append_kernel(const AppendArgs a) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int wpt = a.warps_per_token;
    const int64_t t = ((int64_t)blockIdx.x * kApWarps + warp) >> a.wpt_log;
    if (t >= a.n_tokens) return;
    const int nb = a.nb, hpi = 32 / nb, hl = lane / nb, b = lane - hl * nb;  // heads per iteration, this lane's head and block
    const int d = 16 * nb, rot = a.rot_dim, half = rot / 2;
    const int64_t slot = __ldg(a.slots + t);
    bool store = slot >= 0, bad = false;
    if (slot >= a.n_slots) { store = false; if (lane == 0) atomicCAS(a.status, 0, (int)BDR_ERR_SIZE); }
    int64_t pos = 0;
    if (rot) {
        pos = __ldg(a.positions + t);
        if (pos < 0 || pos >= a.n_pos) {
            bad = true;
            store = false;
            pos = 0;
            if (lane == 0 && slot >= 0) atomicCAS(a.status, 0, (int)BDR_ERR_SIZE);  // nothing was asked for a padding token
        }
    }
    // this block's angles: pair i of the head has angle i; an element beyond rot_dim is not rotated
    constexpr int kAngles = INTERLEAVED ? 8 : 16;
    float cs[kAngles], sn[kAngles];
    if (rot) {
        const float* cr = a.cosv + pos * a.ld_rot;
        const float* sr = a.sinv + pos * a.ld_rot;
        constexpr int UA = U >= 4 ? 4 : 1;
#pragma unroll
        for (int i = 0; i < kAngles; i += UA) {
            const int e = INTERLEAVED ? 8 * b + i : 16 * b + i;  // (half layout: element index, its angle is e or e - half)
            const int at = INTERLEAVED ? e : (e < half ? e : e - half);
            uint32_t c4[UA], s4[UA];
            const bool in = !bad && (INTERLEAVED ? e < half : e < rot);  // a table may have no row at all
            if (in) {
                load_units<float, UA>(cr + at, c4);
                load_units<float, UA>(sr + at, s4);
            }
#pragma unroll
            for (int k = 0; k < UA; ++k) {
                cs[i + k] = in ? __uint_as_float(c4[k]) : 1.f;
                // half layout, first half: a cos - b sin = a cos + b (-sin), bit for bit
                sn[i + k] = in ? __uint_as_float(s4[k] ^ (!INTERLEAVED && e < half ? 0x80000000u : 0u)) : 0.f;
            }
        }
    }
    const int e0 = 16 * b;
    // U == 8: the heads of an iteration (a contiguous run of the token's row) come through a ring of the warp's own in shared
    // memory, three iterations ahead, whatever their kind; else every lane loads for itself.
    constexpr bool kRing = U == 8;
    constexpr int kChunk = 32 * kSlice, D = kApStages;  // elements of an iteration at most
    extern __shared__ __align__(16) uint8_t smem[];
    T* const ring = reinterpret_cast<T*>(smem) + warp * (D * kChunk);
    const int sub = warp & (wpt - 1);  // of the token's warps; iterations are dealt to them in turn
    const int total = a.iters[0] + a.iters[1] + a.iters[2];
    constexpr int kPer = 16 / (int)sizeof(T);
    const int run = hpi * d;  // elements of an iteration
    int ahead = sub, kind = -1, kind_end = 0, to = 0, at = 0, left = 0;
    const T* from = nullptr;
    auto find_kind = [&] {  // where iteration `ahead` finds its heads, and how many elements of the kind are left from there (of this lane's pieces on)
        if (ahead >= total) return;
        while (ahead >= kind_end) kind_end += a.iters[++kind];
        const int first = (ahead - (kind_end - a.iters[kind])) * hpi;
        from = static_cast<const T*>(a.src[kind]) + t * a.ld_src[kind] + (int64_t)first * d + lane * kPer;
        left = (a.heads[kind] - first) * d - lane * kPer;
    };
    auto fetch_next = [&] {
        if (ahead < total) {
            const int n = min(left, run - lane * kPer);
            T* const dst = ring + to + lane * kPer;
#pragma unroll
            for (int i = 0; i < kChunk; i += 32 * kPer)
                if (i < n) cp_async16(dst + i, from + i);
            ahead += wpt;
            from += wpt * run;
            left -= wpt * run;
            if (ahead >= kind_end) find_kind();
        }
        cp_async_commit();
        to = to + kChunk == D * kChunk ? 0 : to + kChunk;
    };
    if constexpr (kRing) {
        find_kind();
#pragma unroll
        for (int i = 0; i + 1 < D; ++i) fetch_next();
    }
    // All heads of one kind (0: queries, 1: keys, 2: values), `before` iterations into the token's work.
    auto heads_of = [&](auto kind, int before) {
        constexpr int KIND = decltype(kind)::value;
        const int n = a.heads[KIND], step = wpt * hpi;
        int h = ((sub - before) & (wpt - 1)) * hpi + hl;
        const bool mine = hl < hpi, turns = KIND < 2 && rot && e0 < rot;
        const T* x = static_cast<const T*>(a.src[KIND]) + t * a.ld_src[KIND] + (int64_t)h * d;
        T* y = static_cast<T*>(a.dst[KIND]) + (KIND == 0 ? t * a.ld_q : t * ((int64_t)n * d)) + (int64_t)h * d + e0;
#pragma unroll 1
        for (; h - hl < n; h += step, x += (int64_t)step * d, y += (int64_t)step * d) {
            const T* head = ring + at + hl * d;
            if constexpr (kRing) {
                fetch_next();
                cp_async_wait<D - 1>();
                __syncwarp();  // every lane's pieces are in place
                at = at + kChunk == D * kChunk ? 0 : at + kChunk;
            }
            if (mine && h < n) {
                uint32_t u[kSlice];
#pragma unroll
                for (int i = 0; i < kSlice; i += U) {
                    if constexpr (kRing) shared_units(head + e0 + i, u + i);
                    else load_units<T, U>(x + e0 + i, u + i);
                }
                if (turns) {
                    if constexpr (INTERLEAVED) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (8 * b + i < half) {
                                const float p = __uint_as_float(u[2 * i]), q = __uint_as_float(u[2 * i + 1]);
                                u[2 * i] = __float_as_uint(__fsub_rn(__fmul_rn(p, cs[i]), __fmul_rn(q, sn[i])));
                                u[2 * i + 1] = __float_as_uint(__fadd_rn(__fmul_rn(q, cs[i]), __fmul_rn(p, sn[i])));
                            }
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < kSlice; i += U) {
                            const int e = e0 + i;
                            if (e < rot) {
                                uint32_t v[U];
                                const int from = e < half ? e + half : e - half;
                                if constexpr (kRing) shared_units(head + from, v);
                                else load_units<T, U>(x + from, v);
#pragma unroll
                                for (int k = 0; k < U; ++k)
                                    u[i + k] = __float_as_uint(__fadd_rn(__fmul_rn(__uint_as_float(u[i + k]), cs[i + k]), __fmul_rn(__uint_as_float(v[k]), sn[i + k])));
                            }
                        }
                    }
                }
                if (KIND < 2 && bad) {
#pragma unroll
                    for (int i = 0; i < kSlice; ++i) u[i] = 0x7FC00000u;
                }
                if constexpr (KIND == 0) {
                    if constexpr (sizeof(T) == 2) {  // round to the tensor's type
                        uint32_t w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const __nv_bfloat162 p = __floats2bfloat162_rn(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
                            w[i] = *reinterpret_cast<const uint32_t*>(&p);
                        }
                        if constexpr (U == 8) {
                            store_block(y, w, a.wide[0]);
                        } else if constexpr (U == 4) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) reinterpret_cast<uint2*>(y)[i] = make_uint2(w[2 * i], w[2 * i + 1]);
                        } else {
#pragma unroll
                            for (int i = 0; i < kSlice; ++i) reinterpret_cast<uint16_t*>(y)[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
                        }
                    } else if constexpr (U >= 4) {
                        store_block(y, u, a.wide[0]);
                    } else {
                        store_slice_guarded(y, 1, kSlice, u);
                    }
                } else {
                    uint32_t yb[kSlice];
                    pack_block_to(a, KIND - 1, slot, h * nb + b, u, yb, store);
                    if (a.dst[KIND]) store_values(y, yb, a.wide[KIND]);  // 16-byte aligned
                }
            }
            if (KIND > 0 && store && a.pad[KIND == 2] && h == hl) pad_lines(a, KIND - 1, slot, lane);
            if constexpr (kRing) __syncwarp();  // the next copies may overwrite the heads
        }
    };
    heads_of(std::integral_constant<int, 0>{}, 0);
    heads_of(std::integral_constant<int, 1>{}, a.iters[0]);
    heads_of(std::integral_constant<int, 2>{}, a.iters[0] + a.iters[1]);
    if constexpr (kRing) cp_async_wait<0>();
}

template <typename T>
static int launch_append(const AppendArgs& a, int unit, bool interleaved, cudaStream_t st) {
    const int64_t tokens_per_cta = kApWarps / a.warps_per_token;
    const unsigned grid = (unsigned)((a.n_tokens + tokens_per_cta - 1) / tokens_per_cta);
    constexpr int kRingBytes = kApWarps * kApStages * 32 * kSlice * (int)sizeof(T);
    static PerDevice once, once_inter;
    if (kernel_setup(once, mx_kv_append_kernel<T, 8, false>, kApThreads, kRingBytes) < 1) return BDR_ERR_CUDA;
    if (kernel_setup(once_inter, mx_kv_append_kernel<T, 8, true>, kApThreads, kRingBytes) < 1) return BDR_ERR_CUDA;
#define BDR_APPEND(U, BYTES)                                                                   \
    (interleaved ? mx_kv_append_kernel<T, U, true><<<grid, kApThreads, BYTES, st>>>(a)         \
                 : mx_kv_append_kernel<T, U, false><<<grid, kApThreads, BYTES, st>>>(a))
    if (unit == 8) BDR_APPEND(8, kRingBytes);
    else if (unit == 4) BDR_APPEND(4, 0);
    else BDR_APPEND(1, 0);
#undef BDR_APPEND
    return cudaGetLastError() == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

// What mx_kv_append and mx_attn_decode need of a cache description (host).
int check_kv_cache(const mx_kv_cache_t* c) {
    if (!c) return BDR_ERR_NULL;
    for (const bdr_config_t* cfg : {&c->cfg_k, &c->cfg_v}) {
        const int rc = check_table2_config(cfg);
        if (rc) return rc;
        if (cfg->rounding != BDR_ROUND_NEAREST_EVEN) return BDR_ERR_UNSUPPORTED;
    }
    if (c->n_pages < 0 || c->page_size < 1 || c->n_kv < 1 || c->head_dim < 1) return BDR_ERR_SIZE;
    if (c->n_pages > ((1ll << 31) - 64) / c->page_size || c->n_kv > 65535) return BDR_ERR_SIZE;
    if (c->head_dim % 16 || c->head_dim > 256) return BDR_ERR_UNSUPPORTED;
    for (const bdr_planes_t* p : {&c->k, &c->v})
        if (p->ld_exps > INT32_MAX || p->ld_micro > INT32_MAX || p->ld_elems > INT32_MAX) return BDR_ERR_SIZE;
    if (c->n_pages == 0) return BDR_OK;
    const int64_t line = (int64_t)c->n_kv * c->head_dim;
    const int rc = check_table2_planes(&c->cfg_k, &c->k, line);
    return rc ? rc : check_table2_planes(&c->cfg_v, &c->v, line);
}

}  // namespace bdr

using namespace bdr;

extern "C" int mx_kv_append(const mx_kv_cache_t* cache, const void* k, int64_t ldk, const void* v, int64_t ldv, bdr_dtype_t dt,
                            int64_t n_tokens, const int64_t* slots, const mx_rotation_t* rot, const void* q, int64_t ldq, int32_t n_q,
                            void* q_out, int64_t ldq_out, void* k_dq, void* v_dq, void* stream) {
    int rc = check_kv_cache(cache);
    if (rc) return rc;
    if (dt != BDR_F32 && dt != BDR_BF16) return BDR_ERR_UNSUPPORTED;
    const int64_t line = (int64_t)cache->n_kv * cache->head_dim, eb = dt == BDR_F32 ? 4 : 2, d = cache->head_dim;
    if (n_tokens < 0 || n_tokens > (1ll << 30) || ldk < line || ldv < line) return BDR_ERR_SIZE;
    const bool rotate = rot && rot->rot_dim != 0;
    if (rotate) {
        if (rot->rot_dim < 0 || rot->rot_dim % 2 || rot->rot_dim > d || rot->n_pos < 0 || rot->ld < rot->rot_dim / 2) return BDR_ERR_SIZE;
    }
    if (q && (n_q < 1 || n_q > 65535 || ldq < n_q * d || ldq_out < n_q * d)) return BDR_ERR_SIZE;
    if (q && q == q_out) return BDR_ERR_UNSUPPORTED;
    if (n_tokens == 0) return BDR_OK;
    if (!k || !v || !slots || (q && !q_out)) return BDR_ERR_NULL;
    if (rotate && (!rot->positions || (rot->n_pos > 0 && (!rot->cos || !rot->sin)))) return BDR_ERR_NULL;
    if ((uintptr_t)slots % 8 || (rotate && (uintptr_t)rot->positions % 8)) return BDR_ERR_MISALIGNED;
    if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)q | (uintptr_t)q_out) % eb) return BDR_ERR_MISALIGNED;
    if (rotate && ((uintptr_t)rot->cos | (uintptr_t)rot->sin) % 4) return BDR_ERR_MISALIGNED;
    if (((uintptr_t)k_dq | (uintptr_t)v_dq) % 16) return BDR_ERR_MISALIGNED;
    AppendArgs a = {};
    a.status = device_status_word();
    if (!a.status) return BDR_ERR_CUDA;
    a.plane[0] = cache->k; a.plane[1] = cache->v;
    a.m[0] = cache->cfg_k.m; a.m[1] = cache->cfg_v.m;
    a.src[0] = q; a.src[1] = k; a.src[2] = v;
    a.dst[0] = q_out; a.dst[1] = k_dq; a.dst[2] = v_dq;
    a.ld_src[0] = ldq; a.ld_src[1] = ldk; a.ld_src[2] = ldv; a.ld_q = ldq_out;
    for (int i = 0; i < 3; ++i) a.wide[i] = (uintptr_t)a.dst[i] % 32 == 0 && (i > 0 || n_tokens == 1 || ldq_out * eb % 32 == 0);
    a.nb = (int)(d / 16);
    a.heads[0] = q ? n_q : 0; a.heads[1] = a.heads[2] = cache->n_kv;
    for (int i = 0; i < 2; ++i) {
        const int64_t n = line / 16;
        a.pad[i] = a.plane[i].ld_exps > n || a.plane[i].ld_micro > n || a.plane[i].ld_elems > n * 2 * (a.m[i] + 1);
    }
    const int hpi = 32 / a.nb;
    for (int i = 0; i < 3; ++i) a.iters[i] = (a.heads[i] + hpi - 1) / hpi;
    a.slots = slots;
    a.n_slots = cache->n_pages * cache->page_size;
    a.n_tokens = n_tokens;
    if (rotate) {
        a.positions = rot->positions; a.cosv = rot->cos; a.sinv = rot->sin;
        a.ld_rot = rot->ld; a.n_pos = rot->n_pos; a.rot_dim = rot->rot_dim;
    }
    // widest unit that every load and store is aligned for (the tables are read four at a time)
    const int half = a.rot_dim / 2;
    const uintptr_t bases = (uintptr_t)k | (uintptr_t)v | (uintptr_t)q | (uintptr_t)q_out;
    const int64_t pitches = n_tokens == 1 ? 0 : (ldk | ldv | (q ? ldq | ldq_out : 0)) * eb;
    const bool tables = !rotate || (((uintptr_t)rot->cos | (uintptr_t)rot->sin) % 16 == 0 && rot->ld % 4 == 0);
    auto fits = [&](int u) {
        const int64_t bytes = std::min<int64_t>(16, u * eb);
        return tables && bases % bytes == 0 && pitches % bytes == 0 && (rotate && rot->interleaved ? half % 4 == 0 : half % u == 0);
    };
    const int unit = fits(8) ? 8 : (fits(4) ? 4 : 1);
    // one warp per token once every SM has its warps; fewer tokens spread each token's heads over up to eight warps
    int wpt = 1;
    while (wpt < kApWarps && n_tokens * wpt < (int64_t)sm_count() * kApWarps) wpt *= 2;
    a.warps_per_token = wpt;
    while (1 << a.wpt_log < wpt) ++a.wpt_log;
    const bool inter = rotate && rot->interleaved;
    cudaStream_t st = (cudaStream_t)stream;
    return dt == BDR_F32 ? launch_append<float>(a, unit, inter, st) : launch_append<__nv_bfloat16>(a, unit, inter, st);
}
