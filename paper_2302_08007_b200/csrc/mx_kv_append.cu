// New keys and values into an MX-packed paged cache, with the position rotation applied on the way:
//     (a, b) -> (a cos - b sin, b cos + a sin)    for the pairs of the first rot_dim elements of every query and key head,
// then Q(.) of the keys and values along the head dimension (blocks of 16 elements, so a head's blocks are its own), and the
// three packed planes of each into the cache line of the token's slot.
//
// The rotated key goes from its fp32 sum into the quantizer without a rounding to the tensor's type in between; products and
// sums are rounded to fp32 one by one (no contraction), so the result does not depend on how a compiler fuses them.
// Streaming: a lane owns one 16-element block of a head and walks over heads of the same token, which keeps the block's
// cosines and sines in registers; its partner elements (rot_dim / 2 away) come from the same cache lines that the warp reads
// anyway.  A CTA's warps share tokens when there are few of them.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "bdr_device.cuh"
#include "bdr_host.h"
#include "mx_frag.cuh"

namespace bdr {

int* device_status_word();

constexpr int kApThreads = 256, kApWarps = kApThreads / 32;

struct AppendArgs {
    bdr_planes_t plane[2];       // keys, values
    int m[2];
    const void* src[3];          // q, k, v
    void* dst[3];                // rotated q, quantized k, quantized v (the last two contiguous; NULL = not wanted)
    int64_t ld_src[3], ld_q;
    int heads[3], iters[3];      // heads of each, and warp iterations over them
    const int64_t *slots, *positions;
    const float *cosv, *sinv;
    int64_t ld_rot, n_pos, n_slots, n_tokens;
    int rot_dim, nb, warps_per_token;
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

template <int W>
__device__ __forceinline__ void store_codes(uint8_t* p, const uint32_t (&u)[kSlice], const uint32_t (&rq)[kSlice],
                                            const uint32_t (&cb)[kSlice / 2]) {
    uint32_t words[(kSlice * W + 31) / 32];
    pack_words<W, kSlice, 2>(u, rq, cb, words);
    if constexpr (W == 8) {
        *reinterpret_cast<uint4*>(p) = make_uint4(words[0], words[1], words[2], words[3]);
    } else {  // 10 or 6 bytes at a two-byte boundary
#pragma unroll
        for (int h = 0; h < W; ++h) *reinterpret_cast<uint16_t*>(p + 2 * h) = (uint16_t)(words[h >> 1] >> (16 * (h & 1)));
    }
}

// One block of 16 values (fp32 bits u) of the key (which = 0) or value line of a slot.
__device__ __forceinline__ void pack_block_to(const AppendArgs& a, int which, int64_t slot, int block, const uint32_t (&u)[kSlice],
                                              uint32_t (&yb)[kSlice], bool store) {
    QParams qp;
    qp.k1 = 16; qp.k2 = 2; qp.d2 = 1; qp.m = a.m[which]; qp.rounding = BDR_ROUND_NEAREST_EVEN;
    qp.beta = 1;
    qp.qmax = (1u << qp.m) - 1u;
    uint32_t ej[kSlice / 2], eb[1] = {0}, rq[kSlice], cb[kSlice / 2], tau[kSlice / 2];
    subblock_exponents<2>(u, ej);
#pragma unroll
    for (int j = 0; j < kSlice / 2; ++j) eb[0] = max(eb[0], ej[j]);
    double e2 = 0.0, s2 = 0.0;
    quantize_slice<2, kSlice, false, true, true>(u, ej, eb, qp, yb, rq, cb, tau, e2, s2);
    if (!store) return;
    const bdr_planes_t& p = a.plane[which];
    uint32_t micro = 0;
#pragma unroll
    for (int j = 0; j < kSlice / 2; ++j) micro |= tau[j] << j;
    p.exps[slot * p.ld_exps + block] = (uint8_t)(eb[0] >> 23);
    p.micro[slot * p.ld_micro + block] = (uint8_t)micro;
    uint8_t* codes = p.elems + slot * p.ld_elems;
    switch (qp.m) {
        case 2: store_codes<3>(codes + block * 6, u, rq, cb); break;
        case 4: store_codes<5>(codes + block * 10, u, rq, cb); break;
        default: store_codes<8>(codes + block * 16, u, rq, cb); break;
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
__global__ void __launch_bounds__(kApThreads) mx_kv_append_kernel(const AppendArgs a) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int wpt = a.warps_per_token;
    const int64_t t = (int64_t)blockIdx.x * (kApWarps / wpt) + warp / wpt;
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
            if (lane == 0) atomicCAS(a.status, 0, (int)BDR_ERR_SIZE);
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
            const bool in = INTERLEAVED ? e < half : e < rot;
            if (in) {
                load_units<float, UA>(cr + at, c4);
                load_units<float, UA>(sr + at, s4);
            }
#pragma unroll
            for (int k = 0; k < UA; ++k) {
                cs[i + k] = in ? __uint_as_float(c4[k]) : 1.f;
                sn[i + k] = in ? __uint_as_float(s4[k]) : 0.f;
            }
        }
    }
    const int total = a.iters[0] + a.iters[1] + a.iters[2];
    for (int it = warp % wpt; it < total; it += wpt) {
        const int kind = it < a.iters[0] ? 0 : (it < a.iters[0] + a.iters[1] ? 1 : 2);
        const int first = kind == 0 ? it : (kind == 1 ? it - a.iters[0] : it - a.iters[0] - a.iters[1]);
        const int h = first * hpi + hl;
        if (hl < hpi && h < a.heads[kind]) {
            const T* x = static_cast<const T*>(a.src[kind]) + t * a.ld_src[kind] + (int64_t)h * d;
            uint32_t u[kSlice];
#pragma unroll
            for (int i = 0; i < kSlice; i += U) load_units<T, U>(x + 16 * b + i, u + i);
            if (rot && kind < 2) {
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
                        const int e = 16 * b + i;
                        if (e < rot) {
                            uint32_t v[U];
                            load_units<T, U>(x + (e < half ? e + half : e - half), v);
#pragma unroll
                            for (int k = 0; k < U; ++k) {
                                const float own = __fmul_rn(__uint_as_float(u[i + k]), cs[i + k]);
                                const float other = __fmul_rn(__uint_as_float(v[k]), sn[i + k]);
                                u[i + k] = __float_as_uint(e < half ? __fsub_rn(own, other) : __fadd_rn(own, other));
                            }
                        }
                    }
                }
            }
            if (kind < 2 && bad) {
#pragma unroll
                for (int i = 0; i < kSlice; ++i) u[i] = 0x7FC00000u;
            }
            if (kind == 0) {
                T* y = static_cast<T*>(a.dst[0]) + t * a.ld_q + (int64_t)h * d + 16 * b;
                if constexpr (sizeof(T) == 2) {  // round to the tensor's type
#pragma unroll
                    for (int i = 0; i < kSlice; ++i)
                        u[i] = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(__uint_as_float(u[i]))) << 16;
                }
                if constexpr (U >= 4) {
                    if constexpr (U == 8 || sizeof(T) == 4) {
                        store_slice_vec(y, u);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            reinterpret_cast<uint2*>(y)[i] = make_uint2((u[4 * i] >> 16) | u[4 * i + 1], (u[4 * i + 2] >> 16) | u[4 * i + 3]);
                    }
                } else {
                    store_slice_guarded(y, 1, kSlice, u);
                }
            } else {
                uint32_t yb[kSlice];
                pack_block_to(a, kind - 1, slot, h * nb + b, u, yb, store);
                if (a.dst[kind]) {
                    T* y = static_cast<T*>(a.dst[kind]) + (t * a.heads[1] + h) * d + 16 * b;  // 16-byte aligned
                    store_slice_vec(y, yb);
                }
            }
        }
        if (store && kind > 0 && first == 0) pad_lines(a, kind - 1, slot, lane);
    }
}

template <typename T>
static int launch_append(const AppendArgs& a, int unit, bool interleaved, cudaStream_t st) {
    const int64_t tokens_per_cta = kApWarps / a.warps_per_token;
    const unsigned grid = (unsigned)((a.n_tokens + tokens_per_cta - 1) / tokens_per_cta);
#define BDR_APPEND(U)                                                                          \
    (interleaved ? mx_kv_append_kernel<T, U, true><<<grid, kApThreads, 0, st>>>(a)             \
                 : mx_kv_append_kernel<T, U, false><<<grid, kApThreads, 0, st>>>(a))
    if (unit == 8) BDR_APPEND(8);
    else if (unit == 4) BDR_APPEND(4);
    else BDR_APPEND(1);
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
    if (rotate && (!rot->cos || !rot->sin || !rot->positions)) return BDR_ERR_NULL;
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
    a.nb = (int)(d / 16);
    a.heads[0] = q ? n_q : 0; a.heads[1] = a.heads[2] = cache->n_kv;
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
    const bool inter = rotate && rot->interleaved;
    cudaStream_t st = (cudaStream_t)stream;
    return dt == BDR_F32 ? launch_append<float>(a, unit, inter, st) : launch_append<__nv_bfloat16>(a, unit, inter, st);
}
