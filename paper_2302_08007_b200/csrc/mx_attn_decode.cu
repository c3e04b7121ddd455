// Entry point of mx_attn_decode: argument checks, the split of the work, and the kernel that joins the parts of sequences
// that several workers share.
#include <algorithm>
#include <cmath>

#include "bdr_async.cuh"
#include "mx_attn_decode.cuh"

namespace bdr {

int check_kv_cache(const mx_kv_cache_t* c);
template <> int launch_attn<3>(const AttnArgs&, int, int, int, bool, bool, int, cudaStream_t);
template <> int launch_attn<5>(const AttnArgs&, int, int, int, bool, bool, int, cudaStream_t);
template <> int launch_attn<8>(const AttnArgs&, int, int, int, bool, bool, int, cudaStream_t);

// One CTA per sequence and query head: sums the parts that the workers left, in the order of their positions.  A sequence
// that one worker covered is finished already; one without positions gets zeros.  The parts are dealt to the CTA's warps
// (32 lanes read a row of a part, 16 bytes each), whose sums are added in order at the end.
// Launched while the workers still run (programmatic dependent launch): what it needs of `lengths` it has read by the time
// their results are complete.
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;
template <bool F32>
__global__ void __launch_bounds__(kJoinThreads) mx_attn_join_kernel(const AttnArgs a) {
    __shared__ float2 wml[kJoinWarps];
    __shared__ __align__(16) float wo[kJoinWarps][256];
    const int b = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    using T = typename std::conditional<F32, float, __nv_bfloat16>::type;
    T* out = static_cast<T*>(a.out) + (int64_t)b * a.ldo + (int64_t)head * a.d;
    const SeqRange r = seq_range(a, b);
    int w0 = 0, w1 = -1;
    const TileCounts c = count_tiles(a, lane, b);
    const Split split(a, c.total);
    if (r.count > 0) {
        w0 = split.holder(c.prefix);
        w1 = split.holder(c.prefix + r.count - 1);
    }
    cudaGridDependencySynchronize();
    if (w0 == w1) return;
    if (r.count == 0) {
        for (int e = threadIdx.x; e < a.d; e += kJoinThreads) {
            if constexpr (F32) out[e] = 0.f;
            else out[e] = __float2bfloat16_rn(0.f);
        }
        if (threadIdx.x == 0 && a.lse) a.lse[(int64_t)b * a.n_q + head] = -INFINITY;
        return;
    }
    float m = kAtNone, l = 0.f, acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.f;
    const int rows4 = a.d / 4;  // 16-byte words of a row: at most 64
    // a lane looks up one part, then the warp adds the parts it found one by one
    for (int base = w0; base <= w1; base += kJoinThreads) {
        const int mine = base + warp + kJoinWarps * lane;
        float2 x = make_float2(kAtNone, 0.f);
        int64_t part = -1;
        if (mine <= w1) {
            part = ((int64_t)mine * 2 + (split.begin(mine) < c.prefix ? 1 : 0)) * a.n_q + head;
            x = __ldcg(a.part_ml + part);
        }
        float top = x.x;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        top = fmaxf(top, m);
        const float old = exp2_approx(m - top);
        m = top;
        l *= old;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] *= old;
        const float f = exp2_approx(x.x - m);
        float sum = x.y * f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        l += sum;
        const int count = min(32, (w1 - base - warp) / kJoinWarps + 1);
#pragma unroll 4
        for (int i = 0; i < count; ++i) {
            const int64_t row = __shfl_sync(0xFFFFFFFFu, part, i);
            const float fi = __shfl_sync(0xFFFFFFFFu, f, i);
            if (row < 0) continue;
            const float4* src = reinterpret_cast<const float4*>(a.part_o + row * a.d);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (lane + 32 * h < rows4) {
                    const float4 v = __ldcg(src + lane + 32 * h);
                    acc[4 * h] += v.x * fi;
                    acc[4 * h + 1] += v.y * fi;
                    acc[4 * h + 2] += v.z * fi;
                    acc[4 * h + 3] += v.w * fi;
                }
        }
    }
    if (lane == 0) wml[warp] = make_float2(m, l);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (lane + 32 * h < rows4)
            *reinterpret_cast<float4*>(&wo[warp][4 * (lane + 32 * h)]) = make_float4(acc[4 * h], acc[4 * h + 1], acc[4 * h + 2], acc[4 * h + 3]);
    __syncthreads();
    float mm = kAtNone, ll = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) mm = fmaxf(mm, wml[w].x);
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
        const float f = exp2_approx(wml[w].x - mm);
        ll += wml[w].y * f;
        if (threadIdx.x < a.d) v += wo[w][threadIdx.x] * f;
    }
    if (threadIdx.x < a.d) {
        v *= ll == 0.f ? 0.f : 1.f / ll;
        if constexpr (F32) out[threadIdx.x] = v;
        else out[threadIdx.x] = __float2bfloat16_rn(v);
    }
    if (threadIdx.x == 0 && a.lse) a.lse[(int64_t)b * a.n_q + head] = (mm + log2f(ll)) * 0.69314718055994531f;
}

template <bool F32>
static int launch_join(const AttnArgs& a, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.n_seqs, (unsigned)a.n_q);
    cfg.blockDim = dim3(kJoinThreads);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, mx_attn_join_kernel<F32>, a) == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

// How units, columns and warps are laid out for a cache and a number of query heads.
struct AttnPlan {
    int maxb, nt, merge, per_pass, passes, n_units, hw, tw, groups, workers;
    bool full;
};
static AttnPlan plan_attn(const mx_kv_cache_t& c, int n_q, bool f32) {
    AttnPlan p;
    const int nb = c.head_dim / 16, group = n_q / c.n_kv;
    p.maxb = nb > 8 ? 16 : 8;
    const int most = p.maxb == 8 && !f32 ? 2 : 1;  // groups of eight columns that fit in the registers
    // heads of up to 64 elements share a warp (their columns are zero for the other heads' elements): all of its lanes decode
    p.merge = std::min(8 / std::min(nb, 8), c.n_kv);
    while (p.merge > 1 && p.merge * group > 8 * most) --p.merge;
    p.nt = std::min(most, (p.merge * group + 7) / 8);
    p.passes = p.merge > 1 ? 1 : (group + 8 * p.nt - 1) / (8 * p.nt);
    p.per_pass = (group + p.passes - 1) / p.passes;
    p.n_units = (c.n_kv + p.merge - 1) / p.merge * p.passes;
    p.full = p.merge * nb == p.maxb && c.n_kv % p.merge == 0;
    const int warps = p.maxb == 8 && p.nt == 1 ? AttnShape<8, 1, false>::kWarps : AttnShape<16, 1, false>::kWarps;
    p.hw = f32 ? AttnShape<8, 1, true>::kMaxUnits : AttnShape<8, 1, false>::kMaxUnits;  // neighbouring units side by side: they share the sectors of the scale planes
    while (p.n_units % p.hw) p.hw /= 2;
    p.tw = warps / p.hw;
    p.groups = p.n_units / p.hw;
    p.workers = std::max(1, sm_count() / p.groups);
    return p;
}

}  // namespace bdr

using namespace bdr;

extern "C" {

int64_t mx_attn_decode_workspace_bytes(const mx_kv_cache_t* cache, int64_t n_seqs, int32_t n_q) {
    if (check_kv_cache(cache) || n_seqs < 0 || n_q < 1 || n_q % cache->n_kv) return 0;
    // the caller does not say which type the queries have: the larger of the two plans
    const int64_t parts = (int64_t)std::max(plan_attn(*cache, n_q, false).workers, plan_attn(*cache, n_q, true).workers) * 2 * n_q;
    return (parts * (cache->head_dim * 4 + 8) + 255) / 256 * 256;
}

int mx_attn_decode(const mx_kv_cache_t* cache, const void* q, int64_t ldq, bdr_dtype_t dt, int64_t n_seqs, int32_t n_q,
                   const int32_t* page_table, int64_t ld_table, int64_t max_pages, const int32_t* lengths, float scale, int32_t window,
                   void* out, int64_t ldo, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_kv_cache(cache);
    if (rc) return rc;
    if (dt != BDR_F32 && dt != BDR_BF16) return BDR_ERR_UNSUPPORTED;
    if (n_q < 1 || n_q % cache->n_kv || n_q > 65535) return BDR_ERR_SIZE;
    const int64_t row = (int64_t)n_q * cache->head_dim, eb = dt == BDR_F32 ? 4 : 2;
    if (n_seqs < 0 || ldq < row || ldo < row || max_pages < 0 || ld_table < max_pages || window < 0) return BDR_ERR_SIZE;
    if (max_pages > ((1ll << 31) - 4096) / cache->page_size || n_seqs > ((1ll << 31) - 1) / n_q) return BDR_ERR_SIZE;
    if (n_seqs == 0) return BDR_OK;
    if (!q || !out || !lengths || (max_pages > 0 && !page_table)) return BDR_ERR_NULL;
    if (((uintptr_t)q | (uintptr_t)out) % eb || ((uintptr_t)page_table | (uintptr_t)lengths | (uintptr_t)lse) % 4) return BDR_ERR_MISALIGNED;
    if (!workspace || workspace_bytes < mx_attn_decode_workspace_bytes(cache, n_seqs, n_q)) return BDR_ERR_WORKSPACE;
    if ((uintptr_t)workspace % 16) return BDR_ERR_MISALIGNED;
    // in base 2, and with the factor that the first way of decoding leaves out, it has to be finite as well
    if (!(std::fabs(scale) < 0x1p94f)) return BDR_ERR_BAD_CONFIG;
    const bool f32 = dt == BDR_F32;
    const AttnPlan p = plan_attn(*cache, n_q, f32);
    if (p.groups > 65535) return BDR_ERR_SIZE;
    AttnArgs a = {};
    a.status = device_status_word();
    if (!a.status) return BDR_ERR_CUDA;
    a.k = cache->k; a.v = cache->v;
    a.q = q; a.out = out; a.lse = lse; a.table = page_table; a.lengths = lengths;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + (int64_t)p.workers * 2 * n_q * cache->head_dim);
    a.ldq = ldq; a.ldo = ldo; a.ld_table = ld_table;
    a.n_seqs = (int)n_seqs; a.n_q = n_q; a.n_kv = cache->n_kv; a.group = n_q / cache->n_kv;
    a.d = cache->head_dim; a.nb = cache->head_dim / 16;
    a.merge = p.merge; a.per_pass = p.per_pass; a.passes = p.passes; a.n_units = p.n_units;
    a.hw = p.hw; a.tw = p.tw; a.workers = p.workers;
    a.n_pages = (int)cache->n_pages; a.max_pages = (int)max_pages; a.cap = (int)max_pages * cache->page_size; a.window = window;
    a.page = make_fastdiv((uint32_t)cache->page_size);
    a.by_workers = make_fastdiv((uint32_t)p.workers);
    a.inv_pass = 65536 / p.per_pass + 1;
    while (1 << a.hw_log < p.hw) ++a.hw_log;
    a.q_vec = (uintptr_t)q % (2 * eb) == 0 && (n_seqs == 1 || ldq % 2 == 0);
    a.o_vec = (uintptr_t)out % 16 == 0 && (n_seqs == 1 || ldo * eb % 16 == 0);
    a.scale2 = 2.f * scale * 1.44269504088896341f;
    a.scale2_fast = a.scale2 * frag::kFastFactor;
    if (max_pages == 0) { a.table = lengths; a.ld_table = 0; }  // never used, but read
    cudaStream_t st = (cudaStream_t)stream;
    const int wv = cache->cfg_v.m + 1;
    switch (cache->cfg_k.m) {
        case 2: rc = launch_attn<3>(a, wv, p.maxb, p.nt, f32, p.full, p.groups, st); break;
        case 4: rc = launch_attn<5>(a, wv, p.maxb, p.nt, f32, p.full, p.groups, st); break;
        default: rc = launch_attn<8>(a, wv, p.maxb, p.nt, f32, p.full, p.groups, st); break;
    }
    if (rc) return rc;
    return f32 ? launch_join<true>(a, st) : launch_join<false>(a, st);
}

}  // extern "C"
