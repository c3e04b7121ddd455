// Entry point of mx_attn_decode: argument checks, the split of the work, and the kernel that joins the parts of sequences
// that several workers share.
#include <algorithm>
#include <cmath>

#include "mx_attn_decode.cuh"

namespace bdr {

int* device_status_word();
int check_kv_cache(const mx_kv_cache_t* c);
template <> int launch_attn<3>(const AttnArgs&, int, int, int, bool, int, cudaStream_t);
template <> int launch_attn<5>(const AttnArgs&, int, int, int, bool, int, cudaStream_t);
template <> int launch_attn<8>(const AttnArgs&, int, int, int, bool, int, cudaStream_t);

// One CTA per sequence and query head: sums the parts that the workers left, in the order of their positions.  A sequence
// that one worker covered is finished already; one without positions gets zeros.
constexpr int kJoinThreads = 128;
template <bool F32>
__global__ void __launch_bounds__(kJoinThreads) mx_attn_join_kernel(const AttnArgs a) {
    const int b = blockIdx.x / a.n_q, head = blockIdx.x - b * a.n_q, lane = threadIdx.x & 31;
    using T = typename std::conditional<F32, float, __nv_bfloat16>::type;
    T* out = static_cast<T*>(a.out) + (int64_t)b * a.ldo + (int64_t)head * a.d;
    const SeqRange r = seq_range(a, b);
    if (r.count == 0) {
        for (int e = threadIdx.x; e < a.d; e += kJoinThreads) {
            if constexpr (F32) out[e] = 0.f;
            else out[e] = __float2bfloat16_rn(0.f);
        }
        if (threadIdx.x == 0 && a.lse) a.lse[(int64_t)b * a.n_q + head] = -INFINITY;
        return;
    }
    const int64_t total = total_tiles(a, lane);
    int unused = 0;
    const int64_t p = walk_tiles(a, lane, b, -1, unused);
    // the last worker whose part starts at or before a tile holds it
    auto holder = [&](int64_t tile) {
        int w = (int)((tile * a.workers + a.workers - 1) / total);  // begin(w) = floor(total w / workers) <= tile
        while (w + 1 <= a.workers - 1 && worker_begin(total, w + 1, a.workers) <= tile) ++w;
        while (w > 0 && (w > a.workers - 1 || worker_begin(total, w, a.workers) > tile)) --w;
        return w;
    };
    const int w0 = holder(p), w1 = holder(p + r.count - 1);
    if (w0 == w1) return;
    float m = -INFINITY;
    for (int w = w0; w <= w1; ++w) {
        const int64_t begin = worker_begin(total, w, a.workers);
        if (begin == worker_begin(total, w + 1, a.workers)) continue;  // a worker without work
        m = fmaxf(m, a.part_ml[((int64_t)w * 2 + (begin < p ? 1 : 0)) * a.n_q + head].x);
    }
    float acc[2] = {0.f, 0.f}, l = 0.f;
    for (int w = w0; w <= w1; ++w) {
        const int64_t begin = worker_begin(total, w, a.workers);
        if (begin == worker_begin(total, w + 1, a.workers)) continue;
        const int64_t part = ((int64_t)w * 2 + (begin < p ? 1 : 0)) * a.n_q + head;
        const float2 x = a.part_ml[part];
        const float f = x.x == -INFINITY ? 1.f : exp2_approx(x.x - m);
        l += x.y * f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = threadIdx.x + i * kJoinThreads;
            if (e < a.d) acc[i] += a.part_o[part * a.d + e] * f;
        }
    }
    const float norm = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int e = threadIdx.x + i * kJoinThreads;
        if (e < a.d) {
            if constexpr (F32) out[e] = acc[i] * norm;
            else out[e] = __float2bfloat16_rn(acc[i] * norm);
        }
    }
    if (threadIdx.x == 0 && a.lse) a.lse[(int64_t)b * a.n_q + head] = (m + log2f(l)) * 0.69314718055994531f;
}

// How units, columns and warps are laid out for a cache and a number of query heads.
struct AttnPlan {
    int maxb, nt, merge, per_pass, passes, n_units, hw, groups, workers;
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
    p.hw = kAtWarps;
    while (p.n_units % p.hw) p.hw /= 2;
    p.groups = p.n_units / p.hw;
    p.workers = std::max(1, 2 * sm_count() / p.groups);
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
    if (!(std::fabs(scale) < INFINITY)) return BDR_ERR_BAD_CONFIG;
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
    a.hw = p.hw; a.tw = kAtWarps / p.hw; a.workers = p.workers;
    a.n_pages = (int)cache->n_pages; a.max_pages = (int)max_pages; a.cap = (int)max_pages * cache->page_size; a.window = window;
    a.page = make_fastdiv((uint32_t)cache->page_size);
    a.scale2 = 2.f * scale * 1.44269504088896341f;
    cudaStream_t st = (cudaStream_t)stream;
    const int wv = cache->cfg_v.m + 1;
    switch (cache->cfg_k.m) {
        case 2: rc = launch_attn<3>(a, wv, p.maxb, p.nt, f32, p.groups, st); break;
        case 4: rc = launch_attn<5>(a, wv, p.maxb, p.nt, f32, p.groups, st); break;
        default: rc = launch_attn<8>(a, wv, p.maxb, p.nt, f32, p.groups, st); break;
    }
    if (rc) return rc;
    if (f32) mx_attn_join_kernel<true><<<(unsigned)(n_seqs * n_q), kJoinThreads, 0, st>>>(a);
    else mx_attn_join_kernel<false><<<(unsigned)(n_seqs * n_q), kJoinThreads, 0, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? BDR_OK : BDR_ERR_CUDA;
}

}  // extern "C"
