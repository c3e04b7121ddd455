// Softmax cross entropy over a vocabulary, from packed hidden states A [M, K] and packed vocabulary weights W [V, K]: with l = A W^T,
//     lse_i = log sum_j exp(l_ij),   loss_i = lse_i - l_i,t_i      (rows whose target is negative do not count: loss 0, no gradient)
//     d_ij = dloss_i (exp(l_ij - lse_i) - [j = t_i]),   dA = d W,   dW = d^T A
// The logits of a batch are never stored.  Forward: the epilogue of the product reduces a row's 128 columns to their maximum and their sum of
// exponentials (fp32), which a second kernel joins; the thread that meets a row's target column writes that logit.  Backward: pieces of
// the vocabulary, each computed again, turned into d (bf16, or three bf16 parts) by the epilogue, and multiplied with W and A by the two
// products of mx_grad_gemm.cu; dA is summed over the pieces in fp32, in order.
//
// The epilogue's exponentials (one per logit and SM at a time: 16 a clock) take a tenth of the product's time at K = 4096 and run beside it.  Measured: 4096 x 32000 x
// 4096 forward, MX9/MX6 4 x 160 us = 1680 TFLOP/s and 30 us of decoding that nothing hides, MX6 on the 8-bit path 337 us = 3190 TFLOP/s; the same with d written 369 us.
#include <algorithm>

#include "mx_frag.cuh"
#include "mx_fused_f8.cuh"
#include "mx_fused_gemm.cuh"

namespace bdr {
namespace {

using fused::kRows;
using fused::Rows;

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two parts of a row, each a maximum and the sum of the exponentials of what is above it.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x), ref = m == -INFINITY ? 0.f : m;
    return make_float2(m, a.y * exp2_of((a.x - ref) * kLog2e) + b.y * exp2_of((b.x - ref) * kLog2e));
}

// GRAD: the epilogue writes d instead of a row's maxima and sums
template <bool GRAD>
struct EntropyJob {
    struct Params {
        CUtensorMap a, w;         // bf16 [M][K]; [columns of this piece][K]
        int n_items, n_long, extra, bn, tiles_m, tiles_n, band_rows, steps, splits, span;
        float* partials;
        int* counters;
        int M, cols;
        int64_t col0;             // the piece's first column
        const int64_t* targets;
        float2* parts;            // [columns / (bn / 2)][M]: maximum, sum of exp(l - maximum)
        int part0;                // the piece's first
        float* hit;               // [M]: the target's logit
        const float *lse, *dloss;
        const float* largest;     // of |dloss|, among the rows that count
        Rows d;                   // [n_parts][M][piece]
        int64_t vocab;
        int n_parts;
        fused::F8 f8;             // 8-bit operands, where they are used
        const int* gate;
        int* status;
    };
    struct Item { int steps, tm, tn, tile, split; };
    static constexpr bool b_mn = false;
    static constexpr int kSpan = 0;
    static constexpr bool kCut = true, kBack = false;
    static __device__ __forceinline__ int rows(const Params& p) { return p.M; }
    static __device__ __forceinline__ int chunks(int bn, int) { return bn / 64; }
    static __device__ __forceinline__ int chunk(int bn, int half, int i) { return half * (bn / 2) + 32 * i; }
    static __device__ __forceinline__ void prefetch(const Params& p) { prefetch_map(&p.a); prefetch_map(&p.w); }
    static __device__ __forceinline__ bool a_mn(const Item&) { return false; }
    static __device__ __forceinline__ Item item(const Params& p, int i) {
        Item it;
        const int tiles = p.tiles_m * p.tiles_n;
        it.split = i / tiles;
        it.tile = i - it.split * tiles;
        it.steps = min(p.span, p.steps - it.split * p.span);
        gemm_tile_coords(it.tile, p.tiles_m, p.tiles_n, p.band_rows, it.tm, it.tn);
        return it;
    }
    static __device__ __forceinline__ void load(const Params& p, const Item& it, int kk, int rank, uint8_t* dst, uint64_t* bar) {
        kk += it.split * p.span;
        tma_load_3d(dst, &p.a, kk * kBK, (it.tm * 2 + rank) * kRows, 0, bar);
        tma_load_3d(dst + fused::kOperandBytes, &p.w, kk * kBK, it.tn * p.bn + rank * (p.bn >> 1), 0, bar);
    }
    static __device__ __forceinline__ void load8(const Params& p, const Item& it, int kk, int rank, uint8_t* dst, uint64_t* bar) {
        tma_load_3d(dst, &p.f8.a, kk * fused::kK8, (it.tm * 2 + rank) * kRows, 0, bar);
        tma_load_3d(dst + kRows * fused::kK8, &p.f8.w, kk * fused::kK8, (it.tn * 2 + rank) * kRows, 0, bar);
        uint8_t* const sf = dst + fused::kTiles8;
        bulk_load_g2s(sf, p.f8.sf_a + ((int64_t)kk * p.f8.row_tiles_a + it.tm * 2 + rank) * 512, 512, bar);
        bulk_load_g2s(sf + 512, p.f8.sf_w + ((int64_t)kk * p.f8.row_tiles_w + it.tn * 2) * 512, 1024, bar);
    }
    static __device__ __forceinline__ int column(int half, int q) { return half * 128 + 32 * q; }

    // What a thread knows of its row, and of the columns of its half.
    struct Row {
        int64_t row0, row, at;   // of the warp, of the lane; the target's column among these
        int width, first, rows;  // columns, the first in the piece; rows of the warp that are there
        bool live, counts;
        float lse, scale;        // GRAD
        float top, sum;          // else: so far
    };
    static __device__ __forceinline__ Row begin(const Params& p, const Item& it, const fused::Epi& e) {
        Row r;
        r.row0 = (int64_t)it.tm * 256 + e.r0;
        r.row = r.row0 + e.lane;
        r.width = p.bn >> 1;
        r.first = it.tn * p.bn + e.half * r.width;
        r.rows = (int)min((int64_t)32, p.M - r.row0);
        r.live = r.row < p.M;
        const int64_t target = r.live ? p.targets[r.row] : -1;
        r.at = target - p.col0 - r.first;
        r.counts = row_counts(target, p.vocab);
        if constexpr (GRAD) {
            r.lse = r.live ? p.lse[r.row] : 0.f;
            r.scale = r.live ? p.dloss[r.row] / *p.largest : 0.f;
        } else {
            r.top = -INFINITY;
            r.sum = 0.f;
        }
        return r;
    }
    // 32 logits of every row, from column c of the half
    static __device__ __forceinline__ void take(const Params& p, const fused::Epi& e, Row& r, int c, float (&v)[32]) {
        const int n = p.cols - r.first - c;
        if constexpr (!GRAD) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = j < n ? v[j] : -INFINITY;
            if (r.at >= c && r.at < c + 32 && r.at < c + n) {
                float x = 0.f;
#pragma unroll
                for (int j = 0; j < 32; ++j) x = r.at - c == j ? v[j] : x;
                p.hit[r.row] = x;
            }
            float m = v[0];
#pragma unroll
            for (int j = 1; j < 32; ++j) m = fmaxf(m, v[j]);
            m = fmaxf(m, r.top);
            const float ref = m == -INFINITY ? 0.f : m;  // nothing yet: every term is zero (a NaN among the terms stays one)
            float s = r.sum * exp2_of((r.top - ref) * kLog2e);
#pragma unroll
            for (int j = 0; j < 32; ++j) s += exp2_of((v[j] - ref) * kLog2e);
            r.top = m;
            r.sum = s;
        } else {
            if (r.rows <= 0 || n <= 0) return;  // (the same for the whole warp)
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const float x = exp2_of((v[j] - r.lse) * kLog2e) - (r.at - c == j ? 1.f : 0.f);
                v[j] = r.counts ? r.scale * x : 0.f;
            }
            fused::store_parts(e, p.d, p.M, r.row0, r.first + c, r.rows, p.n_parts, v);
        }
    }
    static __device__ __forceinline__ void end(const Params& p, const Row& r) {
        if constexpr (!GRAD)
            if (r.live && r.first < p.cols) p.parts[(int64_t)(p.part0 + r.first / r.width) * p.M + r.row] = make_float2(r.top, r.sum);
    }
    static __device__ __forceinline__ void epilogue(const Params& p, const Item& it, const fused::Epi& e) {
        Row r = begin(p, it, e);
#pragma unroll 1
        for (int c = 0; c < r.width; c += 32) {
            __syncwarp();
            uint32_t u[32];
            tmem_ld32(e.tmem + (uint32_t)(e.half * r.width + c), u);
            float v[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(u[j]);
            take(p, e, r, c, v);
        }
        end(p, r);
    }
    static __device__ __forceinline__ void finish(const Params& p, const Item& it, const fused::Epi& e, float (&v)[4][32]) {
        Row r = begin(p, it, e);
#pragma unroll
        for (int q = 0; q < 4; ++q) take(p, e, r, 32 * q, v[q]);
        end(p, r);
    }
};

// where one chain of additions would lose bits of the logits; of the gradients' too, which lse goes with
template <bool GRAD>
struct EntropyJobInSpans : EntropyJob<GRAD> {
    static constexpr int kSpan = fused::kBackSpan;
    static constexpr bool kBack = true;
};
template <bool GRAD>
int launch_piece(const typename EntropyJob<GRAD>::Params& p, int m_a, int m_w, cudaStream_t st) {
    return fused::one_chain(m_a, m_w, p.span) ? fused::launch<EntropyJob<GRAD>>(p, st) : fused::launch<EntropyJobInSpans<GRAD>>(p, st);
}

// The loss is not the difference of lse, whose rounding would be all that is left of a small one beside large logits, but the log of the sum beside that
// of two logits, which is exact where they are near.
__device__ __forceinline__ void write_loss(float2 all, float hit, int64_t target, int64_t V, float* loss, float* lse, int* status) {
    const float above = logf(all.y);
    *lse = all.x + above;
    if (target >= V) atomicCAS(status, 0, (int)BDR_ERR_SIZE);
    *loss = target < 0 ? 0.f : (target < V ? (all.x - hit) + above : __int_as_float(0x7FC00000));
}

// Few rows: their logits come from the few-token kernel, [M][pitch] fp32.  A block reduces kChunk columns of a row as the epilogue above does, and the one
// that comes last joins the row's parts, in order (32000 columns of one row: 4 us, a launch and two trips to the L2).
constexpr int kChunk = 2048;
__global__ void __launch_bounds__(256) entropy_rows_kernel(const float* logits, int64_t pitch, int64_t V, const int64_t* targets, float2* parts, int* counters,
                                                           float* loss, float* lse, int* status) {
    asm volatile("griddepcontrol.wait;" ::: "memory");  // launched as a programmatic dependent of the product
    const int64_t row = blockIdx.y, col0 = (int64_t)blockIdx.x * kChunk;
    const float* const l = logits + row * pitch;
    float v[kChunk / 256];
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kChunk / 256; ++i) {
        const int64_t col = col0 + 256 * i + threadIdx.x;
        v[i] = col < V ? l[col] : -INFINITY;
        m = fmaxf(m, v[i]);
    }
    __shared__ float shared[2][8];
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    if ((threadIdx.x & 31) == 0) shared[0][threadIdx.x >> 5] = m;
    __syncthreads();
    for (int i = 0; i < 8; ++i) m = fmaxf(m, shared[0][i]);
    const float ref = m == -INFINITY ? 0.f : m;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kChunk / 256; ++i) s += exp2_of((v[i] - ref) * kLog2e);
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    if ((threadIdx.x & 31) == 0) shared[1][threadIdx.x >> 5] = s;
    __syncthreads();
    __shared__ int last;
    float2* const of_row = parts + row * gridDim.x;
    if (threadIdx.x == 0) {
        s = 0.f;
        for (int i = 0; i < 8; ++i) s += shared[1][i];
        of_row[blockIdx.x] = make_float2(m, s);
        __threadfence();
        last = atomicAdd(&counters[row], 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    float2 all = make_float2(-INFINITY, 0.f);
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 256) all = join(all, __ldcg(&of_row[i]));
    for (int d = 16; d; d >>= 1) all = join(all, make_float2(__shfl_down_sync(0xFFFFFFFFu, all.x, d), __shfl_down_sync(0xFFFFFFFFu, all.y, d)));
    if ((threadIdx.x & 31) == 0) {
        shared[0][threadIdx.x >> 5] = all.x;  // (what the block held there before has been read)
        shared[1][threadIdx.x >> 5] = all.y;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) all = join(all, make_float2(shared[0][i], shared[1][i]));
        const int64_t t = targets[row];
        write_loss(all, t < V && t >= 0 ? l[t] : 0.f, t, V, loss + row, lse + row, status);
    }
}

// Joins a row's maxima and sums: 32 rows per block, their pieces shared out to 32 warps, lanes along the rows as they lie (4096 rows of 250 parts: 5 us).
__global__ void __launch_bounds__(1024) entropy_join_kernel(const float2* parts, int n_parts, int64_t M, const float* hit, const int64_t* targets,
                                                            int64_t V, float* loss, float* lse, int* status) {
    asm volatile("griddepcontrol.wait;" ::: "memory");  // launched as a programmatic dependent of the product
    __shared__ float2 shared[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = (int64_t)blockIdx.x * 32 + lane;
    float2 mine = make_float2(-INFINITY, 0.f);
    if (row < M)
        for (int i = warp; i < n_parts; i += 32) mine = join(mine, parts[(int64_t)i * M + row]);
    shared[warp][lane] = mine;
    __syncthreads();
    if (warp == 0 && row < M) {
        for (int i = 1; i < 32; ++i) mine = join(mine, shared[i][lane]);
        const int64_t t = targets[row];
        write_loss(mine, t >= 0 && t < V ? hit[row] : 0.f, t, V, loss + row, lse + row, status);
    }
}

// Pieces of the vocabulary: as few as keep the decoded weights, and d, within a bound, all of about the same size.
int64_t piece_columns(int64_t V, int64_t most) {
    most = std::max<int64_t>(256, most / 256 * 256);
    const int64_t n = (V + most - 1) / most;
    return round_up((V + n - 1) / n, 256);
}
constexpr int64_t kMostWeights = 512ll << 20;   // bytes of decoded weights at a time
constexpr int64_t kMostD = 256ll << 20;         // bytes of d at a time
// Columns of a piece that are decoded, and multiplied, at a time: a large piece of long lines goes in four parts, each decoded beside the product of the one
// before (in one part and in four, in us, and in a long run: 4096 x 32000 x 4096 MX9/MX6 715 and 696, 753 both; of 2048 K MX9 386 and 389, 397 and 407;
// 2048 x 50000 x 1000 MX9/MX4 187 and 200, 161 and 168).  A part has more tiles than there are clusters, twice over.
constexpr int64_t kLeastBesideK = 4096;
int64_t part_columns(int64_t M, int64_t cols, int64_t K) {
    const int64_t part = round_up((cols + 3) / 4, 256);  // (more than there are, of fewer than 256 columns)
    return part < cols && K >= kLeastBesideK && cols * K >= 1ll << 25 && ((M + 255) / 256) * (part / 256) >= 4 * fused::kClusters / 2 ? part : cols;
}

struct EntropySpace {
    int64_t pitch_k, piece, a, w, parts, hit, flag, partials, counters, n_counters, bytes;
    EntropySpace(int64_t M, int64_t V, int64_t K) {
        pitch_k = line_pitch(K);
        piece = piece_columns(V, kMostWeights / (pitch_k * 2));
        a = 0;
        w = a + round_up(M * pitch_k * 2, 256);  // few rows: their logits instead
        parts = w + (few_rows(M, V, K) ? round_up(M * round_up(V, 64) * 4, 256) : round_up(std::min(piece, V) * pitch_k * 2, 256));
        parts = std::max(parts, fused::f8_bytes(M, std::min(piece, V), K));
        hit = parts + round_up((V + 31) / 32 * M * 8, 256);
        flag = hit + round_up(M * 4, 256);
        const int64_t tiles_m = (M + 255) / 256;
        const fused::Share share = fused::share_product(tiles_m, std::min(piece, V), 1, (K + kBK - 1) / kBK);
        partials = flag + 256;
        counters = partials + round_up(share.partial_bytes(tiles_m), 256);
        n_counters = few_rows(M, V, K) ? M : share.counters(tiles_m);
        bytes = counters + round_up(n_counters * 4, 256);
    }
};
struct EntropyGradSpace {
    int64_t pitch_k, piece, a, w, d, acc, largest, sums, f8, flag, partials, counters, n_counters, bytes;
    EntropyGradSpace(int64_t M, int64_t V, int64_t K, int n_parts) {
        pitch_k = line_pitch(K);
        piece = piece_columns(V, std::min(kMostWeights / (pitch_k * 2), kMostD / (std::max<int64_t>(M, 1) * 2 * n_parts)));
        a = 0;
        w = a + round_up(M * pitch_k * 2, 256);
        d = w + round_up(std::min(piece, V) * pitch_k * 2, 256);
        acc = d + round_up(n_parts * M * piece * 2, 256);
        largest = acc + (piece < V ? round_up(M * pitch_k * 4, 256) : 0);
        sums = largest + 256;
        f8 = sums + grad_sums_bytes(M, std::min(piece, V), K, 1);
        flag = f8 + (fused::takes_f8(4, 4, M, V, V, K) ? fused::f8_bytes(M, std::min(piece, V), K) : 0);
        const int64_t tiles_m = (M + 255) / 256;
        const fused::Share share = fused::share_product(tiles_m, std::min(piece, V), 1, (K + kBK - 1) / kBK);
        partials = flag + 256;
        counters = partials + round_up(share.partial_bytes(tiles_m), 256);
        n_counters = share.counters(tiles_m);
        bytes = counters + round_up(n_counters * 4, 256);
    }
};

constexpr int64_t kMost = 1ll << 28;  // of every size: no product of two sizes and a few bytes leaves 64 bits

template <class Params>
int set_piece(Params& p, int64_t M, int64_t K, int64_t col0, int64_t cols, int64_t pitch_k, const uint8_t* a, const uint8_t* w, bool f8) {
    p.tiles_m = (int)((M + 255) / 256);
    p.steps = (int)((K + kBK - 1) / kBK);
    if (col0 == 0) {  // (the last piece, which may be shorter, keeps the accumulator and the cut)
        const fused::Share share = fused::share_product(p.tiles_m, cols, 1, p.steps, f8);
        p.bn = share.bn;
        p.splits = share.splits;
        p.span = share.span;
    }
    p.tiles_n = (int)((cols + p.bn - 1) / p.bn);
    if (!fused::make_map(&p.a, a, K, M, 1, pitch_k, M * pitch_k, kRows) || !fused::make_map(&p.w, w, K, cols, 1, pitch_k, cols * pitch_k, p.bn / 2))
        return BDR_ERR_CUDA;
    p.n_items = p.n_long = p.tiles_m * p.tiles_n * p.splits;
    p.extra = 0;
    p.band_rows = gemm_band_rows((M + cols) * K * 2);
    p.M = (int)M;
    p.cols = (int)cols;
    p.col0 = col0;
    return BDR_OK;
}

bdr_planes_t lines_from(const bdr_planes_t& w, int64_t line) {
    bdr_planes_t p = w;
    p.exps += line * p.ld_exps;
    p.micro += line * p.ld_micro;
    p.elems += line * p.ld_elems;
    return p;
}

int check_entropy(const bdr_config_t* cfg_a, const bdr_config_t* cfg_w, int64_t M, int64_t V, int64_t K) {
    if (M < 0 || V < 1 || K < 0 || M > kMost || V > kMost || K > kMost) return BDR_ERR_SIZE;
    const int64_t tm = (M + 255) / 256, tv = (V + 255) / 256, tk = (K + 255) / 256;
    if (K == 0 || tm * std::max(tv, tk) >= (1ll << 29) || tv * tk >= (1ll << 29)) return BDR_ERR_UNSUPPORTED;
    const int rc = check_table2_config(cfg_a);
    return rc ? rc : check_table2_config(cfg_w);
}

}  // namespace

// Pieces, and the parts that are decoded at a time, over sizes from one to the largest: none is longer than what it is taken from, and all but the last
// start on a tile.
bool entropy_pieces_hold() {
    const int64_t Ms[] = {1, 255, 4096, 37632, 37633, 131072, kMost};
    const int64_t Vs[] = {1, 2, 127, 255, 256, 257, 300, 1023, 1025, 32000, 140032, 530001, kMost};
    const int64_t Ks[] = {1, 64, 1003, 4096, 131071, 131616, 1 << 22, kMost};
    for (int64_t M : Ms)
        for (int64_t V : Vs)
            for (int64_t K : Ks)
                for (int64_t piece : {EntropySpace(M, V, K).piece, EntropyGradSpace(M, V, K, 1).piece, EntropyGradSpace(M, V, K, fused::kPartsF32).piece}) {
                    if (piece < 1 || (piece < V && piece % 256)) return false;
                    for (int64_t cols : {std::min(piece, V), V - (V - 1) / piece * piece}) {  // the first, the last
                        const int64_t part = part_columns(M, cols, K);
                        if (part < 1 || part > cols || (part < cols && part % 256)) return false;
                    }
                }
    return true;
}

}  // namespace bdr

using namespace bdr;

extern "C" {

int64_t mx_cross_entropy_workspace_bytes(int64_t M, int64_t V, int64_t K) {
    if (M < 0 || V < 1 || K < 1 || M > kMost || V > kMost || K > kMost) return 0;
    return EntropySpace(M, V, K).bytes;
}

int mx_cross_entropy(const bdr_config_t* cfg_a, const bdr_planes_t* a, const bdr_config_t* cfg_w, const bdr_planes_t* w, int64_t M, int64_t V,
                     int64_t K, const int64_t* targets, float* loss, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_entropy(cfg_a, cfg_w, M, V, K);
    if (rc || M == 0) return rc;
    if ((rc = check_fused_operands(cfg_a, a, cfg_w, w, K))) return rc;
    if (!targets || !loss || !lse) return BDR_ERR_NULL;
    if ((uintptr_t)targets % 8 || ((uintptr_t)loss | (uintptr_t)lse) % 4) return BDR_ERR_MISALIGNED;
    const EntropySpace s(M, V, K);
    if (!workspace || workspace_bytes < s.bytes) return BDR_ERR_WORKSPACE;
    if ((uintptr_t)workspace % 256) return BDR_ERR_MISALIGNED;
    cudaStream_t st = (cudaStream_t)stream;
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    if (few_rows(M, V, K)) {
        __nv_bfloat16* const x = reinterpret_cast<__nv_bfloat16*>(ws + s.a);
        float* const logits = reinterpret_cast<float*>(ws + s.w);
        int* const counters = reinterpret_cast<int*>(ws + s.counters);
        float2* const parts = reinterpret_cast<float2*>(ws + s.parts);
        int* const status = device_status_word();
        if (!status) return BDR_ERR_CUDA;
        const int64_t pitch = round_up(V, 64), chunks = (V + kChunk - 1) / kChunk;
        if ((rc = decode_pair(*a, cfg_a->m, M, x, *w, cfg_w->m, 0, nullptr, K, s.pitch_k, st, nullptr, counters, s.n_counters))) return rc;
        if ((rc = mx_gemv(cfg_w, w, V, K, x, BDR_BF16, s.pitch_k, M, logits, BDR_F32, pitch, stream))) return rc;
        return launch_dependent(entropy_rows_kernel, dim3((unsigned)chunks, (unsigned)M), dim3(256), st, (const float*)logits, pitch, V, targets, parts, counters, loss, lse,
                                status);
    }
    EntropyJob<false>::Params p = {};
    p.targets = targets;
    p.vocab = V;
    p.parts = reinterpret_cast<float2*>(ws + s.parts);
    p.partials = reinterpret_cast<float*>(ws + s.partials);
    p.counters = reinterpret_cast<int*>(ws + s.counters);
    p.hit = reinterpret_cast<float*>(ws + s.hit);
    p.status = device_status_word();
    if (!p.status) return BDR_ERR_CUDA;
    __nv_bfloat16 *const wa = reinterpret_cast<__nv_bfloat16*>(ws + s.a), *const ww = reinterpret_cast<__nv_bfloat16*>(ws + s.w);
    const bool f8 = fused::takes_f8(cfg_a->m, cfg_w->m, M, V, V, K);
    const bool beside = fused::one_chain(cfg_a->m, cfg_w->m, (K + kBK - 1) / kBK);  // (else the product leaves no registers for the decoding)
    for (int64_t v = 0; v < V; v += s.piece) {
        const int64_t cols = std::min(s.piece, V - v);
        const bdr_planes_t lines = lines_from(*w, v);
        if ((rc = set_piece(p, M, K, v, cols, s.pitch_k, ws + s.a, ws + s.w, f8))) return rc;
        if (f8) {  // the bytes lie where the bf16 operands would: those are written only once the 8-bit kernel has found nothing to do
            if ((rc = fused::encode_f8(*a, cfg_a->m, M, lines, cfg_w->m, cols, 1, K, ws, reinterpret_cast<int*>(ws + s.flag), &p.f8, &p.gate, st))) return rc;
            if ((rc = fused::launch_f8<EntropyJob<false>>(p, st))) return rc;
        }
        const int64_t part = f8 || !beside ? cols : part_columns(M, cols, K);
        for (int64_t c = 0; c < cols; c += part) {
            const int64_t n = std::min(part, cols - c);
            // (with an 8-bit path in front, A's bf16 values are overwritten by the next piece's bytes)
            if ((rc = decode_pair(*a, cfg_a->m, c == 0 && (v == 0 || f8) ? M : 0, wa, lines_from(*w, v + c), cfg_w->m, n, ww + c * s.pitch_k, K, s.pitch_k, st, p.gate,
                                  p.counters, s.n_counters, c > 0)))
                return rc;
            if (part < cols && (rc = set_piece(p, M, K, v + c, n, s.pitch_k, ws + s.a, ws + s.w + c * s.pitch_k * 2, f8))) return rc;
            if ((rc = launch_piece<false>(p, cfg_a->m, cfg_w->m, st))) return rc;
            p.part0 += (int)((n + p.bn / 2 - 1) / (p.bn / 2));
        }
    }
    const int n_parts = p.part0;
    return launch_dependent(entropy_join_kernel, dim3((unsigned)((M + 31) / 32)), dim3(1024), st, (const float2*)p.parts, n_parts, M, (const float*)p.hit, targets,
                            V, loss, lse, p.status);
}

int64_t mx_cross_entropy_bwd_workspace_bytes(int64_t M, int64_t V, int64_t K, bdr_dtype_t dt) {
    if (M < 0 || V < 1 || K < 1 || M > kMost || V > kMost || K > kMost) return 0;
    return EntropyGradSpace(M, V, K, dt == BDR_F32 ? fused::kPartsF32 : 1).bytes;
}

int mx_cross_entropy_bwd(const bdr_config_t* cfg_a, const bdr_planes_t* a, const bdr_config_t* cfg_w, const bdr_planes_t* w, int64_t M, int64_t V,
                         int64_t K, const int64_t* targets, const float* lse, const float* dloss, void* da, int64_t ld_da, void* dw, int64_t ld_dw,
                         bdr_dtype_t dt, void* workspace, int64_t workspace_bytes, void* stream) {
    if (dt != BDR_F32 && dt != BDR_BF16) return BDR_ERR_UNSUPPORTED;
    int rc = check_entropy(cfg_a, cfg_w, M, V, K);
    if (rc) return rc;
    const int width = dt == BDR_F32 ? 4 : 2;
    for (int i = 0; i < 2; ++i) {
        const void* g = i ? dw : da;
        if (!g || (i == 0 && M == 0)) continue;
        if ((i ? ld_dw : ld_da) < K) return BDR_ERR_SIZE;
        if ((uintptr_t)g % width) return BDR_ERR_MISALIGNED;
    }
    cudaStream_t st = (cudaStream_t)stream;
    if (M == 0) {  // a sum over nothing
        if (dw && cudaMemset2DAsync(dw, ld_dw * width, 0, K * width, V, st) != cudaSuccess) return BDR_ERR_CUDA;
        return BDR_OK;
    }
    if (!da && !dw) return BDR_OK;
    if ((rc = check_fused_operands(cfg_a, a, cfg_w, w, K))) return rc;
    if (!targets || !lse || !dloss) return BDR_ERR_NULL;
    if ((uintptr_t)targets % 8 || ((uintptr_t)dloss | (uintptr_t)lse) % 4) return BDR_ERR_MISALIGNED;
    const int n_parts = dt == BDR_F32 ? fused::kPartsF32 : 1;
    const EntropyGradSpace s(M, V, K, n_parts);
    if (!workspace || workspace_bytes < s.bytes) return BDR_ERR_WORKSPACE;
    if ((uintptr_t)workspace % 256) return BDR_ERR_MISALIGNED;
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    EntropyJob<true>::Params p = {};
    p.targets = targets;
    p.vocab = V;
    p.lse = lse;
    p.dloss = dloss;
    p.d = fused::make_rows(ws + s.d, s.piece, false);
    p.partials = reinterpret_cast<float*>(ws + s.partials);
    p.counters = reinterpret_cast<int*>(ws + s.counters);
    p.n_parts = n_parts;
    p.status = device_status_word();
    if (!p.status) return BDR_ERR_CUDA;
    GradProducts g = {};
    g.d = reinterpret_cast<__nv_bfloat16*>(ws + s.d);
    g.a = reinterpret_cast<__nv_bfloat16*>(ws + s.a);
    g.w = reinterpret_cast<__nv_bfloat16*>(ws + s.w);
    g.M = M; g.K = K; g.pitch_d = s.piece; g.pitch_k = s.pitch_k;
    g.segs = 1; g.parts = n_parts;
    g.da = da; g.ld_da = ld_da; g.ld_dw = ld_dw;
    g.targets = targets; g.vocab = V;
    g.f32 = dt == BDR_F32;
    g.acc = s.piece < V ? reinterpret_cast<float*>(ws + s.acc) : nullptr;
    g.ld_acc = s.pitch_k;
    g.sums = reinterpret_cast<float*>(ws + s.sums);
    g.scale = p.largest = reinterpret_cast<const float*>(ws + s.largest);
    // With the equal weights of a mean the term of the target, which outweighs all others of its row, is then near -1 and rounds to less than the step of 1
    // (as 1/3891, say, it loses up to 2^-8: gradients of 4096 x 32000 x 4096 were off by 2.6e-3, now 1.9e-3, of which 1.6e-3 are their own rounding).
    const Largest largest = {dloss, targets, M, V, reinterpret_cast<float*>(ws + s.largest)};
    __nv_bfloat16 *const wa = reinterpret_cast<__nv_bfloat16*>(ws + s.a), *const ww = reinterpret_cast<__nv_bfloat16*>(ws + s.w);
    const bool f8 = fused::takes_f8(cfg_a->m, cfg_w->m, M, V, V, K);
    const bool beside = fused::one_chain(cfg_a->m, cfg_w->m, (K + kBK - 1) / kBK);  // (else the product leaves no registers for the decoding)
    for (int64_t v = 0; v < V; v += s.piece) {
        const int64_t cols = std::min(s.piece, V - v);
        const bdr_planes_t lines = lines_from(*w, v);
        const int64_t part = f8 || !beside ? cols : part_columns(M, cols, K);
        if ((rc = decode_pair(*a, cfg_a->m, v == 0 ? M : 0, wa, lines, cfg_w->m, part, ww, K, s.pitch_k, st, nullptr, p.counters, s.n_counters, false,
                              v == 0 ? &largest : nullptr)))
            return rc;
        if ((rc = set_piece(p, M, K, v, cols, s.pitch_k, ws + s.a, ws + s.w, f8))) return rc;
        if (f8) {
            if ((rc = fused::encode_f8(*a, cfg_a->m, M, lines, cfg_w->m, cols, 1, K, ws + s.f8, reinterpret_cast<int*>(ws + s.flag), &p.f8, &p.gate, st))) return rc;
            if ((rc = fused::launch_f8<EntropyJob<true>>(p, st))) return rc;
        }
        for (int64_t c = 0; c < cols; c += part) {
            const int64_t n = std::min(part, cols - c);
            if (c > 0 && (rc = decode_pair(*a, cfg_a->m, 0, wa, lines_from(*w, v + c), cfg_w->m, n, ww + c * s.pitch_k, K, s.pitch_k, st, nullptr, p.counters,
                                           s.n_counters, true)))
                return rc;
            if (part < cols && (rc = set_piece(p, M, K, v + c, n, s.pitch_k, ws + s.a, ws + s.w + c * s.pitch_k * 2, f8))) return rc;
            p.d = fused::make_rows(ws + s.d + c * 2, s.piece, false);
            if ((rc = launch_piece<true>(p, cfg_a->m, cfg_w->m, st))) return rc;
        }
        g.N = cols;
        g.dw = dw ? static_cast<char*>(dw) + v * ld_dw * width : nullptr;
        g.first = v == 0;
        g.last = v + s.piece >= V;
        if ((rc = launch_grad_products(g, st))) return rc;
    }
    return BDR_OK;
}

}  // extern "C"
