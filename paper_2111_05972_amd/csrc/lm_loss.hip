// Softmax cross entropy of a vocabulary shard for gfx950, without keeping the logits: z = x w^T with x [M, H], w [V, H].
//
//   forward   per token the log-sum-exp of its z and the z of its label, if that is in the shard
//   backward  dz = (exp(z - lse) - onehot(label)) * dloss,  dx = dz w,  dw = dz^T x
//
// bf16.  Forward is a GEMM on the tiles of gemm_bf16_pp.h whose epilogue reduces a tile of logits, still float in the accumulators,
// to a maximum and a sum of exponentials per row: 8 bytes per row and tile of columns leave the chip, and a kernel joins the tiles
// of a row in their order.  Backward works the logits out again piece by piece of the vocabulary; the epilogue turns them into dz,
// rounded to bf16 as an operand of the two products that follow, which go out as one group.  A piece of dz is at most 128 MiB, so
// that both products find it in the infinity cache; where there are several, dx is added up in float.
// What is rounded is dz divided by alpha, the largest |dloss|, and the products are multiplied by it again in float.  The dz of a label is close to
// -dloss; where dloss is one number for all (a mean over the tokens) its rounding would be one and the same factor on all of them, up to 2^-8, and no
// rounding error: against 64 bits dx and dw were 2.4 times as far off as rounding their values alone, so 1.4 times.
// (Of few tokens the labels' dz are nearly all of dx and dw, and their roundings, 2^-8 at most, do not average out: up to 1.8 times as far off at one to eight
// tokens.)
// 8 M H V flops in all, bound by the matrix cores (board power): 4096 x 12576 x 5120 forward 405 us (1.30 PFLOP/s), dz 439, dx and dw 774 (1.36 PFLOP/s).
// For few tokens bound by reading w three times and writing dw: 37 x 50257 x 4096 forward 120 us (3.4 TB/s, 197 tiles on 256 units), dz 97, dx and dw 199
// (4.1 TB/s).
//
// float.  The logits of a piece go to the workspace (8 bytes of traffic against 2 H flops at a sixteenth of the bf16 rate), and
// row kernels reduce them, or turn them into dz in place.  512 x 7631 x 1024: the products 86 and 150 us (93 and 106 TFLOP/s of the 154 that a large
// one reaches), the row kernels 7 and 10 us (the 15.6 MB of logits come from the infinity cache).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gemm_bf16_pp.h"

namespace tpl {
namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr int64_t PIECE_BYTES = (int64_t)128 << 20;

struct LossParams {
    GemmParams g;              // A: x, B: rows of w of this piece
    PPRun run[2];              // tiles whose K is whole; the last ones, cut into K shares
    const int* labels;
    int first;                 // number in the vocabulary of the piece's row 0
    // forward
    float2* part;              // [tile of columns][M]: maximum (log2 units), sum
    float* target;             // [M], written by the tile that holds a row's label
    int part0;                 // tiles of columns before this piece
    // backward
    const float* lse; const float* dloss; float* alpha;
    int own_alpha;             // alpha is worked out by the workgroups that use it, and left for the launches behind
    int vocab;                 // labels outside [0, vocab) are ignored
    bf16_t* dz; int ldz;       // [M, ldz], columns past the piece zero
};

// Value of accumulator column e (0..7) of unit u in a row block, see pp_row_block.
__device__ __forceinline__ float pp_col(const f32x4 (&x)[4], bool odd, int u, int e) {
    return e < 4 ? (odd ? x[2 * u + 1][e] : x[2 * u][e]) : (odd ? x[2 * u][e - 4] : x[2 * u + 1][e - 4]);
}

// One block of 16 rows of a wavefront (see pp_row_block): maximum (log2 units) and sum over the wavefront's columns to red[wavefront of columns]
// [row of the tile], and the target's logit.
template <typename TL>
__device__ __forceinline__ void stats_block(const LossParams& lp, const PPLane& el, const f32x4 (&x)[4], int row, int label, bool edge, int m0, float2* red) {
    const GemmParams& p = lp.g;
    float v[16];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[8 * u + e] = pp_col(x, el.odd, u, e);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int at = label - el.col[u];
        if (at >= 0 && at < 8) {
            float z = v[8 * u];
#pragma unroll
            for (int e = 1; e < 8; ++e) z = at == e ? v[8 * u + e] : z;
            if (el.col[u] + at < p.N) lp.target[row] = z;
        }
    }
    if (edge) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[8 * u + e] = el.col[u] + e < p.N ? v[8 * u + e] : -INFINITY;
    }
    float m = v[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) m = fmaxf(m, v[e]);
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64)) * LOG2E;
    const float mu = m == -INFINITY ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) s += __builtin_amdgcn_exp2f(fmaf(v[e], LOG2E, -mu));
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    if ((threadIdx.x & 63) < 16) red[pp_wave() % TL::WN * TL::BM + row - m0] = make_float2(m, s);
}
// The wavefronts' columns of a row joined, in their order.
template <typename TL>
__device__ __forceinline__ void stats_row(const LossParams& lp, int row, int m0, int n0, const float2* red) {
    float m = -INFINITY, s = 0.0f;
#pragma unroll
    for (int n = 0; n < TL::WN; ++n) m = fmaxf(m, red[n * TL::BM + row - m0].x);
    const float mu = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int n = 0; n < TL::WN; ++n) s = fmaf(red[n * TL::BM + row - m0].y, __builtin_amdgcn_exp2f(red[n * TL::BM + row - m0].x - mu), s);
    lp.part[(int64_t)(lp.part0 + n0 / TL::BN) * lp.g.M + row] = make_float2(m, s);
}
__device__ __forceinline__ int label_of(const LossParams& lp, int row) { return row < lp.g.M ? (int)((unsigned)lp.labels[row] - (unsigned)lp.first) : -1; }

template <typename TL>
__device__ __forceinline__ void stats_epilogue(const LossParams& lp, const PPAcc<TL>& acc, const PPWork& w, char* smem) {
    const PPLane el = pp_lane<TL>(lp.g, w.m0, w.n0);
    float2* red = reinterpret_cast<float2*>(smem);
    int label[TL::UA][4];
#pragma unroll
    for (int h = 0; h < TL::UA; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) label[h][i] = label_of(lp, el.row + h * TL::A_ROWS + 16 * i);
    const bool edge = w.n0 + TL::BN > lp.g.N;                      // uniform
    __syncthreads();                                               // the loads of every wavefront have landed: LDS is free
#pragma unroll
    for (int h = 0; h < TL::UA; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) stats_block<TL>(lp, el, acc[h][i], el.row + h * TL::A_ROWS + 16 * i, label[h][i], edge, w.m0, red);
    __syncthreads();
    const int row = w.m0 + threadIdx.x;
    if (threadIdx.x < TL::BM && row < lp.g.M) stats_row<TL>(lp, row, w.m0, w.n0, red);
}

// A block of 16 rows of dz.
struct RowTerms { int label; float lse2, d; };
__device__ __forceinline__ RowTerms row_terms(const LossParams& lp, int row, float alpha) {
    const int at = row < lp.g.M ? row : 0;
    return RowTerms{lp.labels[at], lp.lse[at] * LOG2E, lp.dloss[at] / alpha};
}
__device__ __forceinline__ void grad_block(const LossParams& lp, const PPLane& el, const f32x4 (&x)[4], int row, const RowTerms& r) {
    const GemmParams& p = lp.g;
    if (row >= p.M) return;
    const bool known = r.label >= 0 && r.label < lp.vocab;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (el.col[u] >= lp.ldz) continue;
        const int at = (int)((unsigned)r.label - (unsigned)lp.first) - el.col[u];
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float y = __builtin_amdgcn_exp2f(fmaf(pp_col(x, el.odd, u, e), LOG2E, -r.lse2));
            y = (at == e ? y - 1.0f : y) * r.d;
            v[e] = known && el.col[u] + e < p.N ? y : 0.0f;
        }
        *reinterpret_cast<uint4*>(lp.dz + (int64_t)row * lp.ldz + el.col[u]) = pack8(v);
    }
}
template <typename TL>
__device__ __forceinline__ void grad_epilogue(const LossParams& lp, const PPAcc<TL>& acc, const PPWork& w, float alpha) {
    const PPLane el = pp_lane<TL>(lp.g, w.m0, w.n0);
#pragma unroll
    for (int h = 0; h < TL::UA; ++h) {
        RowTerms r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = row_terms(lp, el.row + h * TL::A_ROWS + 16 * i, alpha);
#pragma unroll
        for (int i = 0; i < 4; ++i) grad_block(lp, el, acc[h][i], el.row + h * TL::A_ROWS + 16 * i, r[i]);
    }
}

// alpha = the largest |dloss| of a token that counts (1 where there is none or it is 0), by all N threads of a workgroup.
template <int N>
__device__ __forceinline__ float largest_dloss(const float* dloss, const int* labels, int64_t vocab, int64_t M, float* tmp) {
    float m = 0.0f;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < M; i += N) m = fmaxf(m, labels[i] >= 0 && labels[i] < vocab ? fabsf(dloss[i]) : 0.0f);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = m;
    __syncthreads();
    m = tmp[0];
    for (int w = 1; w < N / 64; ++w) m = fmaxf(m, tmp[w]);
    return m > 0.0f && m < INFINITY ? m : 1.0f;
}

template <typename TL, bool GRAD>
__global__ __launch_bounds__(512, 2) void lm_loss_kernel(LossParams lp) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ float own;
    if (GRAD && lp.own_alpha) {
        const float alpha = largest_dloss<512>(lp.dloss, lp.labels, lp.vocab, lp.g.M, reinterpret_cast<float*>(smem));
        if (threadIdx.x == 0) {
            own = alpha;
            if (blockIdx.x == 0) *lp.alpha = alpha;
        }
        __syncthreads();                                           // the rest of LDS is free
    }
    const int whole = lp.run[0].count, bid = blockIdx.x;
    const PPRun& run = lp.run[bid < whole ? 0 : 1];               // whole tiles first, then the K shares of the others
    const PPWork w = bid < whole ? pp_work<TL>(lp.g, run, share_of_block(bid, whole)) : pp_work<TL>(lp.g, run, share_of_block(bid - whole, gridDim.x - whole));
    PPAcc<TL> acc;
    pp_products<TL, true, true, false>(lp.g, w, smem, acc);
    if (w.partial) pp_store_partial<TL, 0>(lp.g, acc, w.m0 + pp_wave() / TL::WN * 64, w.partial);
    else if constexpr (GRAD) grad_epilogue<TL>(lp, acc, w, lp.own_alpha ? own : *lp.alpha);
    else stats_epilogue<TL>(lp, acc, w, smem);
}
// The tiles whose K was cut: the shares' sums in share order, then the epilogue.  A workgroup per block of 16 rows of a wavefront.
template <typename TL, bool GRAD>
__global__ __launch_bounds__(512) void lm_loss_sum_kernel(LossParams lp, int shares) {
    __shared__ float2 red[TL::WN * TL::BM];
    const PPRun& run = lp.run[1];
    const int local = blockIdx.x / (4 * TL::UA), block = blockIdx.x % (4 * TL::UA);
    int tm, tn;
    tile_coords(run.tile0 + local, lp.g.tiles_m, lp.g.tiles_n, lp.g.band, tm, tn);
    const int m0 = tm * TL::BM, n0 = tn * TL::BN, first = m0 + (block >> 2) * TL::A_ROWS + (block & 3) * 16;
    if (first >= lp.g.M) return;
    const PPLane el = pp_lane<TL>(lp.g, m0, n0);
    const int row = el.row + first - m0;
    f32x4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v) x[j][v] = 0.0f;
    if (__builtin_amdgcn_readfirstlane(row - (int)(threadIdx.x & 15)) < lp.g.M)          // blocks past M were not stored
        for (int s = 0; s < shares; ++s) {
            const float4* src = pp_partial(run.partial + ((int64_t)s * run.count + local) * TL::FLOATS, block);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 y = src[j * 512];
                x[j][0] += y.x; x[j][1] += y.y; x[j][2] += y.z; x[j][3] += y.w;
            }
        }
    if constexpr (GRAD) {
        grad_block(lp, el, x, row, row_terms(lp, row, *lp.alpha));
    } else {
        stats_block<TL>(lp, el, x, row, label_of(lp, row), n0 + TL::BN > lp.g.N, m0, red);
        __syncthreads();
        const int r = threadIdx.x, to = first + (r >> 4) * 64 + (r & 15);                // the rows of this block of all wavefronts
        if (r < 16 * TL::WM && to < lp.g.M) stats_row<TL>(lp, to, m0, n0, red);
    }
}

__global__ __launch_bounds__(1024) void lm_alpha_kernel(const float* __restrict__ dloss, const int* __restrict__ labels, int64_t vocab, int64_t M, float* __restrict__ alpha) {
    __shared__ float tmp[16];
    const float m = largest_dloss<1024>(dloss, labels, vocab, M, tmp);
    if (threadIdx.x == 0) alpha[0] = m;
}

// (log-sum-exp, target logit) of every token from its tiles' (maximum, sum), in tile order by 16 lanes.
__global__ __launch_bounds__(256) void lm_join_tiles_kernel(const float2* __restrict__ part, const float* __restrict__ target, const int* __restrict__ labels,
                                                            int64_t first, int64_t V, int64_t M, int tiles, float* __restrict__ stats) {
    const int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15);
    const int g = threadIdx.x >> 4;
    __shared__ float2 red[16][16];
    float m = -INFINITY, s = 0.0f;
    if (row < M)
        for (int t = g; t < tiles; t += 16) {
            const float2 x = part[(int64_t)t * M + row];
            const float n = fmaxf(m, x.x), mu = n == -INFINITY ? 0.0f : n;
            s = s * __builtin_amdgcn_exp2f(m - mu) + x.y * __builtin_amdgcn_exp2f(x.x - mu);
            m = n;
        }
    red[g][threadIdx.x & 15] = make_float2(m, s);
    __syncthreads();
    if (threadIdx.x >= 16 || row >= M) return;
    m = -INFINITY;
    for (int i = 0; i < 16; ++i) m = fmaxf(m, red[i][threadIdx.x].x);
    const float mu = m == -INFINITY ? 0.0f : m;
    s = 0.0f;
    for (int i = 0; i < 16; ++i) s = fmaf(red[i][threadIdx.x].y, __builtin_amdgcn_exp2f(red[i][threadIdx.x].x - mu), s);
    const int64_t at = (int64_t)labels[row] - first;
    stats[2 * row] = (m + log2f(s)) * LN2;
    stats[2 * row + 1] = at >= 0 && at < V ? target[row] : -INFINITY;
}

// float: a workgroup to a token and piece of logits.  state: (maximum, sum, target) so far.
__device__ __forceinline__ float block_reduce(float v, bool max, float* tmp) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max ? fmaxf(v, __shfl_xor(v, o, 64)) : v + __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    return max ? fmaxf(fmaxf(tmp[0], tmp[1]), fmaxf(tmp[2], tmp[3])) : (tmp[0] + tmp[1]) + (tmp[2] + tmp[3]);
}
__global__ __launch_bounds__(256) void lm_stats_f32_kernel(const float* __restrict__ z, int ldz, int n, const int* __restrict__ labels, int64_t first, int begin,
                                                           int end, float4* __restrict__ state, float* __restrict__ stats) {
    __shared__ float tmp[4];
    const int64_t row = blockIdx.x;
    const float* zr = z + row * ldz;
    float m = -INFINITY, s = 0.0f;                            // this thread's share of the row, in one pass
#pragma unroll 4
    for (int i = 4 * threadIdx.x; i < n; i += 1024) {
        const float4 x4 = *reinterpret_cast<const float4*>(zr + i);
        const float x[4] = {x4.x, i + 1 < n ? x4.y : -INFINITY, i + 2 < n ? x4.z : -INFINITY, i + 3 < n ? x4.w : -INFINITY};
        const float top = fmaxf(m, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]))), mu = top == -INFINITY ? 0.0f : top;
        s *= expf(m - mu);
        s += (expf(x[0] - mu) + expf(x[1] - mu)) + (expf(x[2] - mu) + expf(x[3] - mu));
        m = top;
    }
    float4 old = make_float4(-INFINITY, 0.0f, -INFINITY, 0.0f);
    if (!begin) old = state[row];
    const float top = fmaxf(block_reduce(m, true, tmp), old.x), mu = top == -INFINITY ? 0.0f : top;
    s = block_reduce(s * expf(m - mu), false, tmp) + old.y * expf(old.x - mu);
    if (threadIdx.x) return;
    const int64_t at = (int64_t)labels[row] - first;
    const float target = at >= 0 && at < n ? zr[at] : old.z;
    if (end) {
        stats[2 * row] = mu + logf(s);
        stats[2 * row + 1] = target;
    } else {
        state[row] = make_float4(top, s, target, 0.0f);
    }
}
__global__ __launch_bounds__(256) void lm_grad_f32_kernel(float* __restrict__ z, int ldz, int n, const int* __restrict__ labels, int64_t first, int64_t vocab,
                                                          const float* __restrict__ lse, const float* __restrict__ dloss) {
    const int64_t row = blockIdx.x;
    const int64_t label = labels[row], at = label - first;
    const bool known = label >= 0 && label < vocab;
    const float l = lse[row], d = dloss[row];
    float* zr = z + row * ldz;
#pragma unroll 4
    for (int i = 4 * threadIdx.x; i < ldz; i += 1024) {
        const float4 x4 = *reinterpret_cast<const float4*>(zr + i);
        float x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float p = expf(x[e] - l);
            x[e] = known && i + e < n ? (i + e == at ? p - 1.0f : p) * d : 0.0f;
        }
        *reinterpret_cast<float4*>(zr + i) = make_float4(x[0], x[1], x[2], x[3]);
    }
}

// The ranks' statistics of a token joined, and its loss.
__global__ __launch_bounds__(256) void lm_join_kernel(int64_t M, int ranks, int64_t vocab, const float2* __restrict__ stats, const int* __restrict__ labels,
                                                      float* __restrict__ loss, float* __restrict__ lse) {
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= M) return;
    const int label = labels[row];
    float m = -INFINITY, target = -INFINITY;
    for (int r = 0; r < ranks; ++r) {
        const float2 x = stats[(int64_t)r * M + row];
        m = fmaxf(m, x.x);
        target = fmaxf(target, x.y);
    }
    const float mu = m == -INFINITY ? 0.0f : m;
    float s = 0.0f;
    for (int r = 0; r < ranks; ++r) s += expf(stats[(int64_t)r * M + row].x - mu);
    const float l = mu + logf(s);
    lse[row] = l;
    loss[row] = label >= 0 && label < vocab ? l - target : 0.0f;
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
// Rows of w in a piece: forward keeps nothing of it, so only the 2 GiB that an operand may have bound it (bf16).
int64_t piece_rows(int dtype, int64_t M, int64_t H, int64_t V, bool keeps_logits) {
    const int64_t es = dtype == BF16 ? 2 : 4;
    int64_t n = std::min<int64_t>(V, 0x7FFFFFFFll / (H * es) - 8);
    if (keeps_logits) n = std::min(n, std::max<int64_t>(PIECE_BYTES / (M * es), 256));
    return n >= V ? V : std::max<int64_t>(n / 256 * 256, 8);
}
int64_t row_stride(int dtype, int64_t n) { return dtype == BF16 ? (n + 7) / 8 * 8 : (n + 3) / 4 * 4; }

// How the logits of n rows of w go out: on which tile (0: 256 x 256, 1: 256 x 128, 2: 128 x 256), and how many of its tiles, the last ones, in how many K
// shares.  At most 128 tokens: 128 x 256.  Else by the time that the list of tiles takes dealt out to the units, us of a k-step of 32 and of a
// tile's start and end as in the group planner (gemm_bf16.hip): a last round that is not full is cut where its sums cost less than it saves.
// 4096 x 12576 x 5120, 800 tiles on 256 units: 446 us uncut.
struct LossPlan { int tile, tiles, cut, shares, nk; };
constexpr int LOSS_BM[3] = {256, 256, 128}, LOSS_BN[3] = {256, 128, 256};
LossPlan loss_plan(int64_t M, int64_t n, int64_t H) {
    constexpr double STEP[3] = {0.72, 0.42, 0.55}, ENDS[3] = {9.0, 8.0, 8.0};
    const int cus = compute_units(), nk = (int)((H + DK - 1) / DK);
    LossPlan best{};
    double best_us = INFINITY;
    for (int t = M <= 128 ? 2 : 0; t < (M <= 128 ? 3 : 2); ++t) {
        const int tiles = (int)(((M + LOSS_BM[t] - 1) / LOSS_BM[t]) * ((n + LOSS_BN[t] - 1) / LOSS_BN[t])), rest = tiles % cus;
        for (int want = 1; want <= 16; ++want) {
            LossPlan p{t, tiles, 0, 1, nk};
            double us = (tiles + cus - 1) / cus * (nk * STEP[t] + ENDS[t]);
            if (want > 1) {
                p.nk = ((nk + want - 1) / want + 1) & ~1;             // two k-steps at a time
                p.shares = (nk + p.nk - 1) / p.nk;
                p.cut = rest;
                if (rest == 0 || p.shares != want || p.nk < 12) continue;
                us = tiles / cus * (nk * STEP[t] + ENDS[t]) + (rest * want + cus - 1) / cus * (p.nk * STEP[t] + ENDS[t]) +
                     6.0 + (double)rest * want * LOSS_BM[t] * LOSS_BN[t] * 8.0 / 8.0e6;
            }
            if (us < best_us) { best_us = us; best = p; }
        }
    }
    return best;
}
size_t partial_bytes(const LossPlan& p) { return up256((size_t)p.cut * p.shares * LOSS_BM[p.tile] * LOSS_BN[p.tile] * sizeof(float)) * (p.shares > 1); }
int column_tiles(const LossPlan& p, int64_t n) { return (int)((n + LOSS_BN[p.tile] - 1) / LOSS_BN[p.tile]); }

template <typename TL, bool GRAD>
hipError_t launch_tile(LossParams lp, const LossPlan& pl, float* partial, hipStream_t s) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&lm_loss_kernel<TL, GRAD>), hipFuncAttributeMaxDynamicSharedMemorySize, TL::LDS_BYTES);
    if (attr != hipSuccess) return attr;
    lp.g.tiles_m = (lp.g.M + TL::BM - 1) / TL::BM;
    lp.g.tiles_n = (lp.g.N + TL::BN - 1) / TL::BN;
    lp.g.band = std::min(lp.g.tiles_m, 4);                  // as the group launches: 32 tiles of an XCD as 4 rows x 8 columns
    lp.run[0] = PPRun{0, pl.tiles - pl.cut, lp.g.nk_total, nullptr};
    lp.run[1] = PPRun{pl.tiles - pl.cut, pl.cut, pl.nk, partial};
    hipLaunchKernelGGL((lm_loss_kernel<TL, GRAD>), dim3((unsigned)(lp.run[0].count + pl.cut * pl.shares)), dim3(512), TL::LDS_BYTES, s, lp);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pl.cut == 0) return e;
    hipLaunchKernelGGL((lm_loss_sum_kernel<TL, GRAD>), dim3((unsigned)(pl.cut * 4 * TL::UA)), dim3(512), 0, s, lp, pl.shares);
    return hipGetLastError();
}
template <bool GRAD>
hipError_t launch_logits(const LossParams& lp, const LossPlan& pl, void* partial, hipStream_t s) {
    float* q = (float*)partial;
    return pl.tile == 2   ? launch_tile<PPTile<2, 1>, GRAD>(lp, pl, q, s)
           : pl.tile == 1 ? launch_tile<PPTile<4, 1>, GRAD>(lp, pl, q, s)
                          : launch_tile<PPTile<2, 2>, GRAD>(lp, pl, q, s);
}
// Whether the workgroups of dz work alpha out themselves, which costs each about a microsecond, or a kernel before them, which costs 1.5 to 2 and reads
// the tokens with one workgroup: few tokens and at most two rounds of tiles (3 x 288 x 434 backward 18.5 -> 17.0 us, 55 x 3888 x 1423 36.1 -> 34.4, 500 x 11368 x 269
// 49.3 -> 47.0; with 4.5 rounds of two pieces 523 -> 534).
bool own_alpha(const LmLossArgs& a, int64_t piece) { return a.M <= 1024 && piece >= a.V && loss_plan(a.M, a.V, a.H).tiles <= 2 * compute_units(); }
LossParams loss_params(const LmLossArgs& a, int64_t v0, int64_t n) {
    LossParams lp{};
    lp.g.A = (const bf16_t*)a.x;
    lp.g.B = (const bf16_t*)a.w + v0 * a.H;
    lp.g.M = (int)a.M; lp.g.N = (int)n; lp.g.K = (int)a.H;
    lp.g.lda = lp.g.ldb = (int)a.H;
    lp.g.nk_total = (lp.g.K + DK - 1) / DK;
    lp.labels = a.labels; lp.first = (int)(a.first + v0);
    lp.lse = a.lse; lp.dloss = a.dloss; lp.vocab = (int)a.vocab;
    return lp;
}
// dx (+)= dz w and dw = dz^T x of a piece of n rows of w.
void products(const LmLossArgs& a, int64_t v0, int64_t n, void* dz, float* acc, const float* alpha, GemmArgs (&g)[2]) {
    const size_t es = a.dtype == BF16 ? 2 : 4;
    const bool first = v0 == 0, last = v0 + n == a.V;
    g[0] = g[1] = GemmArgs{};
    for (GemmArgs& q : g) { q.dtype = a.dtype; q.epi = a.dtype == BF16 ? EPI_SCALE : EPI_NONE; q.alpha = alpha; q.A = dz; q.lda = row_stride(a.dtype, n); q.N = a.H; }
    g[0].M = a.M; g[0].K = n;
    g[0].B = (const char*)a.w + v0 * a.H * es;
    g[0].C = a.dx;
    if (a.dtype == BF16 && !(first && last)) { g[0].acc = acc; g[0].acc_mode = (first ? 0 : ACC_ADD) | (last ? ACC_LAST : 0); }
    if (a.dtype == F32 && !first) g[0].resid = a.dx;
    g[1].trans_a = 1; g[1].M = n; g[1].K = a.M;
    g[1].B = a.x;
    g[1].C = (char*)a.dw + v0 * a.H * es;
}
// The logits of a piece, float: a group of one, the launch whose B may end before N (512 x 7632 x 1024: 87 us, 92 TFLOP/s, by either launch).
GemmArgs logits_f32(const LmLossArgs& a, int64_t v0, int64_t n) {
    GemmArgs g{};
    g.dtype = F32; g.trans_b = 1; g.M = a.M; g.N = row_stride(F32, n); g.K = a.H; g.epi = EPI_NONE;
    g.A = a.x; g.B = (const float*)a.w + v0 * a.H; g.b_rows = n; g.C = a.ws;
    return g;
}
struct LossWs { int64_t piece; size_t acc, alpha, gemm, total; };
LossWs layout(int dtype, int64_t M, int64_t H, int64_t V, bool bwd) {
    LossWs w{};
    w.piece = piece_rows(dtype, M, H, V, bwd || dtype == F32);
    const size_t es = dtype == BF16 ? 2 : 4;
    size_t off = 0;
    if (dtype == BF16 && !bwd) {
        // statistics of the tiles, the targets, sums of K shares
        int64_t tiles = 0;
        size_t need = 0;
        for (int64_t v0 = 0; v0 < V; v0 += w.piece) {
            const int64_t n = std::min(w.piece, V - v0);
            const LossPlan pl = loss_plan(M, n, H);
            tiles += column_tiles(pl, n);
            need = std::max(need, partial_bytes(pl));
        }
        w.acc = up256((size_t)tiles * M * sizeof(float2));
        w.gemm = w.acc + up256(M * sizeof(float));
        w.total = w.gemm + need;
        return w;
    }
    off += up256((size_t)M * row_stride(dtype, w.piece) * es);
    w.acc = off;
    off += dtype == F32 ? up256(M * sizeof(float4)) : w.piece < V ? up256((size_t)M * H * sizeof(float)) : 0;
    w.alpha = off;
    off += 256;
    w.gemm = off;
    size_t need = 0;
    LmLossArgs a{};
    a.dtype = dtype; a.M = M; a.H = H; a.V = V;
    for (int64_t v0 = 0; v0 < V; v0 += w.piece) {
        const int64_t n = std::min(w.piece, V - v0);
        if (dtype == F32) {
            const GemmArgs g = logits_f32(a, v0, n);
            need = std::max(need, gemm_f32_group_workspace_bytes(&g, 1));
        }
        if (!bwd) continue;
        GemmArgs g[2];
        products(a, v0, n, nullptr, reinterpret_cast<float*>(256), nullptr, g);    // plans look at whether there is an acc, not at where
        if (dtype == BF16) need = std::max(need, partial_bytes(loss_plan(M, n, H)));
        need = std::max(need, dtype == BF16 ? gemm_bf16_group_workspace_bytes(g, 2) : gemm_f32_group_workspace_bytes(g, 2));
    }
    w.total = off + up256(need);
    return w;
}
}  // namespace

size_t lm_loss_workspace_bytes(int dtype, int64_t M, int64_t H, int64_t V, bool bwd) { return layout(dtype, M, H, V, bwd).total; }

hipError_t lm_loss_fwd(const LmLossArgs& a) {
    const LossWs w = layout(a.dtype, a.M, a.H, a.V, false);
    hipError_t e = hipSuccess;
    int tiles = 0;
    for (int64_t v0 = 0; v0 < a.V; v0 += w.piece) {
        const int64_t n = std::min(w.piece, a.V - v0);
        if (a.dtype == F32) {
            const GemmArgs g = logits_f32(a, v0, n);
            if ((e = gemm_f32_group(&g, 1, (char*)a.ws + w.gemm, a.ws_bytes - w.gemm, a.stream)) != hipSuccess) return e;
            hipLaunchKernelGGL(lm_stats_f32_kernel, dim3((unsigned)a.M), dim3(256), 0, a.stream, (const float*)a.ws, (int)row_stride(F32, n), (int)n, a.labels,
                               a.first + v0, v0 == 0, v0 + n == a.V, (float4*)((char*)a.ws + w.acc), a.stats);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            continue;
        }
        LossParams lp = loss_params(a, v0, n);
        const LossPlan pl = loss_plan(a.M, n, a.H);
        lp.part = (float2*)a.ws; lp.target = (float*)((char*)a.ws + w.acc); lp.part0 = tiles;
        if ((e = launch_logits<false>(lp, pl, (char*)a.ws + w.gemm, a.stream)) != hipSuccess) return e;
        tiles += column_tiles(pl, n);
    }
    if (a.dtype == F32) return e;
    hipLaunchKernelGGL(lm_join_tiles_kernel, dim3((unsigned)((a.M + 15) / 16)), dim3(256), 0, a.stream, (const float2*)a.ws, (const float*)((char*)a.ws + w.acc), a.labels,
                       a.first, a.V, a.M, tiles, a.stats);
    return hipGetLastError();
}

hipError_t lm_loss_bwd(const LmLossArgs& a) {
    const LossWs w = layout(a.dtype, a.M, a.H, a.V, true);
    char* ws = (char*)a.ws;
    hipError_t e = hipSuccess;
    const bool own = a.dtype == BF16 && own_alpha(a, w.piece);
    if (a.dtype == BF16 && !own) {
        hipLaunchKernelGGL(lm_alpha_kernel, dim3(1), dim3(1024), 0, a.stream, a.dloss, a.labels, a.vocab, a.M, (float*)(ws + w.alpha));
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    for (int64_t v0 = 0; v0 < a.V; v0 += w.piece) {
        const int64_t n = std::min(w.piece, a.V - v0);
        if (a.dtype == F32) {
            const GemmArgs g = logits_f32(a, v0, n);
            if ((e = gemm_f32_group(&g, 1, (char*)a.ws + w.gemm, a.ws_bytes - w.gemm, a.stream)) != hipSuccess) return e;
            hipLaunchKernelGGL(lm_grad_f32_kernel, dim3((unsigned)a.M), dim3(256), 0, a.stream, (float*)ws, (int)row_stride(F32, n), (int)n, a.labels, a.first + v0,
                               a.vocab, a.lse, a.dloss);
            e = hipGetLastError();
        } else {
            LossParams lp = loss_params(a, v0, n);
            lp.dz = (bf16_t*)ws; lp.ldz = (int)row_stride(BF16, n); lp.alpha = (float*)(ws + w.alpha); lp.own_alpha = own;
            e = launch_logits<true>(lp, loss_plan(a.M, n, a.H), ws + w.gemm, a.stream);
        }
        if (e != hipSuccess) return e;
        GemmArgs g[2];
        products(a, v0, n, ws, (float*)(ws + w.acc), (float*)(ws + w.alpha), g);
        e = a.dtype == BF16 ? gemm_bf16_group(g, 2, ws + w.gemm, a.ws_bytes - w.gemm, a.stream) : gemm_f32_group(g, 2, ws + w.gemm, a.ws_bytes - w.gemm, a.stream);
        if (e != hipSuccess) return e;
    }
    return e;
}

hipError_t lm_loss_join(int64_t M, int64_t ranks, int64_t vocab, const float* stats, const int* labels, float* loss, float* lse, hipStream_t s) {
    hipLaunchKernelGGL(lm_join_kernel, dim3((unsigned)((M + 255) / 256)), dim3(256), 0, s, M, (int)ranks, vocab, (const float2*)stats, labels, loss, lse);
    return hipGetLastError();
}

}  // namespace tpl
