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
// 8 M H V flops in all, bound by the matrix cores (board power), for few tokens by reading w twice and writing dw.
//
// float.  The logits of a piece go to the workspace (8 bytes of traffic against 2 H flops at a sixteenth of the bf16 rate), and
// row kernels reduce them, or turn them into dz in place.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gemm_bf16_pp.h"

namespace tpl {
namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr int64_t PIECE_BYTES = (int64_t)128 << 20;

struct LossParams {
    GemmParams g;              // A: x, B: rows of w of this piece
    PPRun run;
    const int* labels;
    int first;                 // number in the vocabulary of the piece's row 0
    // forward
    float2* part;              // [tile of columns][M]: maximum (log2 units), sum
    float* target;             // [M], written by the tile that holds a row's label
    int part0;                 // tiles of columns before this piece
    // backward
    const float* lse; const float* dloss;
    int vocab;                 // labels outside [0, vocab) are ignored
    bf16_t* dz; int ldz;       // [M, ldz], columns past the piece zero
};

// Value of accumulator column e (0..7) of unit u in a row block, see pp_row_block.
__device__ __forceinline__ float pp_col(const f32x4 (&x)[4], bool odd, int u, int e) {
    return e < 4 ? (odd ? x[2 * u + 1][e] : x[2 * u][e]) : (odd ? x[2 * u][e - 4] : x[2 * u + 1][e - 4]);
}

template <typename TL>
__device__ __forceinline__ void stats_epilogue(const LossParams& lp, const PPAcc<TL>& acc, const PPWork& w, char* smem) {
    const GemmParams& p = lp.g;
    const PPLane el = pp_lane<TL>(p, w.m0, w.n0);
    const int lane = threadIdx.x & 63, wave = pp_wave(), wn = wave % TL::WN;
    float2* red = reinterpret_cast<float2*>(smem);                 // [wavefront of columns][row of the tile]
    int label[TL::UA][4];
#pragma unroll
    for (int h = 0; h < TL::UA; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = el.row + h * TL::A_ROWS + 16 * i;
            label[h][i] = row < p.M ? lp.labels[row] - lp.first : -1;
        }
    const bool edge = w.n0 + TL::BN > p.N;                         // uniform
    __syncthreads();                                               // the loads of every wavefront have landed: LDS is free
#pragma unroll
    for (int h = 0; h < TL::UA; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = el.row + h * TL::A_ROWS + 16 * i;
            float v[16];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[8 * u + e] = pp_col(acc[h][i], el.odd, u, e);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int at = label[h][i] - el.col[u];
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
            if (lane < 16) red[wn * TL::BM + row - w.m0] = make_float2(m, s);
        }
    __syncthreads();
    const int r = threadIdx.x, row = w.m0 + r;
    if (r >= TL::BM || row >= p.M) return;
    float m = -INFINITY, s = 0.0f;
#pragma unroll
    for (int n = 0; n < TL::WN; ++n) m = fmaxf(m, red[n * TL::BM + r].x);
    const float mu = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int n = 0; n < TL::WN; ++n) s = fmaf(red[n * TL::BM + r].y, __builtin_amdgcn_exp2f(red[n * TL::BM + r].x - mu), s);
    lp.part[(int64_t)(lp.part0 + w.n0 / TL::BN) * p.M + row] = make_float2(m, s);
}

template <typename TL>
__device__ __forceinline__ void grad_epilogue(const LossParams& lp, const PPAcc<TL>& acc, const PPWork& w) {
    const GemmParams& p = lp.g;
    const PPLane el = pp_lane<TL>(p, w.m0, w.n0);
#pragma unroll
    for (int h = 0; h < TL::UA; ++h) {
        int label[4];
        float lse2[4], d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = el.row + h * TL::A_ROWS + 16 * i, at = row < p.M ? row : 0;
            label[i] = lp.labels[at];
            lse2[i] = lp.lse[at] * LOG2E;
            d[i] = lp.dloss[at];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = el.row + h * TL::A_ROWS + 16 * i;
            if (row >= p.M) continue;
            const bool known = label[i] >= 0 && label[i] < lp.vocab;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (el.col[u] >= lp.ldz) continue;
                const int at = label[i] - lp.first - el.col[u];
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float x = __builtin_amdgcn_exp2f(fmaf(pp_col(acc[h][i], el.odd, u, e), LOG2E, -lse2[i]));
                    x = (at == e ? x - 1.0f : x) * d[i];
                    v[e] = known && el.col[u] + e < p.N ? x : 0.0f;
                }
                *reinterpret_cast<uint4*>(lp.dz + (int64_t)row * lp.ldz + el.col[u]) = pack8(v);
            }
        }
    }
}

template <typename TL, bool GRAD>
__global__ __launch_bounds__(512, 2) void lm_loss_kernel(LossParams lp) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const PPWork w = pp_work<TL>(lp.g, lp.run, share_of_block(blockIdx.x, gridDim.x));
    PPAcc<TL> acc;
    pp_products<TL, true, true, false>(lp.g, w, smem, acc);
    if constexpr (GRAD) grad_epilogue<TL>(lp, acc, w);
    else stats_epilogue<TL>(lp, acc, w, smem);
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
    float m = -INFINITY;
    for (int i = threadIdx.x; i < n; i += 256) m = fmaxf(m, zr[i]);
    m = block_reduce(m, true, tmp);
    float4 old = make_float4(-INFINITY, 0.0f, -INFINITY, 0.0f);
    if (!begin) old = state[row];
    m = fmaxf(m, old.x);
    const float mu = m == -INFINITY ? 0.0f : m;
    float s = 0.0f;
    for (int i = threadIdx.x; i < n; i += 256) s += expf(zr[i] - mu);
    s = block_reduce(s, false, tmp) + old.y * expf(old.x - mu);
    if (threadIdx.x) return;
    const int64_t at = (int64_t)labels[row] - first;
    const float target = at >= 0 && at < n ? zr[at] : old.z;
    if (end) {
        stats[2 * row] = mu + logf(s);
        stats[2 * row + 1] = target;
    } else {
        state[row] = make_float4(m, s, target, 0.0f);
    }
}
__global__ __launch_bounds__(256) void lm_grad_f32_kernel(float* __restrict__ z, int ldz, int n, const int* __restrict__ labels, int64_t first, int64_t vocab,
                                                          const float* __restrict__ lse, const float* __restrict__ dloss) {
    const int64_t row = blockIdx.x;
    const int64_t label = labels[row], at = label - first;
    const bool known = label >= 0 && label < vocab;
    const float l = lse[row], d = dloss[row];
    float* zr = z + row * ldz;
    for (int i = threadIdx.x; i < ldz; i += 256) {
        float x = 0.0f;
        if (known && i < n) {
            x = expf(zr[i] - l);
            x = (i == at ? x - 1.0f : x) * d;
        }
        zr[i] = x;
    }
}

// The ranks' statistics of a token joined, and its loss.
__global__ __launch_bounds__(256) void lm_join_kernel(int64_t M, int ranks, int64_t vocab, const float2* __restrict__ stats, const int* __restrict__ labels,
                                                      float* __restrict__ loss, float* __restrict__ lse) {
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= M) return;
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
    loss[row] = labels[row] >= 0 && labels[row] < vocab ? l - target : 0.0f;
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

// The tile of the logits: the wide one for at most 128 rows, else the one whose list of tiles is over first.  us of a k-step of 32 and of
// a tile's start and end are those of the group planner (gemm_bf16.hip).
int loss_tile(int64_t M, int64_t V, int64_t H) {
    if (M <= 128) return 2;
    const double nk = (double)((H + 31) / 32), cus = compute_units();
    auto us = [&](int64_t bn, double step, double ends) { return std::ceil((double)(((M + 255) / 256) * ((V + bn - 1) / bn)) / cus) * (nk * step + ends); };
    return us(128, 0.42, 7.5) < us(256, 0.72, 8.0) ? 1 : 0;
}
int tile_columns(int tile) { return tile == 1 ? 128 : 256; }

template <typename TL, bool GRAD>
hipError_t launch_tile(LossParams lp, hipStream_t s) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&lm_loss_kernel<TL, GRAD>), hipFuncAttributeMaxDynamicSharedMemorySize, TL::LDS_BYTES);
    if (attr != hipSuccess) return attr;
    lp.g.tiles_m = (lp.g.M + TL::BM - 1) / TL::BM;
    lp.g.tiles_n = (lp.g.N + TL::BN - 1) / TL::BN;
    lp.g.band = std::min(lp.g.tiles_m, 4);                  // as the group launches: 32 tiles of an XCD as 4 rows x 8 columns
    lp.run = PPRun{0, lp.g.tiles_m * lp.g.tiles_n, lp.g.nk_total, nullptr};
    hipLaunchKernelGGL((lm_loss_kernel<TL, GRAD>), dim3((unsigned)lp.run.count), dim3(512), TL::LDS_BYTES, s, lp);
    return hipGetLastError();
}
template <bool GRAD>
hipError_t launch_logits(const LossParams& lp, int tile, hipStream_t s) {
    return tile == 2 ? launch_tile<PPTile<2, 1>, GRAD>(lp, s) : tile == 1 ? launch_tile<PPTile<4, 1>, GRAD>(lp, s) : launch_tile<PPTile<2, 2>, GRAD>(lp, s);
}
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
void products(const LmLossArgs& a, int64_t v0, int64_t n, void* dz, float* acc, GemmArgs (&g)[2]) {
    const size_t es = a.dtype == BF16 ? 2 : 4;
    const bool first = v0 == 0, last = v0 + n == a.V;
    g[0] = g[1] = GemmArgs{};
    for (GemmArgs& q : g) { q.dtype = a.dtype; q.epi = EPI_NONE; q.A = dz; q.lda = row_stride(a.dtype, n); q.N = a.H; }
    g[0].M = a.M; g[0].K = n;
    g[0].B = (const char*)a.w + v0 * a.H * es;
    g[0].C = a.dx;
    if (a.dtype == BF16 && !(first && last)) { g[0].acc = acc; g[0].acc_mode = (first ? 0 : ACC_ADD) | (last ? ACC_LAST : 0); }
    if (a.dtype == F32 && !first) g[0].resid = a.dx;
    g[1].trans_a = 1; g[1].M = n; g[1].K = a.M;
    g[1].B = a.x;
    g[1].C = (char*)a.dw + v0 * a.H * es;
}
struct LossWs { int64_t piece; size_t dz, acc, gemm, total; };
LossWs layout(int dtype, int64_t M, int64_t H, int64_t V, bool bwd) {
    LossWs w{};
    w.piece = piece_rows(dtype, M, H, V, bwd || dtype == F32);
    const size_t es = dtype == BF16 ? 2 : 4;
    size_t off = 0;
    if (dtype == BF16 && !bwd) {
        w.dz = 0;                                           // partial statistics, then the targets
        int64_t tiles = 0;
        for (int64_t v0 = 0; v0 < V; v0 += w.piece) {
            const int64_t n = std::min(w.piece, V - v0), bn = tile_columns(loss_tile(M, n, H));
            tiles += (n + bn - 1) / bn;
        }
        w.acc = up256((size_t)tiles * M * sizeof(float2));
        w.total = w.acc + up256(M * sizeof(float));
        return w;
    }
    off += up256((size_t)M * row_stride(dtype, w.piece) * es);
    w.acc = off;
    off += dtype == F32 ? up256(M * sizeof(float4)) : w.piece < V ? up256((size_t)M * H * sizeof(float)) : 0;
    w.gemm = off;
    size_t need = 0;
    LmLossArgs a{};
    a.dtype = dtype; a.M = M; a.H = H; a.V = V;
    for (int64_t v0 = 0; v0 < V; v0 += w.piece) {
        const int64_t n = std::min(w.piece, V - v0);
        if (dtype == F32) need = std::max(need, gemm_f32_workspace_bytes(M, row_stride(F32, n), H));
        if (!bwd) continue;
        GemmArgs g[2];
        products(a, v0, n, nullptr, reinterpret_cast<float*>(256), g);    // plans look at whether there is an acc, not at where
        need = std::max(need, dtype == BF16 ? gemm_bf16_group_workspace_bytes(g, 2) : gemm_f32_group_workspace_bytes(g, 2));
    }
    w.total = off + up256(need);
    return w;
}
hipError_t logits_f32(const LmLossArgs& a, const LossWs& w, int64_t v0, int64_t n) {
    GemmArgs g{};
    g.dtype = F32; g.trans_b = 1; g.M = a.M; g.N = row_stride(F32, n); g.K = a.H; g.epi = EPI_NONE;
    g.A = a.x; g.B = (const float*)a.w + v0 * a.H; g.b_rows = n; g.C = a.ws;
    g.ws = (char*)a.ws + w.gemm; g.ws_bytes = a.ws_bytes - w.gemm; g.stream = a.stream;
    return gemm_f32(g);
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
            if ((e = logits_f32(a, w, v0, n)) != hipSuccess) return e;
            hipLaunchKernelGGL(lm_stats_f32_kernel, dim3((unsigned)a.M), dim3(256), 0, a.stream, (const float*)a.ws, (int)row_stride(F32, n), (int)n, a.labels,
                               a.first + v0, v0 == 0, v0 + n == a.V, (float4*)((char*)a.ws + w.acc), a.stats);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            continue;
        }
        LossParams lp = loss_params(a, v0, n);
        const int tile = loss_tile(a.M, n, a.H);
        lp.part = (float2*)a.ws; lp.target = (float*)((char*)a.ws + w.acc); lp.part0 = tiles;
        if ((e = launch_logits<false>(lp, tile, a.stream)) != hipSuccess) return e;
        tiles += (int)((n + tile_columns(tile) - 1) / tile_columns(tile));
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
    for (int64_t v0 = 0; v0 < a.V; v0 += w.piece) {
        const int64_t n = std::min(w.piece, a.V - v0);
        if (a.dtype == F32) {
            if ((e = logits_f32(a, w, v0, n)) != hipSuccess) return e;
            hipLaunchKernelGGL(lm_grad_f32_kernel, dim3((unsigned)a.M), dim3(256), 0, a.stream, (float*)ws, (int)row_stride(F32, n), (int)n, a.labels, a.first + v0,
                               a.vocab, a.lse, a.dloss);
            e = hipGetLastError();
        } else {
            LossParams lp = loss_params(a, v0, n);
            lp.dz = (bf16_t*)ws; lp.ldz = (int)row_stride(BF16, n);
            e = launch_logits<true>(lp, loss_tile(a.M, n, a.H), a.stream);
        }
        if (e != hipSuccess) return e;
        GemmArgs g[2];
        products(a, v0, n, ws, (float*)(ws + w.acc), g);
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
