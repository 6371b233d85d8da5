// bf16 softmax attention of packed sequences with grouped heads for gfx950, forward and backward, head sizes that are a multiple
// of 8 up to 128 (DH: rounded up to 32, 64, 96, 128; columns past dh read as zero and are not stored).
//
// qkv [M, (nq + 2 nkv) dh], columns (q | k | v, head, dh); o [M, nq dh]; lse, dsum [M, nq] float.  Rows of a key head are flattened
// (attn_packed.h): everything below is attention of one key head with len * G query rows.  Softmax is computed in one pass over the
// keys with a running reference point and sum; backward works the probabilities out again from LSE.
//
// Layouts are those of attn_bf16.hip: forward and dQ compute the transposed score tile (lane = query row), dK/dV the untransposed
// one (lane = key), tiles of 64 rows go global -> LDS directly and are requested a step ahead.  Here every tile has a descriptor of
// its own that starts at the tile and ends with the sequence: rows of the next sequence read zero whatever is in them, and no offset
// grows with the length, so the rows of a batch may be any number of bytes.  A tile of Q and dO holds flattened rows; their
// addresses come from a division by G of a number below 64 + G, one multiplication.
//
// Precision.  Probabilities and dS are rounded to bf16 as matrix operands, at every head size (attn_bf16.hip keeps them float at head sizes other than 64
// and 128): each is off by at most 2^-8 of itself, and these roundings have no common sign.  Sums, statistics and D are float.
// Against 64 bits o and dqkv are 1.4 times as far off as their rounding alone.
//
// Infinities and NaN in masked places.  Zero times infinity is NaN, so a masked row of V (K; Q, dO) in the tile that the diagonal
// crosses would reach rows that do not see it.  A wavefront that ends with a value that is not finite computes its rows again, row by
// row, where a masked row is not read (attn_rows.h): only causal, as without a mask every row is seen.
//
// Every result is summed in a fixed order by one workgroup, or in chunk order where a strip was cut: no atomics.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_frag.h"
#include "attn_packed_dev.h"
#include "attn_rows.h"
#include "device_math.h"
#include "kernels.h"
#include "lds_dma.h"

namespace tpl {
namespace {

using Params = PackParams<bf16_t>;
using BStrip = Strip<bf16_t>;

// 64 rows of K or V from row `row0` on: the descriptor begins there and ends with the sequence.
__device__ __forceinline__ i32x4 tile_rsrc(const bf16_t* base, int64_t ld, int row0, int rows, int dh) {
    const int left = rows - row0 < PACK_TILE ? rows - row0 : PACK_TILE;
    return make_rsrc(base + row0 * ld, left > 0 ? (unsigned)(((left - 1) * ld + dh) * 2) : 0u);
}
// The loads of a tile of flattened rows of Q (and dO): position i of this thread is chunk `c` of row `row` of the tile.
template <int DH, int NT> struct FlatTile {
    static constexpr int N = NCHUNKS<DH, NT>;
    int row[N];
    unsigned col[N];              // byte in the row, HEAD_OOB past the head size
    __device__ __forceinline__ void init(int dh, int t) {
        constexpr int NC = DH / 8;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = t + NT * i;
            row[i] = at / NC;
            const int c = (at % NC) ^ swz<DH>(row[i]);
            col[i] = c * 8 < dh ? (unsigned)c * 16u : HEAD_OOB;
        }
    }
    // flattened rows 64 qt ... of a tensor whose queries have row stride ld into the LDS tile at `lds`; zeros past the sequence
    __device__ __forceinline__ void load(const Params& p, const BStrip& s, const bf16_t* base, int64_t ld, int qt, unsigned lds, int wave) const {
        const int r0 = qt * PACK_TILE, q0 = r0 / p.G, skip = r0 - q0 * p.G;          // uniform
        const int left = min(s.it.len - q0, (PACK_TILE - 1 + skip) / p.G + 1);       // queries of the tile
        const i32x4 r = make_rsrc(base + q0 * ld, left > 0 ? (unsigned)((left - 1) * ld * 2) + (unsigned)(p.G * p.dh * 2) : 0u);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((i + 1) * NT <= PACK_TILE * DH / 8 || i * NT + wave * 64 < PACK_TILE * DH / 8) {
                const unsigned x = (unsigned)(row[i] + skip), q = x * p.div_g >> 16, g = x - q * (unsigned)p.G;
                const bool in = (int)q < left && col[i] != HEAD_OOB;
                buffer_load_lds_b128(r, lds + (unsigned)(i * NT + wave * 64) * 16u, in ? q * (unsigned)(ld * 2) + g * (unsigned)(p.dh * 2) + col[i] : HEAD_OOB);
            }
    }
};
// The rows that a wavefront keeps in registers, 32 of a strip's 128, come through LDS too, two tiles at `strip`: loads of a lane's own row touch 32 lines of
// 128 bytes each, and every line four times (16 sequences of 512, 16 / 2 heads of 128: dQ waited 5.3 us of 14 to a strip for Q and dO, so 3.2; backward
// 145 -> 139 us, 120.8 -> 113.0 with 256 to a sequence; sequences of 16 tokens with heads of 64 take 9 % longer, the rest within 2 %).
template <int DH> __device__ __forceinline__ void strip_frags(bf16x8 (&f)[DH / 16], unsigned strip, int quarter, int lane) {
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) f[ks] = lds_frag_k<0>(strip + (quarter >> 1) * tile_bytes<DH>() + frag_k_off<DH>((quarter & 1) * 32, ks, lane));
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) settle(f[ks]);
}

// ---- forward ----------------------------------------------------------------------------------------------------------
// Workgroup = (128 flattened rows, key head), four wavefronts of 32 rows each, two workgroups to a unit; K and V in tiles of 64 through two LDS
// stages.  Bound by what the products, the softmax and the LDS reads of a step take one after another: 16384 tokens in 3 documents, 12 / 4 heads of 128, causal
// 389 us, 971 TFLOP/s (a library product of 8192^3 reaches 1370 to 1600); 12 documents of 8192 tokens, 16 / 2 heads 87 us.  Eight wavefronts, two to 32 rows with half of each tile's keys, halve the chain of dependent steps but read K and V by rows twice:
// where a unit has one strip they took -5 to +10 % of the time, where it has two up to 38 % more (4096 tokens of 32 to 800, 16 / 2 heads of 128).
constexpr int WAVES4 = 256;
template <int DH> constexpr int fwd_lds() { return 4 * tile_bytes<DH>(); }

template <int DH, bool CAUSAL>
__global__ __launch_bounds__(WAVES4, 2) void attn_packed_fwd_kernel(Params p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int TB = tile_bytes<DH>(), NF = DH / 16, NT = DH / 32, HALF = 32 * DH * 2;
    constexpr int NCH = NCHUNKS<DH, WAVES4>;
    BStrip s;
    if (!take_strip(p, 0, blockIdx.x, s)) return;
    const int t = threadIdx.x, lane = t & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int r0 = s.it.first + wave * 32, r = r0 + (lane & 31), len = s.it.len;
    const bool valid = r < s.rows;
    const Row me = row_of(p, valid ? r : s.rows - 1);
    const int q_lo = (int)((unsigned)min(r0, s.rows - 1) / (unsigned)p.G), q_hi = (int)((unsigned)min(r0 + 31, s.rows - 1) / (unsigned)p.G);
    const float c2 = LOG2E * p.scale;

    f32x16 oacc[NT];
#pragma unroll
    for (int dt = 0; dt < NT; ++dt) oacc[dt] = zero16();
    float m = -INFINITY, lsum = 0.0f;

    const int kv_end = r0 >= s.rows ? 0 : CAUSAL ? q_hi + 1 : len;    // keys that any row of this wavefront sees
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_void_ptr)smem;
    unsigned off[NCH];
    dma_offsets<DH, WAVES4>(off, s.ld, p.dh, t);
    auto fetch_tile = [&](int kt, unsigned stage) {
        tile_dma<DH, WAVES4>(tile_rsrc(s.k, s.ld, kt * PACK_TILE, len, p.dh), stage, off, 0, wave);
        tile_dma<DH, WAVES4>(tile_rsrc(s.v, s.ld, kt * PACK_TILE, len, p.dh), stage + TB, off, 0, wave);
    };
    unsigned ka[NF], va[NT][2];
#pragma unroll
    for (int ks = 0; ks < NF; ++ks) { ka[ks] = lds0 + frag_k_off<DH>(0, ks, lane); keep_in_register(ka[ks]); }
#pragma unroll
    for (int dt = 0; dt < NT; ++dt)
#pragma unroll
        for (int g = 0; g < 2; ++g) { va[dt][g] = lds0 + TB + frag_t_off<DH>(dt * 32, 0, g, lane); keep_in_register(va[dt][g]); }
    fetch_tile(s.it.tile0, lds0);
    FlatTile<DH, WAVES4> ft;
    ft.init(p.dh, t);
    for (int j = 0; j < 2; ++j) ft.load(p, s, s.q, s.ld, s.it.first / PACK_TILE + j, lds0 + (2 + j) * TB, wave);
    dma_wait();
    __syncthreads();
    bf16x8 qf[NF];
    strip_frags<DH>(qf, lds0 + 2 * TB, wave, lane);
    __syncthreads();                                              // the second stage is free
    auto step = [&](int kt, auto stg) __attribute__((always_inline)) {
        constexpr int SOFF = decltype(stg)::value * 2 * TB;
        if (kt + 1 < s.it.tile1) fetch_tile(kt + 1, lds0 + (1 - decltype(stg)::value) * 2 * TB);
        const int kv0 = kt * PACK_TILE;
        if (kv0 < kv_end) {                                       // wavefront-uniform
            f32x16 x[2] = {zero16(), zero16()};
            bf16x8 fr[2 * NF];                                    // keys 0..31 and 32..63 in turn, a chain of products each
#pragma unroll
            for (int ks = 0; ks < NF; ++ks) {
                fr[2 * ks] = lds_frag_k<SOFF>(ka[ks]);
                fr[2 * ks + 1] = lds_frag_k<SOFF + HALF>(ka[ks]);
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int ks = 0; ks < NF; ++ks) {
#pragma unroll
                for (int n = 0; n < 2; ++n) x[n] = MFMA(fr[2 * ks + n], qf[ks], x[n]);
            }
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int dt = 0; dt < NT; ++dt) {                     // [16 rows][dt]
                fr[dt] = lds_frag_t<SOFF>(va[dt][0], va[dt][1]);
                fr[NT + dt] = lds_frag_t<SOFF + HALF / 2>(va[dt][0], va[dt][1]);
                fr[2 * NT + dt] = lds_frag_t<SOFF + HALF>(va[dt][0], va[dt][1]);
                fr[3 * NT + dt] = lds_frag_t<SOFF + HALF + HALF / 2>(va[dt][0], va[dt][1]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (kv0 + PACK_TILE > len || (CAUSAL && kv0 + PACK_TILE - 1 > q_lo)) {
                const int seen = min(CAUSAL ? me.q : len, len - 1) - kv0 - half * 4;      // last key this row sees
#pragma unroll
                for (int g = 0; g < 2; ++g)
#pragma unroll
                    for (int v = 0; v < 16; ++v) x[g][v] = 32 * g + (v >> 2) * 8 + (v & 3) <= seen ? x[g][v] : -INFINITY;
            }
            float mb = fmaxf(x[0][0], x[1][0]);
#pragma unroll
            for (int v = 1; v < 16; ++v) mb = fmaxf(fmaxf(mb, x[0][v]), x[1][v]);
            mb = cross_half_max(mb) * c2;                         // c2 > 0: scaling commutes with max
            // The reference point moves only when the maximum has grown by more than RESCALE_LAG (log2 units): any reference point
            // gives the same result up to rounding, and weights reach 2^RESCALE_LAG at most.
            const float mn = (mb - m > RESCALE_LAG) ? mb : m;     // false for NaN (-inf - -inf): m stays
            const float mu = mn == -INFINITY ? 0.0f : mn;
            const float alpha = fast_exp2(m - mu);
            m = mn;
            float ps[2] = {0.0f, 0.0f};
#pragma unroll
            for (int v = 0; v < 16; ++v)
#pragma unroll
                for (int g = 0; g < 2; ++g) { x[g][v] = fast_exp2(fmaf(x[g][v], c2, -mu)); ps[g] += x[g][v]; }
            lsum = lsum * alpha + (ps[0] + ps[1]);
            if (__any(alpha != 1.0f)) {
#pragma unroll
                for (int dt = 0; dt < NT; ++dt)
#pragma unroll
                    for (int v = 0; v < 16; ++v) oacc[dt][v] *= alpha;
            }
            bf16x8 pb[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) pb[n] = pack_regs(x[n >> 1], 8 * (n & 1));
            __builtin_amdgcn_s_setprio(1);
            auto add = [&](int n0) __attribute__((always_inline)) {
#pragma unroll
                for (int n = n0; n < n0 + 2; ++n)
#pragma unroll
                    for (int dt = 0; dt < NT; ++dt) oacc[dt] = MFMA(fr[n * NT + dt], pb[n], oacc[dt]);
            };
            add(0);
            if (!CAUSAL || kv0 + 32 <= q_hi) add(2);   // uniform
            __builtin_amdgcn_s_setprio(0);
        }
        dma_wait();
        __syncthreads();
    };
    for (int kt = s.it.tile0; kt < s.it.tile1;) {
        step(kt, std::integral_constant<int, 0>{});
        if (++kt >= s.it.tile1) break;
        step(kt, std::integral_constant<int, 1>{});
        ++kt;
    }
    lsum += __shfl_xor(lsum, 32, 64);
    const bool whole = s.it.slot < 0;
    float* part = whole ? nullptr : p.part[0] + ((int64_t)s.it.slot * p.nkv + s.hk) * (PACK_BLK * (DH + 2));
    const int rl = wave * 32 + (lane & 31);
    float z = 0.0f;
    if (!whole) {
        // one chunk of a strip: (reference point, sum, O not divided by it) of its keys, float, [row][dh]
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v4[4] = {oacc[dt][4 * i], oacc[dt][4 * i + 1], oacc[dt][4 * i + 2], oacc[dt][4 * i + 3]};
                if (CAUSAL) note4(z, v4);
                store_f4(part + rl * DH + dt * 32 + 8 * i + 4 * half, v4[0], v4[1], v4[2], v4[3]);
            }
        if (half == 0) { part[PACK_BLK * DH + rl] = m; part[PACK_BLK * DH + PACK_BLK + rl] = lsum; }
    } else if (valid) {
        const float inv = 1.0f / lsum;                            // a row sees itself at least: 0 only by underflow or NaN
        bf16_t* op = p.o + (s.it.t0 + me.q) * s.ldo + (int64_t)(s.hk * p.G + me.g) * p.dh;
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v4[4] = {oacc[dt][4 * i] * inv, oacc[dt][4 * i + 1] * inv, oacc[dt][4 * i + 2] * inv, oacc[dt][4 * i + 3] * inv};
                if (CAUSAL) note4(z, v4);
                if (dt * 32 + 8 * i + 4 * half < p.dh) store4(op + dt * 32 + 8 * i + 4 * half, v4[0], v4[1], v4[2], v4[3]);
            }
        if (half == 0) p.lse[s.row0 + (int64_t)me.q * p.nq + me.g] = (m + log2f(lsum)) * LN2;
    }
    if (!CAUSAL || !any_nonfinite(z)) return;
    rows_stored();
    float* q_s = reinterpret_cast<float*>(smem) + wave * DH;   // the ring has been read
    for (int i = r0; i < r0 + 32 && i < s.rows; ++i) {
        const Row w = row_of(p, i);
        load_row(q_s, s.q + w.q * s.ld + w.g * p.dh, p.dh, lane);
        row_loaded();
        bf16_t* op = p.o + (s.it.t0 + w.q) * s.ldo + (int64_t)(s.hk * p.G + w.g) * p.dh;
        const int il = i - s.it.first;
        float mr, lr;
        attn_row_fwd<(DH + 63) / 64>(q_s, s.k, s.v, s.ld, p.dh, s.it.tile0 * PACK_TILE, min(w.q + 1, s.it.tile1 * PACK_TILE), p.scale, whole, lane, mr, lr,
                                     [&](int d, float v) { if (whole) op[d] = (bf16_t)v; else part[il * DH + d] = v; });
        if (lane == 0) {
            if (whole) p.lse[s.row0 + (int64_t)w.q * p.nq + w.g] = mr + logf(lr);
            else { part[PACK_BLK * DH + il] = mr * LOG2E; part[PACK_BLK * DH + PACK_BLK + il] = lr; }
        }
        row_loaded();
    }
}

// ---- D ----------------------------------------------------------------------------------------------------------------
// D = rowsum(dO * O) where a row has many keys.  O has been rounded, by up to 2^-8 of itself, and where keys are few O is as large as V, so that
// the difference dP - D loses half of its digits (error of dQ and dK against 64 bits with correctly rounded ones = 1: 2.3 for sequences of 2 tokens, 1.8 for 8,
// 1.5 for 64, 1.43 for 512).  Rows of at most 64 keys, a tile, therefore get D = rowsum(P * dP), the same sum from unrounded terms: two of the three
// products of dQ, for the strips that begin with such rows.  Workgroups [0, strips) walk those, the others the rows.  Bound by memory: 18 us for the
// 67 MB of O and dO of 8192 tokens of 16 heads of 128 in 12 documents, 25 us where all of 128 sequences have 64 tokens.
template <int DH> constexpr int dsum_lds() { return 2 * tile_bytes<DH>(); }
template <int DH, bool CAUSAL>
__global__ __launch_bounds__(WAVES4, 2) void attn_packed_dsum_kernel(Params p, int strips) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int TB = tile_bytes<DH>(), NF = DH / 16, HALF = 32 * DH * 2, NCH = NCHUNKS<DH, WAVES4>;
    const PackHeader* h = reinterpret_cast<const PackHeader*>(p.plan + p.header);
    if (!pack_matches(h, p.sequences, p.M, p.nq, p.nkv, p.causal)) return;
    if ((int)blockIdx.x >= strips) {
        dsum_rows(p, (int64_t)(blockIdx.x - strips) * 16, (int64_t)(gridDim.x - strips) * 16, PACK_TILE);
        return;
    }
    const int t = threadIdx.x, lane = t & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_void_ptr)smem;
    const float c2 = LOG2E * p.scale;
    const int all = (h->items[0] - h->first_short[0]) * p.nkv;
    for (int i = blockIdx.x; i < all; i += strips) {
        BStrip s;
        s.it = pack_items(p.plan, p.items[0])[h->first_short[0] + i / p.nkv];
        if (CAUSAL ? s.it.tile1 > 2 || s.it.first >= PACK_TILE * p.G : s.it.len > PACK_TILE) continue;   // uniform; such a strip is not cut
        set_strip(p, i % p.nkv, s);
        const int len = s.it.len, r = s.it.first + wave * 32 + (lane & 31);
        const bool valid = r < s.rows;
        const Row me = row_of(p, valid ? r : s.rows - 1);
        const bf16_t* dobase = p.d_o + s.it.t0 * s.ldo + (int64_t)s.hk * p.G * p.dh;
        const int64_t at = s.row0 + (int64_t)me.q * p.nq + me.g;
        const float l2 = p.lse[at] * LOG2E;
        unsigned off[NCH];
        dma_offsets<DH, WAVES4>(off, s.ld, p.dh, t);
        tile_dma<DH, WAVES4>(tile_rsrc(s.k, s.ld, 0, len, p.dh), lds0, off, 0, wave);
        tile_dma<DH, WAVES4>(tile_rsrc(s.v, s.ld, 0, len, p.dh), lds0 + TB, off, 0, wave);
        bf16x8 qf[NF], dof[NF];
#pragma unroll
        for (int ks = 0; ks < NF; ++ks) {
            qf[ks] = frag_k_global(s.q + me.q * s.ld + me.g * p.dh, 0, 0, 1, p.dh, ks, lane);
            dof[ks] = frag_k_global(dobase + me.q * s.ldo + me.g * p.dh, 0, 0, 1, p.dh, ks, lane);
        }
#pragma unroll
        for (int ks = 0; ks < NF; ++ks) { settle(qf[ks]); settle(dof[ks]); }
        dma_wait();
        __syncthreads();
        f32x16 x[2] = {zero16(), zero16()}, dp[2] = {zero16(), zero16()};
#pragma unroll
        for (int ks = 0; ks < NF; ++ks) {
            const unsigned ka = lds0 + frag_k_off<DH>(0, ks, lane);
            x[0] = MFMA(lds_frag_k<0>(ka), qf[ks], x[0]);
            x[1] = MFMA(lds_frag_k<HALF>(ka), qf[ks], x[1]);
            dp[0] = MFMA(lds_frag_k<TB>(ka), dof[ks], dp[0]);
            dp[1] = MFMA(lds_frag_k<TB + HALF>(ka), dof[ks], dp[1]);
        }
        const int seen = min(CAUSAL ? me.q : len, len - 1) - half * 4;
        float d = 0.0f;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                d += 32 * g + (v >> 2) * 8 + (v & 3) <= seen ? fast_exp2(fmaf(x[g][v], c2, -l2)) * dp[g][v] : 0.0f;
        d += __shfl_xor(d, 32, 64);
        if (valid && half == 0 && (!CAUSAL || me.q < PACK_TILE)) p.dsum[at] = d;
        __syncthreads();                                          // the next strip's tiles
    }
}

// The rows of a wavefront again, one by one (see the head of the file).
template <int DH, bool DK_ROLE>
__device__ __forceinline__ void dkv_rows_again(float* k_s, const Params& p, const BStrip& s, int k0, int lane) {
    constexpr int NA = (DH + 63) / 64;
    const int len = s.it.len, G = p.G;
    const bool whole = s.it.slot < 0;
    const bf16_t* dobase = p.d_o + s.it.t0 * s.ldo + (int64_t)s.hk * G * p.dh;
    float* part = whole ? nullptr : p.part[1] + ((int64_t)s.it.slot * p.nkv + s.hk) * (2 * PACK_BLK * DH) + (DK_ROLE ? 0 : PACK_BLK * DH);
    const int64_t col = (int64_t)(p.nq + (DK_ROLE ? 0 : p.nkv) + s.hk) * p.dh;
    const int last = min(s.rows, s.it.tile1 * PACK_TILE);
    for (int j = k0; j < k0 + 32 && j < len; ++j) {
        load_row(k_s, s.k + j * s.ld, p.dh, lane);
        load_row(k_s + DH, s.v + j * s.ld, p.dh, lane);
        row_loaded();
        float sum[NA] = {};
        for (int i = max(j * G, s.it.tile0 * PACK_TILE); i < last; ++i) {          // a row after another: this is no common case
            const Row w = row_of(p, i);
            const bf16_t* qp = s.q + w.q * s.ld + w.g * p.dh;
            const bf16_t* dp = dobase + w.q * s.ldo + w.g * p.dh;
            float a = 0.0f, b = 0.0f, q[NA], g[NA];
#pragma unroll
            for (int n = 0; n < NA; ++n) {
                const int d = lane + 64 * n;
                q[n] = d < p.dh ? to_f32(qp[d]) : 0.0f;
                g[n] = d < p.dh ? to_f32(dp[d]) : 0.0f;
                if (d < p.dh) { a = fmaf(q[n], k_s[d], a); b = fmaf(g[n], k_s[DH + d], b); }
            }
            const float pr = expf(row_sum(a) * p.scale - p.lse[s.row0 + (int64_t)w.q * p.nq + w.g]);
            const float ds = pr * (row_sum(b) - p.dsum[s.row0 + (int64_t)w.q * p.nq + w.g]);
#pragma unroll
            for (int n = 0; n < NA; ++n) sum[n] = DK_ROLE ? fmaf(ds, q[n], sum[n]) : fmaf(pr, g[n], sum[n]);
        }
#pragma unroll
        for (int n = 0; n < NA; ++n) {
            const int d = lane + 64 * n;
            if (d >= p.dh) continue;
            if (whole) p.dqkv[(s.it.t0 + j) * s.ld + col + d] = (bf16_t)(DK_ROLE ? sum[n] * p.scale : sum[n]);
            else part[(j - s.it.first) * DH + d] = sum[n];
        }
        row_loaded();
    }
}

template <int DH>
__device__ __forceinline__ void dq_rows_again(float* q_s, const Params& p, const BStrip& s, int r0, int lane) {
    const bool whole = s.it.slot < 0;
    const bf16_t* dobase = p.d_o + s.it.t0 * s.ldo + (int64_t)s.hk * p.G * p.dh;
    float* part = whole ? nullptr : p.part[0] + ((int64_t)s.it.slot * p.nkv + s.hk) * (PACK_BLK * DH);
    for (int i = r0; i < r0 + 32 && i < s.rows; ++i) {
        const Row w = row_of(p, i);
        load_row(q_s, s.q + w.q * s.ld + w.g * p.dh, p.dh, lane);
        load_row(q_s + DH, dobase + w.q * s.ldo + w.g * p.dh, p.dh, lane);
        row_loaded();
        bf16_t* dqp = p.dqkv + (s.it.t0 + w.q) * s.ld + (int64_t)(s.hk * p.G + w.g) * p.dh;
        const int64_t a = s.row0 + (int64_t)w.q * p.nq + w.g;
        attn_row_dq<(DH + 63) / 64>(q_s, q_s + DH, s.k, s.v, s.ld, p.dh, s.it.tile0 * PACK_TILE, min(w.q + 1, s.it.tile1 * PACK_TILE), p.scale, p.lse[a], p.dsum[a], lane,
                                    [&](int d, float v) { if (whole) dqp[d] = (bf16_t)(v * p.scale); else part[(i - s.it.first) * DH + d] = v; });
        row_loaded();
    }
}

// ---- dK, dV -----------------------------------------------------------------------------------------------------------
// Workgroup = (128 keys, key head), 8 wavefronts: w and w + 4 share 32 keys.  w works out scores and probabilities and accumulates
// dV; w + 4 works out dP and accumulates dK from the same probabilities, which it gets through LDS in float one sub-tile of 32 rows
// later.  Tiles of 64 flattened rows: Q, LSE and D through three stages, as dK still reads the tile before, dO through two.
// Bound by LDS: every 32 keys read the tile of Q and of dO twice, 256 KiB and 64 of P against four products of 64 x 128 x 128, and the three kinds of work
// add up: 2.75 us a tile, 0.78 PFLOP/s over the chip.  12 documents of 8192 tokens, 16 / 2 heads of 128: 334 workgroups of 128 us, before those of dQ.
constexpr int WAVES8 = 512;
constexpr int P_BYTES = 32 * 32 * 4;
template <int DH> constexpr int dkv_lds() { return 5 * tile_bytes<DH>() + 3 * 2 * PACK_TILE * 4 + 2 * 4 * P_BYTES; }
template <int DH, bool CAUSAL, bool DK_ROLE>
__device__ __forceinline__ void dkv_body(char* smem, const Params& p, const BStrip& s) {
    constexpr int TB = tile_bytes<DH>(), NF = DH / 16, NT = DH / 32, HALF = 32 * DH * 2;
    constexpr int TERMS = 5 * TB, PS = TERMS + 3 * 2 * PACK_TILE * 4;  // three Q tiles, two dO tiles, three times LSE*log2e and D, P
    const int t = threadIdx.x, lane = t & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int len = s.it.len, rows = s.rows, G = p.G;
    const int k0 = s.it.first + (wave & 3) * 32, kv = k0 + (lane & 31);
    const bf16_t* dobase = p.d_o + s.it.t0 * s.ldo + (int64_t)s.hk * G * p.dh;
    const float c2 = LOG2E * p.scale;

    f32x16 acc[NT];                                        // dK (DK_ROLE) or dV
#pragma unroll
    for (int dt = 0; dt < NT; ++dt) acc[dt] = zero16();

    const int qt0 = s.it.tile0, ntiles = s.it.tile1;
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_void_ptr)smem;
    FlatTile<DH, WAVES8> ft;
    ft.init(p.dh, t);
    float rl = 0.0f, rd = 0.0f;
    auto g2r = [&](int qt, int stage) {
        ft.load(p, s, s.q, s.ld, qt, lds0 + stage * TB, wave);
        ft.load(p, s, dobase, s.ldo, qt, lds0 + (3 + ((qt - qt0) & 1)) * TB, wave);
        if (t < PACK_TILE) {
            const int r = qt * PACK_TILE + t;
            const Row w = row_of(p, r);
            rl = r < rows ? p.lse[s.row0 + (int64_t)w.q * p.nq + w.g] * LOG2E : 0.0f;
            rd = r < rows ? p.dsum[s.row0 + (int64_t)w.q * p.nq + w.g] : 0.0f;
        }
    };
    auto r2s = [&](int stage) {
        if (t < PACK_TILE) {
            float* st = reinterpret_cast<float*>(smem + TERMS) + stage * 2 * PACK_TILE;
            st[t] = rl;
            st[PACK_TILE + t] = rd;
        }
    };
    // LDS addresses in stage 0: rows as they are (scores: Q, dP: dO), transposed (dV: dO, dK: Q), LSE or D, P.  Those into dO move between
    // its two stages from tile to tile; Q's stage is a constant of the code.
    unsigned ka[NF], ta[NT][2];
#pragma unroll
    for (int ks = 0; ks < NF; ++ks) { ka[ks] = lds0 + (DK_ROLE ? 3 * TB : 0) + frag_k_off<DH>(0, ks, lane); keep_in_register(ka[ks]); }
#pragma unroll
    for (int dt = 0; dt < NT; ++dt)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            ta[dt][g] = lds0 + (DK_ROLE ? 0 : 3 * TB) + frag_t_off<DH>(dt * 32, 0, g, lane);
            keep_in_register(ta[dt][g]);
        }
    unsigned terms = lds0 + TERMS + (DK_ROLE ? PACK_TILE * 4 : 0) + half * 16;
    char* pbuf = smem + PS + (wave & 3) * P_BYTES + lane * 16;
    g2r(qt0, 0);
    r2s(0);
    // the strip's K into the second and third stage of Q, its V into the second of dO and where P will be
    constexpr unsigned V1 = PS - 4 * TB;
    static_assert(TB <= 2 * 4 * P_BYTES, "half a strip of V fits where P will be");
    {
        unsigned off[NCHUNKS<DH, WAVES8>];
        dma_offsets<DH, WAVES8>(off, s.ld, p.dh, t);
        for (int j = 0; j < 2; ++j) {
            tile_dma<DH, WAVES8>(tile_rsrc(s.k, s.ld, s.it.first + j * PACK_TILE, len, p.dh), lds0 + (1 + j) * TB, off, 0, wave);
            tile_dma<DH, WAVES8>(tile_rsrc(s.v, s.ld, s.it.first + j * PACK_TILE, len, p.dh), lds0 + 4 * TB + j * V1, off, 0, wave);
        }
    }
    dma_wait();
    __syncthreads();
    bf16x8 own[NF];                                        // K for the scores, V for dP
    strip_frags<DH>(own, DK_ROLE ? lds0 + 4 * TB + ((wave >> 1) & 1) * (V1 - TB) : lds0 + TB, wave & 3, lane);
    __syncthreads();                                       // those stages are free

    // rows that see one of this wavefront's keys, in scalar registers: with the products in the loop it spilled
    const int see_lo = __builtin_amdgcn_readfirstlane(CAUSAL ? k0 * G - 31 : 0), see_hi = __builtin_amdgcn_readfirstlane(k0 < len ? rows : 0);
    unsigned other = TB;                                   // to the other stage of dO
    f32x16 x;                                              // scores, then P; or dP, then dS
    bool pending = false;                                  // dP of the sub-tile before waits for its P
    auto product = [&](auto stg, auto sbc) __attribute__((always_inline)) {
        constexpr int OFF = (DK_ROLE ? 0 : decltype(stg)::value * TB) + decltype(sbc)::value * HALF;
        bf16x8 fr[NF];
#pragma unroll
        for (int i = 0; i < NF; ++i) fr[i] = lds_frag_k<OFF>(ka[i]);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        x = zero16();
#pragma unroll
        for (int i = 0; i < NF; ++i) x = MFMA(fr[i], own[i], x);
        __builtin_amdgcn_s_setprio(0);
    };
    auto fetch_t = [&](auto stg, auto sbc, bf16x8 (&fr)[NF]) __attribute__((always_inline)) {
        constexpr int OFF = (DK_ROLE ? decltype(stg)::value * TB : 0) + decltype(sbc)::value * HALF;
#pragma unroll
        for (int k = 0; k < NF; ++k)
            fr[k] = k & 1 ? lds_frag_t<OFF + 16 * DH * 2>(ta[k >> 1][0], ta[k >> 1][1]) : lds_frag_t<OFF>(ta[k >> 1][0], ta[k >> 1][1]);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto collect = [&](const bf16x8 (&fr)[NF]) __attribute__((always_inline)) {
        const bf16x8 g[2] = {pack_regs(x, 0), pack_regs(x, 8)};
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int k = 0; k < NF; ++k) acc[k >> 1] = MFMA(fr[k], g[k & 1], acc[k >> 1]);
        __builtin_amdgcn_s_setprio(0);
    };
    auto finish_dk = [&](auto stg, auto sbc) __attribute__((always_inline)) {
        constexpr int STG = decltype(stg)::value, SB = decltype(sbc)::value;
        f32x4 pr[4], d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            pr[i] = *reinterpret_cast<const f32x4*>(pbuf + SB * 4 * P_BYTES + i * 1024);
            d[i] = lds_f4(terms + STG * 2 * PACK_TILE * 4 + SB * 128 + i * 32);
        }
        bf16x8 fr[NF];
        fetch_t(stg, sbc, fr);
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = pr[v >> 2][v & 3] * (x[v] - d[v >> 2][v & 3]);
        collect(fr);
    };
    // A sub-tile of 32 rows: all of it in the dV role; dP, after the rest of the sub-tile before, in the dK role.
    auto slot = [&](int qt, auto stg, auto sbc, auto before) __attribute__((always_inline)) {
        constexpr int STG = decltype(stg)::value, SB = decltype(sbc)::value;
        const int qs0 = qt * PACK_TILE + SB * 32;
        const bool skip = qs0 < see_lo || qs0 >= see_hi;                 // alike in both roles
        if constexpr (DK_ROLE) {
            if (pending) finish_dk(before, std::integral_constant<int, SB ^ 1>{});
            pending = !skip;
            if (!skip) product(stg, sbc);
        } else if (!skip) {
            product(stg, sbc);
            bf16x8 fr[NF];
            fetch_t(stg, sbc, fr);
            if (qs0 + 31 >= rows || k0 + 31 >= len || (CAUSAL && (k0 + 31) * G > qs0)) {   // wave-uniform: diagonal or an end
                const int from = kv < len ? (CAUSAL ? kv * G : 0) - qs0 - 4 * half : 1 << 30, to = rows - qs0 - 4 * half;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int r = 8 * (v >> 2) + (v & 3);
                    x[v] = r >= from && r < to ? x[v] : -INFINITY;                    // exp2(-inf) = 0
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 l = lds_f4(terms + STG * 2 * PACK_TILE * 4 + SB * 128 + i * 32);
                f32x4 pr;
#pragma unroll
                for (int j = 0; j < 4; ++j) pr[j] = x[4 * i + j] = fast_exp2(fmaf(x[4 * i + j], c2, -l[j]));
                *reinterpret_cast<f32x4*>(pbuf + SB * 4 * P_BYTES + i * 1024) = pr;
            }
            collect(fr);
        }
    };
    using C0 = std::integral_constant<int, 0>; using C1 = std::integral_constant<int, 1>; using C2 = std::integral_constant<int, 2>;
    auto step = [&](int qt, auto stg, auto next, auto before) __attribute__((always_inline)) {
        const bool more = qt + 1 < ntiles;
        if (more) g2r(qt + 1, decltype(next)::value);     // read for the last time before the barrier before last
        slot(qt, stg, C0{}, before);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // P; the next tile stays in flight
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        slot(qt, stg, C1{}, stg);
        if (more) r2s(decltype(next)::value);
        if constexpr (DK_ROLE) {
#pragma unroll
            for (int ks = 0; ks < NF; ++ks) ka[ks] += other;
        } else {
#pragma unroll
            for (int dt = 0; dt < NT; ++dt) { ta[dt][0] += other; ta[dt][1] += other; }
        }
        other = 0u - other;
        dma_wait();
        __syncthreads();
    };
    for (int qt = qt0; qt < ntiles;) {
        step(qt, C0{}, C1{}, C2{});
        if (++qt >= ntiles) break;
        step(qt, C1{}, C2{}, C0{});
        if (++qt >= ntiles) break;
        step(qt, C2{}, C0{}, C1{});
        ++qt;
    }
    if (DK_ROLE && pending) {
        const int last = (ntiles - 1 - qt0) % 3;          // the stage of the last tile
        terms += last * 2 * PACK_TILE * 4;
#pragma unroll
        for (int dt = 0; dt < NT; ++dt) { ta[dt][0] += last * TB; ta[dt][1] += last * TB; }
        finish_dk(C0{}, C1{});
    }
    if (CAUSAL) __syncthreads();                          // the ring is overwritten where rows are computed again
    const bool whole = s.it.slot < 0;
    const int kl = (wave & 3) * 32 + (lane & 31);
    float* part = whole ? nullptr : p.part[1] + ((int64_t)s.it.slot * p.nkv + s.hk) * (2 * PACK_BLK * DH) + (DK_ROLE ? 0 : PACK_BLK * DH);
    const int64_t col = (int64_t)(p.nq + (DK_ROLE ? 0 : p.nkv) + s.hk) * p.dh;
    float z = 0.0f;
    if (!whole) {
        // one chunk of a strip: float sums, not scaled, [dK | dV][key][dh]
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v4[4] = {acc[dt][4 * i], acc[dt][4 * i + 1], acc[dt][4 * i + 2], acc[dt][4 * i + 3]};
                if (CAUSAL) note4(z, v4);
                store_f4(part + kl * DH + dt * 32 + 8 * i + 4 * half, v4[0], v4[1], v4[2], v4[3]);
            }
    } else if (kv < len) {
        bf16_t* outp = p.dqkv + (s.it.t0 + kv) * s.ld + col;
        const float f = DK_ROLE ? p.scale : 1.0f;
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v4[4] = {acc[dt][4 * i] * f, acc[dt][4 * i + 1] * f, acc[dt][4 * i + 2] * f, acc[dt][4 * i + 3] * f};
                if (CAUSAL) note4(z, v4);
                if (dt * 32 + 8 * i + 4 * half < p.dh) store4(outp + dt * 32 + 8 * i + 4 * half, v4[0], v4[1], v4[2], v4[3]);
            }
    }
    if (!CAUSAL || !any_nonfinite(z)) return;
    rows_stored();
    dkv_rows_again<DH, DK_ROLE>(reinterpret_cast<float*>(smem) + wave * 2 * DH, p, s, k0, lane);
}

// ---- dQ ---------------------------------------------------------------------------------------------------------------
// Workgroup = (128 flattened rows, key head), 8 wavefronts: w takes 32 rows (w % 4) and one 32-key half (w / 4) of every tile; the
// halves are added through LDS at the end.  Transposed score tile: lane = row.  1.18 us a tile, 1.36 PFLOP/s over the chip, and about 6 us to begin and
// end a strip (item 0.9, loads 2.6 to 3.2, end 2.2): 1038 workgroups of 22 us in the batch above, both lists in one launch of 276 us.
template <int DH> constexpr int dq_lds() { return std::max(6 * tile_bytes<DH>(), 4 * 64 * (DH / 2) * 4); }
template <int DH, bool CAUSAL>
__device__ __forceinline__ void dq_body(char* smem, const Params& p, const BStrip& s) {
    constexpr int TB = tile_bytes<DH>(), NF = DH / 16, NT = DH / 32;
    constexpr int NCH = NCHUNKS<DH, WAVES8>;
    const int t = threadIdx.x, lane = t & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6), qs = wave & 3, kvh = wave >> 2;
    const int len = s.it.len;
    const int r0 = s.it.first + qs * 32, r = r0 + (lane & 31);
    const bool valid = r < s.rows;
    const Row me = row_of(p, valid ? r : s.rows - 1);
    const int q_lo = (int)((unsigned)min(r0, s.rows - 1) / (unsigned)p.G), q_hi = (int)((unsigned)min(r0 + 31, s.rows - 1) / (unsigned)p.G);
    const float c2 = LOG2E * p.scale;
    const int64_t at = s.row0 + (int64_t)me.q * p.nq + me.g;
    const float l2 = valid ? p.lse[at] * LOG2E : 0.0f, dsum = valid ? p.dsum[at] : 0.0f;
    const bf16_t* dobase = p.d_o + s.it.t0 * s.ldo + (int64_t)s.hk * p.G * p.dh;
    f32x16 dq[NT];
#pragma unroll
    for (int dt = 0; dt < NT; ++dt) dq[dt] = zero16();

    const int kv_end = r0 >= s.rows ? 0 : CAUSAL ? q_hi + 1 : len;
    const int tile0 = s.it.tile0, ntiles = s.it.tile1;
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_void_ptr)smem;
    unsigned off[NCH];
    dma_offsets<DH, WAVES8>(off, s.ld, p.dh, t);
    auto fetch_tile = [&](int kt, unsigned stage) {
        tile_dma<DH, WAVES8>(tile_rsrc(s.k, s.ld, kt * PACK_TILE, len, p.dh), stage, off, 0, wave);
        tile_dma<DH, WAVES8>(tile_rsrc(s.v, s.ld, kt * PACK_TILE, len, p.dh), stage + TB, off, 0, wave);
    };
    fetch_tile(tile0, lds0);
    FlatTile<DH, WAVES8> ft;
    ft.init(p.dh, t);
    for (int j = 0; j < 2; ++j) {
        ft.load(p, s, s.q, s.ld, s.it.first / PACK_TILE + j, lds0 + (2 + j) * TB, wave);
        ft.load(p, s, dobase, s.ldo, s.it.first / PACK_TILE + j, lds0 + (4 + j) * TB, wave);
    }
    settle(l2);
    settle(dsum);
    dma_wait();
    __syncthreads();
    bf16x8 qf[NF], dof[NF];
    strip_frags<DH>(qf, lds0 + 2 * TB, qs, lane);
    strip_frags<DH>(dof, lds0 + 4 * TB, qs, lane);
    __syncthreads();                                       // the second stage is free
    unsigned ka[NF], ta[NT][2];
#pragma unroll
    for (int ks = 0; ks < NF; ++ks) { ka[ks] = lds0 + frag_k_off<DH>(kvh * 32, ks, lane); keep_in_register(ka[ks]); }
#pragma unroll
    for (int dt = 0; dt < NT; ++dt)
#pragma unroll
        for (int g = 0; g < 2; ++g) { ta[dt][g] = lds0 + frag_t_off<DH>(dt * 32, kvh * 32, g, lane); keep_in_register(ta[dt][g]); }
    auto step = [&](int kt, auto stg) __attribute__((always_inline)) {
        constexpr int OFF = decltype(stg)::value * 2 * TB;
        if (kt + 1 < ntiles) fetch_tile(kt + 1, lds0 + (1 - decltype(stg)::value) * 2 * TB);
        const int kv0 = kt * PACK_TILE + kvh * 32;
        if (kv0 < kv_end) {                                        // wavefront-uniform
            // the fragments of the three products (K, V, K transposed) through a rolling window of W registers
            f32x16 x = zero16(), dp = zero16();
            constexpr int W = DH <= 64 ? NF : NF / 2;
            bf16x8 fr[W];
            auto fetch = [&](int i) __attribute__((always_inline)) {      // i is a compile-time constant after unrolling
                if (i < NF) return lds_frag_k<OFF>(ka[i]);
                if (i < 2 * NF) return lds_frag_k<OFF + TB>(ka[i - NF]);
                const int k = i - 2 * NF;
                return k & 1 ? lds_frag_t<OFF + 16 * DH * 2>(ta[k >> 1][0], ta[k >> 1][1]) : lds_frag_t<OFF>(ta[k >> 1][0], ta[k >> 1][1]);
            };
#pragma unroll
            for (int i = 0; i < W; ++i) fr[i] = fetch(i);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < 2 * NF; ++i) {
                if (i < NF) x = MFMA(fr[i % W], qf[i], x);
                else dp = MFMA(fr[i % W], dof[i - NF], dp);
                fr[i % W] = fetch(i + W);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
            if (r0 + 31 >= s.rows || kv0 + 31 >= len || (CAUSAL && kv0 + 31 > q_lo)) {
                const int seen = valid ? min(CAUSAL ? me.q : len, len - 1) - kv0 - half * 4 : -1;
#pragma unroll
                for (int v = 0; v < 16; ++v) x[v] = (v >> 2) * 8 + (v & 3) <= seen ? x[v] : -INFINITY;
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) dp[v] = fast_exp2(fmaf(x[v], c2, -l2)) * (dp[v] - dsum);
            const bf16x8 g[2] = {pack_regs(dp, 0), pack_regs(dp, 8)};
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int k = 0; k < NF; ++k) {
                dq[k >> 1] = MFMA(fr[k % W], g[k & 1], dq[k >> 1]);
                if (k + W < NF) {
                    fr[k % W] = fetch(2 * NF + k + W);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            __builtin_amdgcn_s_setprio(0);
        }
        dma_wait();
        __syncthreads();
    };
    for (int kt = tile0; kt < ntiles;) {
        step(kt, std::integral_constant<int, 0>{});
        if (++kt >= ntiles) break;
        step(kt, std::integral_constant<int, 1>{});
        ++kt;
    }
    float* mg = reinterpret_cast<float*>(smem) + (qs * (DH / 2)) * 64 + lane;   // element i at mg[i * 64]
    if (kvh == 1) {
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) mg[(dt * 16 + v) * 64] = dq[dt][v];
    }
    __syncthreads();
    if (kvh == 1) return;
    const bool whole = s.it.slot < 0;
    float* part = whole ? nullptr : p.part[0] + ((int64_t)s.it.slot * p.nkv + s.hk) * (PACK_BLK * DH);
    float z = 0.0f;
    if (!whole) {
        // one chunk of a strip: float sums, not scaled, [row][dh]
        float* pp = part + (qs * 32 + (lane & 31)) * DH;
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v4[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v4[j] = dq[dt][4 * i + j] + mg[(dt * 16 + 4 * i + j) * 64];
                if (CAUSAL) note4(z, v4);
                store_f4(pp + dt * 32 + 8 * i + 4 * half, v4[0], v4[1], v4[2], v4[3]);
            }
    } else if (valid) {
        bf16_t* dqp = p.dqkv + (s.it.t0 + me.q) * s.ld + (int64_t)(s.hk * p.G + me.g) * p.dh;
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v4[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v4[j] = (dq[dt][4 * i + j] + mg[(dt * 16 + 4 * i + j) * 64]) * p.scale;
                if (CAUSAL) note4(z, v4);
                if (dt * 32 + 8 * i + 4 * half < p.dh) store4(dqp + dt * 32 + 8 * i + 4 * half, v4[0], v4[1], v4[2], v4[3]);
            }
    }
    if (!CAUSAL || !any_nonfinite(z)) return;
    rows_stored();
    dq_rows_again<DH>(reinterpret_cast<float*>(smem) + qs * (DH / 2) * 64, p, s, r0, lane);   // this wavefront alone reads its merge area
}

// Workgroups: those of dK/dV, then those of dQ, then what the host, which does not know the lengths, has launched too many (between the two lists they kept
// units waiting: 64 sequences of 128, 8 heads of 64, 43.8 -> 39.9 us, 512 of 16 100.9 -> 94.3).
// Up to head size 64 two workgroups share a compute unit (128 registers, 80 KB of LDS each).
template <int DH, bool CAUSAL>
__global__ __launch_bounds__(WAVES8, DH <= 64 ? 4 : 2) void attn_packed_bwd_kernel(Params p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    // another call's plan: some number within the list, so that what is read of it before it is refused is in the plan
    const int of_kv = (int)min((unsigned)reinterpret_cast<const PackHeader*>(p.plan + p.header)->items[1], (unsigned)p.kv_items) * p.nkv, wg = blockIdx.x;
    BStrip s;
    if (wg >= of_kv) {
        if (take_strip(p, 0, wg - of_kv, s)) dq_body<DH, CAUSAL>(smem, p, s);
        return;
    }
    if (!take_strip(p, 1, wg, s)) return;
    // the role is uniform per wavefront; both bodies run the same loop and the same barriers
    if ((threadIdx.x >> 6) < 4) dkv_body<DH, CAUSAL, false>(smem, p, s);
    else dkv_body<DH, CAUSAL, true>(smem, p, s);
}

template <int DH, bool CAUSAL>
hipError_t run_fwd(const PackAttnArgs& a) {
    const PackShares shares = pack_shares(a.M, a.nq, a.nkv, compute_units());
    const PackLayout L = pack_layout(a.sequences, a.M, a.nq, a.nkv, shares);
    Params p = make_params<bf16_t>(a, L);
    p.part[0] = (float*)a.ws;
    constexpr int lds = fwd_lds<DH>();
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&attn_packed_fwd_kernel<DH, CAUSAL>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL((attn_packed_fwd_kernel<DH, CAUSAL>), dim3((unsigned)(L.cap[0] * a.nkv)), dim3(WAVES4), lds, a.stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || shares.of[0] == 0) return e;
    hipLaunchKernelGGL((attn_packed_fwd_join_kernel<bf16_t, DH>), dim3(join_wgs(L, a.nkv)), dim3(32 * JOIN_ROWS), 0, a.stream, p);
    return hipGetLastError();
}
template <int DH, bool CAUSAL>
hipError_t run_bwd(const PackAttnArgs& a) {
    const PackShares shares = pack_shares(a.M, a.nq, a.nkv, compute_units());
    const PackLayout L = pack_layout(a.sequences, a.M, a.nq, a.nkv, shares);
    Params p = make_params<bf16_t>(a, L);
    const Ws w = ws_of(a, true);
    p.part[0] = (float*)a.ws;
    p.part[1] = (float*)((char*)a.ws + w.part[0]);
    const int strips = (int)std::min<int64_t>(L.cap[0] * a.nkv, 2 * compute_units()), rows = (int)std::min<int64_t>((a.M * a.nq + 15) / 16, 8 * compute_units());
    hipLaunchKernelGGL((attn_packed_dsum_kernel<DH, CAUSAL>), dim3((unsigned)(strips + rows)), dim3(WAVES4), dsum_lds<DH>(), a.stream, p, strips);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    p.kv_items = (int)L.cap[1];
    constexpr int lds = std::max(dkv_lds<DH>(), dq_lds<DH>());
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&attn_packed_bwd_kernel<DH, CAUSAL>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL((attn_packed_bwd_kernel<DH, CAUSAL>), dim3((unsigned)((L.cap[0] + L.cap[1]) * a.nkv)), dim3(WAVES8), lds, a.stream, p);
    e = hipGetLastError();
    if (e != hipSuccess || shares.of[0] == 0) return e;
    hipLaunchKernelGGL((attn_packed_bwd_join_kernel<bf16_t, DH>), dim3(join_wgs(L, a.nkv)), dim3(32 * JOIN_ROWS), 0, a.stream, p);
    return hipGetLastError();
}
template <bool CAUSAL>
hipError_t run(const PackAttnArgs& a, bool bwd) {
    switch (padded(a.dh)) {
        case 32: return bwd ? run_bwd<32, CAUSAL>(a) : run_fwd<32, CAUSAL>(a);
        case 64: return bwd ? run_bwd<64, CAUSAL>(a) : run_fwd<64, CAUSAL>(a);
        case 96: return bwd ? run_bwd<96, CAUSAL>(a) : run_fwd<96, CAUSAL>(a);
        default: return bwd ? run_bwd<128, CAUSAL>(a) : run_fwd<128, CAUSAL>(a);
    }
}
}  // namespace

hipError_t attn_packed_bf16(const PackAttnArgs& a, bool bwd) { return a.causal ? run<true>(a, bwd) : run<false>(a, bwd); }

}  // namespace tpl
