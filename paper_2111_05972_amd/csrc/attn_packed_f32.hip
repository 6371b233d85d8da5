// float softmax attention of packed sequences with grouped heads for gfx950 on MFMA 32x32x2 f32, forward and backward, head sizes that are a
// multiple of 8 up to 128.  Operands stay float: nothing is rounded besides the sums.
//
// As attn_f32.hip: matrix time (64 cycles an instruction) dwarfs everything else, so a workgroup owns 32 rows (flattened query rows, or keys) and
// its four wavefronts walk every fourth 32-row tile of the other side with LDS tiles of their own, no barrier in the loop; the four results are
// combined through LDS in wavefront order.  Strips of the plan are 128 rows by 64-row tiles: four workgroups to a strip, each taking the tiles of
// its own 32 rows.  Infinities and NaN in masked places as in attn_packed_bf16.hip.
// Bound by a wavefront alone on its SIMD, whose matrix, vector and LDS times add up: 2 sequences of 2048, 8 heads of 128, causal, forward 261 us
// (66 TFLOP/s of the 154 that a large product reaches), backward 786 (77 with the scores worked out twice); without a mask 397 (87) and 1290 (93).  Two
// sequences of 128, 2 / 1 heads of 64: 7.6 and 22 us, launches and the longest strip.
#include <hip/hip_runtime.h>

#include "attn_f32_frag.h"
#include "attn_packed_dev.h"
#include "attn_rows.h"
#include "device_math.h"
#include "kernels.h"
#include "lds_dma.h"

namespace tpl {
namespace {

using FParams = PackParams<float>;
using FStrip = Strip<float>;
constexpr int QUARTERS = PACK_BLK / XT;

// The 32-key tiles of an item that rows of queries q_lo .. q_hi see (`seen`: the first key that none of them does): number i begins with key at(i).  With a window those of
// the first keys, then those of the window: an item's 64-key tiles are a strip's, four times as many rows.
template <bool WIN> struct XTiles {
    int n, first, second, from;           // tiles; first ones; where the others begin, counted as the item does
    const FParams& p;
    const FStrip& s;
    __device__ __forceinline__ XTiles(const FParams& p_, const FStrip& s_, int q_lo, int seen) : p(p_), s(s_) {
        const int t0 = 2 * s.it.tile0, nt = min(2 * s.it.tile1, (seen + XT - 1) / XT - (WIN ? 2 * s.it.skip : 0));
        first = WIN ? max(0, min(nt, (p.sinks + XT - 1) / XT) - t0) : 0;
        second = WIN ? max(t0 + first, max(0, q_lo + 1 - p.window) / XT - 2 * s.it.skip) : t0;
        from = t0;
        n = first + max(0, nt - second);
    }
    __device__ __forceinline__ int at(int i) const {
        if (!WIN) return (from + i) * XT;
        const int t = i < first ? from + i : second + i - first;
        return (t & 1) * XT + tile_of(p, s, t >> 1) * PACK_TILE;
    }
};
// 32 rows of K or V from row `row0` on: zero past the sequence.
__device__ __forceinline__ i32x4 xtile_rsrc(const float* base, int64_t ld, int row0, int rows, int dh) {
    const int left = rows - row0 < XT ? rows - row0 : XT;
    return make_rsrc(base + (left > 0 ? row0 * ld : 0), left > 0 ? (unsigned)(((left - 1) * ld + dh) * 4) : 0u);
}
// 32 flattened rows from r0 on into the LDS tile at `lds`, from rows of stride ld; nothing is read (zeros are written) past the sequence.
template <int DH>
__device__ __forceinline__ void xfetch_flat(const FParams& p, const FStrip& s, const float* base, int64_t ld, int r0, unsigned lds, int lane) {
    constexpr int NC = DH / 4;
    const int rc = min(r0, s.rows - 1), q0 = rc / p.G, skip = rc - q0 * p.G;              // uniform
    const int left = r0 < s.rows ? min(s.it.len - q0, (XT - 1 + skip) / p.G + 1) : 0;
    const i32x4 r = make_rsrc(base + q0 * ld, left > 0 ? (unsigned)((left - 1) * ld * 4) + (unsigned)(p.G * p.dh * 4) : 0u);
#pragma unroll
    for (int i = 0; i < xloads<DH>(); ++i) {
        const int at = lane + 64 * i, row = at / NC, c = (at % NC) ^ xswz<DH>(row);
        const unsigned x = (unsigned)(row + skip), q = x * p.div_g >> 16, g = x - q * (unsigned)p.G;
        const bool in = (int)q < left && 4 * c < p.dh;
        buffer_load_lds_b128(r, lds + i * 1024, in ? q * (unsigned)(ld * 4) + g * (unsigned)(p.dh * 4) + (unsigned)c * 16u : X_OOB);
    }
}

// Workgroup `u` of a launch: a quarter of a strip of list 0 (forward), of list 1 or 0 (backward).  Long strips by lists, their four quarters one after
// another, longest first; then the short ones (first_short), chunks of cut strips among them.  Where these are many, a workgroup has all of one, a
// wavefront to a quarter (ALONE);
// otherwise all first quarters, all second ones and so on, as those of short sequences have no more than one.  Workgroups that find none of their
// own come last: among the others they made these wait.  52 sequences of 117 tokens together, 8 heads of 128, forward and backward: 66 and 193 us with four
// workgroups to a strip one after another, so 21 and 61; all strips as the short ones: 29 sequences of 9224 tokens, 8 heads of 32, forward 62 -> 74.
// Returns the list, -1: there is no such quarter.
constexpr int ALONE = -1;
template <bool MANY> __device__ __forceinline__ int take_quarter(const FParams& p, bool bwd, int u, FStrip& s, int& sub) {
    const PackHeader* h = reinterpret_cast<const PackHeader*>(p.plan + p.header);
    if (!pack_matches(h, p)) return -1;
    const int first[2] = {h->first_short[0] * p.nkv, bwd ? h->first_short[1] * p.nkv : 0};
    const int after[2] = {h->items[0] * p.nkv - first[0], bwd ? h->items[1] * p.nkv - first[1] : 0};        // short ones
    for (int side = 1; side >= 0; --side) {
        if (u < QUARTERS * first[side]) {
            sub = u % QUARTERS;
            strip_at(p, side, u / QUARTERS, s);
            return side;
        }
        u -= QUARTERS * first[side];
    }
    const int all = after[0] + after[1];
    const bool alone = MANY && all > p.many;
    if (u >= (alone ? 1 : QUARTERS) * all) return -1;
    sub = alone ? ALONE : u / all;
    u %= all;
    const int side = u < after[1];
    strip_at(p, side, side ? first[1] + u : first[0] + u - after[1], s);
    return side;
}
// The result of a wavefront that had all tiles: every accumulator times f to put(d block, i, four rows' values); returns as xcombine.
template <int DH, typename Put>
__device__ __forceinline__ float xalone(const f32x16 (&acc)[DH / 32], float f, Put put) {
    float z = 0.0f;
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float r[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) { r[j] = acc[d][4 * i + j] * f; z = fmaf(r[j], 0.0f, z); }
            put(d, i, r);
        }
    return z;
}

template <int DH, bool MANY, bool WIN>
__global__ __launch_bounds__(256) void attn_packed_f32_fwd_kernel(FParams p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int TB = xtile_bytes<DH>(), NL = xloads<DH>();
    FStrip s;
    int sub;
    if (take_quarter<MANY>(p, false, blockIdx.x, s, sub) < 0) return;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool alone = MANY && sub == ALONE;                      // this wavefront has its quarter to itself, and meets no barrier
    if (alone) sub = wave;
    const int r0 = s.it.first + sub * XT, len = s.it.len, mine = alone ? 0 : wave, step = alone ? 1 : 4;
    if (r0 >= s.rows) return;
    const int r = r0 + (lane & 31);
    const bool valid = r < s.rows;
    const Row me = row_of(p, valid ? r : s.rows - 1);
    const int q_lo = (int)((unsigned)r0 / (unsigned)p.G), q_hi = (int)((unsigned)min(r0 + 31, s.rows - 1) / (unsigned)p.G);
    float qr[DH / 2];
    xrow<DH>(qr, s.q + me.q * s.ld + me.g * p.dh, 0, 0, valid ? 1 : 0, p.dh, lane);
    f32x16 acc[DH / 32];
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[d][v] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    const XTiles<WIN> tiles(p, s, q_lo, p.mask != PACK_ALL ? q_hi + 1 : len);
    const int nt = tiles.n;
    char* kt_ = smem + wave * 2 * TB;
    const unsigned lk = (unsigned)(uintptr_t)(lds_void_ptr)kt_, lv = lk + TB;
    unsigned off[NL];
    xoffsets<DH>(off, s.ld, p.dh, lane);
    auto fetch = [&](const float* base, unsigned lds, int t) { xfetch<DH>(xtile_rsrc(base, s.ld, t < nt ? tiles.at(t) : len, len, p.dh), lds, off, 0, s.ld); };
    if (mine < nt) { fetch(s.k, lk, mine); fetch(s.v, lv, mine); }
    for (int t = mine; t < nt; t += step) {
        xwait<NL>();                                              // K of this tile (V is younger)
        f32x16 x = xscores<DH>(kt_, qr, lane);
        xreads_done();
        fetch(s.k, lk, t + step);                                    // past the last tile: zeros, so that the count of loads in flight stays
        const int k0 = tiles.at(t);
        const bool edge = k0 + XT > len || (p.mask != PACK_ALL && k0 + XT - 1 > q_lo) || (WIN && k0 < q_hi + 1 - p.window);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            x[v] *= p.scale;
            if (edge) {
                const int k = k0 + 8 * (v >> 2) + 4 * half + (v & 3);
                if (k >= len || (WIN ? !window_sees(p, me.q, k) : p.mask != PACK_ALL && k > me.q)) x[v] = -INFINITY;
            }
        }
        float mt = x[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) mt = fmaxf(mt, x[v]);
        mt = fmaxf(mt, xother(mt));
        const float mn = fmaxf(m, mt), mu = mn == -INFINITY ? 0.0f : mn, alpha = expf(m - mu);
        m = mn;
        float ps = 0.0f;
#pragma unroll
        for (int v = 0; v < 16; ++v) { x[v] = expf(x[v] - mu); ps += x[v]; }
        l = l * alpha + ps;
#pragma unroll
        for (int d = 0; d < DH / 32; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[d][v] *= alpha;
        xwait<NL>();                                              // V of this tile (the next K is younger)
        xaccumulate<DH>(acc, kt_ + TB, x, lane);
        xreads_done();
        fetch(s.v, lv, t + step);
    }
    xwait<0>();
    l += xother(l);
    const bool whole = s.it.slot < 0;
    float* part = whole ? nullptr : p.part[0] + ((int64_t)s.it.slot * p.nkv + s.hk) * (PACK_BLK * (DH + 2));
    const int rl = sub * XT + (lane & 31);
    const int64_t head = (int64_t)s.hk * p.G;
    float* op = whole ? p.o + (s.it.t0 + me.q) * s.ldo + (head + me.g) * p.dh : part + rl * DH;
    auto put = [&](int d, int i, const float (&v)[4]) {
        const int c = d * 32 + 8 * i + 4 * half;
        if (!whole || (valid && c < p.dh)) *reinterpret_cast<float4*>(op + c) = make_float4(v[0], v[1], v[2], v[3]);
    };
    float z;
    auto stats = [&](float top, float sum) {
        if (!whole) { part[PACK_BLK * DH + rl] = top; part[PACK_BLK * DH + PACK_BLK + rl] = sum; }
        else if (valid) p.lse[s.row0 + (int64_t)me.q * p.nq + me.g] = top + logf(sum);
    };
    if (alone) {                                                  // a short strip, or as short a chunk of one that was cut
        z = xalone<DH>(acc, whole ? 1.0f / l : 1.0f, put);
        if (half == 0) stats(m, l);
    } else {
        float* st = reinterpret_cast<float*>(smem + 8 * TB);      // [wavefront][m, l][row]
        if (half == 0) { st[wave * 64 + lane] = m; st[wave * 64 + 32 + lane] = l; }
        __syncthreads();
        float mt = -INFINITY, f[4], lt = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) mt = fmaxf(mt, st[w * 64 + (lane & 31)]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[w] = expf(st[w * 64 + (lane & 31)] - (mt == -INFINITY ? 0.0f : mt));
            lt = fmaf(st[w * 64 + 32 + (lane & 31)], f[w], lt);
        }
        if (whole) {
#pragma unroll
            for (int w = 0; w < 4; ++w) f[w] /= lt;
        }
        z = xcombine<DH>(smem, acc, f, wave, lane, put);
        if (wave == 0 && half == 0) stats(mt, lt);
    }
    if (p.mask == PACK_ALL || !__any(z != 0.0f)) return;
    rows_stored();
    float* q_s = xrows<DH>(smem, wave);
    for (int i = r0; i < r0 + XT && i < s.rows; ++i) {
        const Row w = row_of(p, i);
        load_row(q_s, s.q + w.q * s.ld + w.g * p.dh, p.dh, lane);
        row_loaded();
        float* oi = whole ? p.o + (s.it.t0 + w.q) * s.ldo + (head + w.g) * p.dh : part + (i - s.it.first) * DH;
        float mr, lr;
        auto store = [&](int d, float v) { if (alone || xmine(d, wave)) oi[d] = v; };
        const int beg = s.it.tile0 * PACK_TILE, end = s.it.tile1 * PACK_TILE;
        if constexpr (WIN)
            attn_row_fwd<(DH + 63) / 64>(q_s, s.k, s.v, s.ld, p.dh, beg, end, p.scale, whole, lane, mr, lr, store, WindowKeys<float>{p, s, w.q});
        else
            attn_row_fwd<(DH + 63) / 64>(q_s, s.k, s.v, s.ld, p.dh, beg, min(w.q + 1, end), p.scale, whole, lane, mr, lr, store);
        if (lane == 0 && (alone || wave == 0)) {
            if (whole) p.lse[s.row0 + (int64_t)w.q * p.nq + w.g] = mr + logf(lr);
            else { part[PACK_BLK * DH + i - s.it.first] = mr; part[PACK_BLK * DH + PACK_BLK + i - s.it.first] = lr; }
        }
        row_loaded();
    }
}

template <int DH, bool MANY, bool WIN>
__device__ __forceinline__ void f32_dq(char* smem, const FParams& p, const FStrip& s, int sub) {
    constexpr int TB = xtile_bytes<DH>(), NL = xloads<DH>();
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool alone = MANY && sub == ALONE;
    if (alone) sub = wave;
    const int r0 = s.it.first + sub * XT, len = s.it.len, mine = alone ? 0 : wave, step = alone ? 1 : 4;
    if (r0 >= s.rows) return;
    const int r = r0 + (lane & 31);
    const bool valid = r < s.rows;
    const Row me = row_of(p, valid ? r : s.rows - 1);
    const int q_lo = (int)((unsigned)r0 / (unsigned)p.G), q_hi = (int)((unsigned)min(r0 + 31, s.rows - 1) / (unsigned)p.G);
    char* kt_ = smem + wave * 2 * TB;
    const unsigned lk = (unsigned)(uintptr_t)(lds_void_ptr)kt_, lv = lk + TB;
    const int64_t head = (int64_t)s.hk * p.G;
    const float* dobase = p.d_o + s.it.t0 * s.ldo + head * p.dh;
    float qr[DH / 2], gr[DH / 2];
    xrow<DH>(qr, s.q + me.q * s.ld + me.g * p.dh, 0, 0, valid ? 1 : 0, p.dh, lane);
    xrow<DH>(gr, dobase + me.q * s.ldo + me.g * p.dh, 0, 0, valid ? 1 : 0, p.dh, lane);
    const int64_t at = s.row0 + (int64_t)me.q * p.nq + me.g;
    const float D = valid ? p.dsum[at] : 0.0f, L = valid ? p.lse[at] : 0.0f;
    f32x16 acc[DH / 32];
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[d][v] = 0.0f;
    const XTiles<WIN> tiles(p, s, q_lo, p.mask != PACK_ALL ? q_hi + 1 : len);
    const int nt = tiles.n;
    unsigned off[NL];
    xoffsets<DH>(off, s.ld, p.dh, lane);
    auto fetch = [&](const float* base, unsigned lds, int t) { xfetch<DH>(xtile_rsrc(base, s.ld, t < nt ? tiles.at(t) : len, len, p.dh), lds, off, 0, s.ld); };
    if (mine < nt) { fetch(s.v, lv, mine); fetch(s.k, lk, mine); }   // V is read first
    for (int t = mine; t < nt; t += step) {
        xwait<NL>();
        f32x16 dp = xscores<DH>(kt_ + TB, gr, lane);              // dP^T = V dO^T
        xreads_done();
        fetch(s.v, lv, t + step);
        xwait<NL>();
        const f32x16 x = xscores<DH>(kt_, qr, lane);
        const int k0 = tiles.at(t);
        const bool edge = k0 + XT > len || (p.mask != PACK_ALL && k0 + XT - 1 > q_lo) || (WIN && k0 < q_hi + 1 - p.window);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            float w = expf(x[v] * p.scale - L);
            w *= dp[v] - D;
            if (edge) {
                const int k = k0 + 8 * (v >> 2) + 4 * half + (v & 3);
                if (k >= len || (WIN ? !window_sees(p, me.q, k) : p.mask != PACK_ALL && k > me.q)) w = 0.0f;
            }
            dp[v] = w;
        }
        xaccumulate<DH>(acc, kt_, dp, lane);                      // dQ^T += K^T dS
        xreads_done();
        fetch(s.k, lk, t + step);
    }
    xwait<0>();
    const bool whole = s.it.slot < 0;
    const float f1 = whole ? p.scale : 1.0f, f[4] = {f1, f1, f1, f1};
    float* part = whole ? nullptr : p.part[0] + ((int64_t)s.it.slot * p.nkv + s.hk) * (PACK_BLK * DH);
    float* dqp = whole ? p.dqkv + (s.it.t0 + me.q) * s.ld + (head + me.g) * p.dh : part + (sub * XT + (lane & 31)) * DH;
    auto put = [&](int d, int i, const float (&v)[4]) {
        const int c = d * 32 + 8 * i + 4 * half;
        if (!whole || (valid && c < p.dh)) *reinterpret_cast<float4*>(dqp + c) = make_float4(v[0], v[1], v[2], v[3]);
    };
    const float z = alone ? xalone<DH>(acc, f1, put) : xcombine<DH>(smem, acc, f, wave, lane, put);
    if (p.mask == PACK_ALL || !__any(z != 0.0f)) return;
    rows_stored();
    float* q_s = xrows<DH>(smem, wave);
    for (int i = r0; i < r0 + XT && i < s.rows; ++i) {
        const Row w = row_of(p, i);
        load_row(q_s, s.q + w.q * s.ld + w.g * p.dh, p.dh, lane);
        load_row(q_s + DH, dobase + w.q * s.ldo + w.g * p.dh, p.dh, lane);
        row_loaded();
        float* dqi = whole ? p.dqkv + (s.it.t0 + w.q) * s.ld + (head + w.g) * p.dh : part + (i - s.it.first) * DH;
        const int64_t a = s.row0 + (int64_t)w.q * p.nq + w.g;
        auto store = [&](int d, float v) { if (alone || xmine(d, wave)) dqi[d] = v * f1; };
        const int beg = s.it.tile0 * PACK_TILE, end = s.it.tile1 * PACK_TILE;
        if constexpr (WIN)
            attn_row_dq<(DH + 63) / 64>(q_s, q_s + DH, s.k, s.v, s.ld, p.dh, beg, end, p.scale, p.lse[a], p.dsum[a], lane, store, WindowKeys<float>{p, s, w.q});
        else
            attn_row_dq<(DH + 63) / 64>(q_s, q_s + DH, s.k, s.v, s.ld, p.dh, beg, min(w.q + 1, end), p.scale, p.lse[a], p.dsum[a], lane, store);
        row_loaded();
    }
}

template <int DH, bool MANY, bool WIN>
__device__ __forceinline__ void f32_dkv(char* smem, const FParams& p, const FStrip& s, int sub) {
    constexpr int TB = xtile_bytes<DH>();
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool alone = MANY && sub == ALONE;
    if (alone) sub = wave;
    const int k0 = s.it.first + sub * XT, len = s.it.len, mine = alone ? 0 : wave, step = alone ? 1 : 4;
    if (k0 >= len) return;
    const int k = k0 + (lane & 31);
    const bool valid = k < len;
    const int64_t head = (int64_t)s.hk * p.G;
    const float* dobase = p.d_o + s.it.t0 * s.ldo + head * p.dh;
    float kr[DH / 2], vr[DH / 2];
    xrow<DH>(kr, s.k, s.ld, k, len, p.dh, lane);
    xrow<DH>(vr, s.v, s.ld, k, len, p.dh, lane);
    f32x16 dk[DH / 32], dv[DH / 32];
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) { dk[d][v] = 0.0f; dv[d][v] = 0.0f; }
    char* qt_ = smem + wave * 2 * TB;
    const unsigned lq = (unsigned)(uintptr_t)(lds_void_ptr)qt_, lg = lq + TB;
    float* terms = reinterpret_cast<float*>(smem + 8 * TB) + wave * 2 * XT;   // LSE, D of the tile's rows
    // rows that see one of the keys: below `rows`, and with a window all but the first keys are out of sight from some row on
    const int rows = WIN && k0 >= p.sinks ? min(s.rows, (min(k0 + XT, len) - 1 + p.window) * p.G) : s.rows;
    const int gone = WIN && k0 + XT > p.sinks ? (max(k0, p.sinks) + p.window) * p.G : 0x7fffffff;
    const int t0 = max(2 * s.it.tile0, p.mask != PACK_ALL ? k0 * p.G / XT : 0), nt = min(2 * s.it.tile1, (rows + XT - 1) / XT);
    auto term = [&](int t) {                                      // lanes 0..31: LSE, lanes 32..63: D
        const int i = t * XT + (lane & 31);
        const Row w = row_of(p, min(i, s.rows - 1));
        return i < s.rows ? (half ? p.dsum : p.lse)[s.row0 + (int64_t)w.q * p.nq + w.g] : 0.0f;
    };
    auto fetch_q = [&](int t) { xfetch_flat<DH>(p, s, s.q, s.ld, t < nt ? t * XT : s.rows, lq, lane); };
    auto fetch_g = [&](int t) { xfetch_flat<DH>(p, s, dobase, s.ldo, t < nt ? t * XT : s.rows, lg, lane); };
    float tn = 0.0f;
    if (t0 + mine < nt) {
        tn = term(t0 + mine);
        fetch_q(t0 + mine);
        fetch_g(t0 + mine);
    }
    const int from = p.mask != PACK_ALL ? k * p.G : 0;            // the first row that sees this lane's key
    const int to = WIN && k >= p.sinks ? min(s.rows, (min(k, len) + p.window) * p.G) : s.rows;
    for (int t = t0 + mine; t < nt; t += step) {
        const int nx = t + step;
        terms[lane] = tn;
        xwait<0>();
        if (nx < nt) tn = term(nx);
        f32x16 w = xscores<DH>(qt_, kr, lane);
        f32x16 ds = xscores<DH>(qt_ + TB, vr, lane);              // dP = dO V^T
        const int q0 = t * XT;
        const bool edge = q0 + XT > s.rows || k0 + XT > len || (p.mask != PACK_ALL && (k0 + XT - 1) * p.G > q0) || (WIN && q0 + XT > gone);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 l4 = *reinterpret_cast<const float4*>(terms + 8 * i + 4 * half);
            const float4 d4 = *reinterpret_cast<const float4*>(terms + XT + 8 * i + 4 * half);
            const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dv4[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int v = 4 * i + j, row = q0 + 8 * i + 4 * half + j;
                const float e = expf(w[v] * p.scale - lv[j]), g = e * (ds[v] - dv4[j]);
                const bool out = edge && (row >= to || !valid || row < from);
                w[v] = out ? 0.0f : e;
                ds[v] = out ? 0.0f : g;
            }
        }
        xaccumulate<DH>(dv, qt_ + TB, w, lane);                   // dV^T += dO^T P
        xreads_done();
        fetch_g(nx);
        xaccumulate<DH>(dk, qt_, ds, lane);                       // dK^T += Q^T dS
        xreads_done();
        fetch_q(nx);
    }
    xwait<0>();
    const bool whole = s.it.slot < 0;
    float* part = whole ? nullptr : p.part[1] + ((int64_t)s.it.slot * p.nkv + s.hk) * (2 * PACK_BLK * DH);
    const int kl = sub * XT + (lane & 31);
    float* kp = whole ? p.dqkv + (s.it.t0 + k) * s.ld + (int64_t)(p.nq + s.hk) * p.dh : part + kl * DH;
    float* vp = whole ? kp + (int64_t)p.nkv * p.dh : part + PACK_BLK * DH + kl * DH;
    const float f1 = whole ? p.scale : 1.0f, fk[4] = {f1, f1, f1, f1}, fv[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    auto put = [&](float* to) {
        return [=](int d, int i, const float (&v)[4]) {
            const int c = d * 32 + 8 * i + 4 * half;
            if (!whole || (valid && c < p.dh)) *reinterpret_cast<float4*>(to + c) = make_float4(v[0], v[1], v[2], v[3]);
        };
    };
    float z;
    if (alone) {
        z = xalone<DH>(dk, f1, put(kp));
        z += xalone<DH>(dv, 1.0f, put(vp));
    } else {
        z = xcombine<DH>(smem, dk, fk, wave, lane, put(kp));
        z += xcombine<DH>(smem, dv, fv, wave, lane, put(vp));
    }
    if (p.mask == PACK_ALL || !__any(z != 0.0f)) return;
    rows_stored();
    constexpr int NA = (DH + 63) / 64;
    float* k_s = xrows<DH>(smem, wave);
    for (int j = k0; j < k0 + XT && j < len; ++j) {
        load_row(k_s, s.k + j * s.ld, p.dh, lane);
        load_row(k_s + DH, s.v + j * s.ld, p.dh, lane);
        row_loaded();
        float dks[NA] = {}, dvs[NA] = {};
        const int last = min(s.rows, s.it.tile1 * PACK_TILE);
        const int end = WIN && j >= p.sinks ? min(last, (j + p.window) * p.G) : last;
        for (int i = max(j * p.G, s.it.tile0 * PACK_TILE); i < end; ++i) {
            const Row w = row_of(p, i);
            const float* qp = s.q + w.q * s.ld + w.g * p.dh;
            const float* gp = dobase + w.q * s.ldo + w.g * p.dh;
            float a = 0.0f, b = 0.0f, q[NA], g[NA];
#pragma unroll
            for (int n = 0; n < NA; ++n) {
                const int d = lane + 64 * n;
                q[n] = d < p.dh ? qp[d] : 0.0f;
                g[n] = d < p.dh ? gp[d] : 0.0f;
                if (d < p.dh) { a = fmaf(q[n], k_s[d], a); b = fmaf(g[n], k_s[DH + d], b); }
            }
            const float e = expf(row_sum(a) * p.scale - p.lse[s.row0 + (int64_t)w.q * p.nq + w.g]);
            const float ds = e * (row_sum(b) - p.dsum[s.row0 + (int64_t)w.q * p.nq + w.g]);
#pragma unroll
            for (int n = 0; n < NA; ++n) { dks[n] = fmaf(ds, q[n], dks[n]); dvs[n] = fmaf(e, g[n], dvs[n]); }
        }
        const int64_t row = (s.it.t0 + j) * s.ld + (int64_t)(p.nq + s.hk) * p.dh;
#pragma unroll
        for (int n = 0; n < NA; ++n) {
            const int d = lane + 64 * n;
            if (d >= p.dh || !(alone || xmine(d, wave))) continue;
            if (whole) { p.dqkv[row + d] = dks[n] * p.scale; p.dqkv[row + (int64_t)p.nkv * p.dh + d] = dvs[n]; }
            else { part[(j - s.it.first) * DH + d] = dks[n]; part[PACK_BLK * DH + (j - s.it.first) * DH + d] = dvs[n]; }
        }
        row_loaded();
    }
}

template <int LANES>
__global__ __launch_bounds__(256) void attn_packed_f32_dsum_kernel(FParams p) {
    dsum_rows<LANES>(p, (int)blockIdx.x, (int)gridDim.x, 0);
}

// Two workgroups share a compute unit up to head size 64 (see attn_f32.hip); wider heads need more than 256 registers.
template <int DH, bool MANY, bool WIN>
__global__ __launch_bounds__(256, DH <= 64 ? 2 : 1) void attn_packed_f32_bwd_kernel(FParams p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    FStrip s;
    int sub;
    const int side = take_quarter<MANY>(p, true, blockIdx.x, s, sub);
    if (side < 0) return;
    if (side) f32_dkv<DH, MANY, WIN>(smem, p, s, sub);
    else f32_dq<DH, MANY, WIN>(smem, p, s, sub);
}

// Short strips above which a wavefront has a quarter to itself: three quarters of the workgroups that run at once.  48 sequences of 918 tokens together,
// 32 / 8 heads of 96, forward and backward 55 and 117 us, so 33 and 98; 60 of 600, 8 heads of 64, 14.7 and 32.4, so 11.2 and 28.5; but 30 of 1489, 2 heads of 64,
// 25 us backward, so 51: each wavefront then has up to six tiles in a row.
int many_strips(int DH) { return compute_units() * (DH <= 32 ? 4 : DH <= 64 ? 2 : 1) * 3 / 4; }
template <int DH, bool MANY, bool WIN>
hipError_t launch(const PackAttnArgs& a, bool bwd) {
    constexpr int lds = xlds_bytes<DH>();
    static const hipError_t attr_f = hipFuncSetAttribute(reinterpret_cast<const void*>(&attn_packed_f32_fwd_kernel<DH, MANY, WIN>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    static const hipError_t attr_b = hipFuncSetAttribute(reinterpret_cast<const void*>(&attn_packed_f32_bwd_kernel<DH, MANY, WIN>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr_f != hipSuccess || attr_b != hipSuccess) return attr_f != hipSuccess ? attr_f : attr_b;
    const PackShares shares = pack_shares(a.M, a.nq, a.nkv, compute_units());
    const PackLayout L = pack_layout(a.sequences, a.M, a.nq, a.nkv, shares);
    FParams p = make_params<float>(a, L);
    p.part[0] = (float*)a.ws;
    p.many = many_strips(DH);
    const dim3 join(join_wgs(L, a.nkv));
    const PackCut cut = cut_of(a);
    hipError_t e;
    if (!bwd) {
        hipLaunchKernelGGL((attn_packed_f32_fwd_kernel<DH, MANY, WIN>), dim3((unsigned)(L.cap[0] * a.nkv * QUARTERS)), dim3(256), lds, a.stream, p);
        if ((e = hipGetLastError()) != hipSuccess || !cut.of[0]) return e;
        hipLaunchKernelGGL((attn_packed_fwd_join_kernel<float, DH>), join, dim3(32 * JOIN_ROWS), 0, a.stream, p);
        return hipGetLastError();
    }
    p.part[1] = (float*)((char*)a.ws + ws_of(a, true).part[0]);
    hipLaunchKernelGGL(attn_packed_f32_dsum_kernel<dsum_lanes<DH>()>, dim3(dsum_wgs<dsum_lanes<DH>()>(a)), dim3(256), 0, a.stream, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((attn_packed_f32_bwd_kernel<DH, MANY, WIN>), dim3((unsigned)((L.cap[0] + L.cap[1]) * a.nkv * QUARTERS)), dim3(256), lds, a.stream, p);
    if ((e = hipGetLastError()) != hipSuccess || !(cut.of[0] || cut.of[1])) return e;
    hipLaunchKernelGGL((attn_packed_bwd_join_kernel<float, DH>), join, dim3(32 * JOIN_ROWS), 0, a.stream, p);
    return hipGetLastError();
}
// MANY: the kernels that can give a wavefront a quarter of its own, 3 % slower in backward where they do not, only where there are sequences enough for it.
template <int DH, bool WIN>
hipError_t run_mask(const PackAttnArgs& a, bool bwd) { return a.sequences * a.nkv > many_strips(DH) ? launch<DH, true, WIN>(a, bwd) : launch<DH, false, WIN>(a, bwd); }
template <int DH>
hipError_t run(const PackAttnArgs& a, bool bwd) { return a.mask == PACK_WINDOW ? run_mask<DH, true>(a, bwd) : run_mask<DH, false>(a, bwd); }
}  // namespace

hipError_t attn_packed_f32(const PackAttnArgs& a, bool bwd) {
    switch ((a.dh + 31) / 32) {
        case 1: return run<32>(a, bwd);
        case 2: return run<64>(a, bwd);
        case 3: return run<96>(a, bwd);
        default: return run<128>(a, bwd);
    }
}

}  // namespace tpl
