// What the kernels of attn_packed_bf16.hip and attn_packed_f32.hip share: parameters, a workgroup's strip, joins of chunks, row dots.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "attn_packed.h"
#include "attn_rows.h"
#include "device_math.h"
#include "kernels.h"

namespace tpl {
namespace {

template <typename T>
struct PackParams {
    int sequences, M, nq, nkv, G, dh, mask, window, sinks;
    unsigned div_g;               // 65536 / G + 1: x / G = x * div_g >> 16 for x < 64 + G
    const int* plan;
    int64_t seen, header, items[2], joins[2];
    const T* qkv; T* o; float* lse;
    const T* d_o; T* dqkv; float* dsum;
    float* part[2];               // sums of chunks: forward or dQ, dK and dV
    int kv_items;                 // bf16 backward: items of list 1 at most
    int many;                     // float: short strips above which a wavefront has a quarter to itself
    float scale;
};
// Whether the plan at hand was made for this call.
template <typename T>
__device__ __forceinline__ bool pack_matches(const PackHeader* h, const PackParams<T>& p) {
    // no word waits for the one before: behind && each was a load of its own
    return ((h->sequences ^ p.sequences) | (h->tokens ^ p.M) | (h->nq ^ p.nq) | (h->nkv ^ p.nkv) | (h->mask ^ p.mask) | (h->window ^ p.window) | (h->sinks ^ p.sinks)) == 0;
}
// What a workgroup works on.
template <typename T>
struct Strip {
    PackItem it;
    int hk;                       // key head
    int64_t ld, ldo;
    int rows;                     // flattened query rows of the sequence
    const T *q, *k, *v;      // the sequence's first row: query head hk G, key head hk
    int64_t row0;                 // index of that query row in lse and dsum
};
// Item number wg / nkv of list `side`, false: there is none, or the plan is another call's.  Key heads fastest: they are as long as
// each other, and with 8 of them (or a multiple) an XCD keeps to one.
template <typename T>
__device__ __forceinline__ void set_strip(const PackParams<T>& p, int hk, Strip<T>& s) {
    s.hk = hk;
    s.ld = (int64_t)(p.nq + 2 * p.nkv) * p.dh;
    s.ldo = (int64_t)p.nq * p.dh;
    s.rows = s.it.len * p.G;
    s.q = p.qkv + s.it.t0 * s.ld + (int64_t)s.hk * p.G * p.dh;
    s.k = p.qkv + s.it.t0 * s.ld + (int64_t)(p.nq + s.hk) * p.dh;
    s.v = s.k + (int64_t)p.nkv * p.dh;
    s.row0 = (int64_t)s.it.t0 * p.nq + (int64_t)s.hk * p.G;
}
template <typename T>
__device__ __forceinline__ bool take_strip(const PackParams<T>& p, int side, int wg, Strip<T>& s) {
    const PackHeader* h = reinterpret_cast<const PackHeader*>(p.plan + p.header);
    const int i = wg / p.nkv;
    s.it = pack_items(p.plan, p.items[side])[i];                  // within the plan: requested beside the header, not after it
    if (!pack_matches(h, p) || i >= h->items[side]) return false;
    set_strip(p, wg - i * p.nkv, s);
    return true;
}
// Item `i` of list `side`, counted with the key heads as above.
template <typename T>
__device__ __forceinline__ void strip_at(const PackParams<T>& p, int side, int i, Strip<T>& s) {
    const int n = i / p.nkv;
    s.it = pack_items(p.plan, p.items[side])[n];
    set_strip(p, i - n * p.nkv, s);
}
// An item's tiles where some are left out: number `v`, counted without these, is tile tile_of(v) of the keys.
template <typename T>
__device__ __forceinline__ int tile_of(const PackParams<T>& p, const Strip<T>& s, int v) { return v * PACK_TILE >= p.sinks ? v + s.it.skip : v; }
// Whether query q sees key j under a window.
template <typename T>
__device__ __forceinline__ bool window_sees(const PackParams<T>& p, int q, int j) { return j <= q && (j > q - p.window || j < p.sinks); }
// For the row-by-row form: key number j of the tiles for query q, -1: it does not see it.
template <typename T>
struct WindowKeys {
    const PackParams<T>& p;
    const Strip<T>& s;
    int q;
    __device__ __forceinline__ int operator()(int j) const {
        const int k = (j & (PACK_TILE - 1)) + tile_of(p, s, j / PACK_TILE) * PACK_TILE;
        return window_sees(p, q, k) ? k : -1;
    }
};
// A flattened row: its query and its head in the group.
struct Row { int q, g; };
template <typename T>
__device__ __forceinline__ Row row_of(const PackParams<T>& p, int r) {
    const int q = (int)((unsigned)r / (unsigned)p.G);
    return Row{q, r - q * p.G};
}

// Reference points of bf16 are in log2 units, of float natural (a product with log2 e would round them).
template <typename T> __device__ __forceinline__ float pack_exp(float x);
template <> __device__ __forceinline__ float pack_exp<bf16_t>(float x) { return __builtin_amdgcn_exp2f(x); }
template <> __device__ __forceinline__ float pack_exp<float>(float x) { return expf(x); }
template <typename T> __device__ __forceinline__ float pack_lse(float m, float l);
template <> __device__ __forceinline__ float pack_lse<bf16_t>(float m, float l) { return (m + log2f(l)) * 0.69314718055994530942f; }
template <> __device__ __forceinline__ float pack_lse<float>(float m, float l) { return m + logf(l); }

// Joins the chunks of the strips that were cut, in chunk order: largest reference point, rescale, add.  A unit of work is JOIN_ROWS rows of a
// strip and key head, four columns to a thread.
constexpr int JOIN_ROWS = 8, JOIN_WGS = PACK_BLK / JOIN_ROWS;
// The host does not know how many strips were cut, mostly few or none, so a few workgroups walk the list: a launch for all there could be
// took 7 us (forward) and 18 (backward) with none (8192 tokens, 2 key heads).
inline unsigned join_wgs(const PackLayout& L, int nkv) { return (unsigned)std::min<int64_t>((L.join_cap[0] + L.join_cap[1]) * JOIN_WGS * nkv, 4 * compute_units()); }
template <typename T> __device__ __forceinline__ void join_store(T* p, const float (&v)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = (T)v[e];
}
template <typename T, int DH>
__global__ __launch_bounds__(32 * JOIN_ROWS) void attn_packed_fwd_join_kernel(PackParams<T> p) {
    constexpr int PSZ = PACK_BLK * (DH + 2);
    const PackHeader* h = reinterpret_cast<const PackHeader*>(p.plan + p.header);
    if (!pack_matches(h, p)) return;
    const int all = h->joins[0] * p.nkv * JOIN_WGS, col = 4 * (threadIdx.x & 31);
    for (int i = blockIdx.x; i < all; i += gridDim.x) {
        const int hk = i % p.nkv, rest = i / p.nkv;
        const PackItem it = pack_items(p.plan, p.joins[0])[rest / JOIN_WGS];
        const int rl = (rest % JOIN_WGS) * JOIN_ROWS + threadIdx.x / 32, r = it.first + rl;
        if (r >= it.len * p.G || col >= p.dh) continue;
        const Row w = row_of(p, r);
        const float* p0 = p.part[0] + ((int64_t)it.slot * p.nkv + hk) * PSZ;
        const int64_t next = (int64_t)p.nkv * PSZ;
        float top = -INFINITY;
        for (int c = 0; c < it.chunks; ++c) top = fmaxf(top, p0[c * next + PACK_BLK * DH + rl]);
        const float mu = top == -INFINITY ? 0.0f : top;
        float total = 0.0f, v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 2
        for (int c = 0; c < it.chunks; ++c) {
            const float* pc = p0 + c * next;
            const float f = pack_exp<T>(pc[PACK_BLK * DH + rl] - mu), l = pc[PACK_BLK * DH + PACK_BLK + rl];
            const float4 x = *reinterpret_cast<const float4*>(pc + rl * DH + col);
            if (l == 0.0f) continue;                              // a chunk of masked keys: what it holds does not count (of NaN keys: l is NaN)
            total = fmaf(l, f, total);
            v[0] = fmaf(x.x, f, v[0]); v[1] = fmaf(x.y, f, v[1]); v[2] = fmaf(x.z, f, v[2]); v[3] = fmaf(x.w, f, v[3]);
        }
        const int64_t head = (int64_t)hk * p.G + w.g;
        const float inv = 1.0f / total, out[4] = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
        join_store(p.o + ((int64_t)(it.t0 + w.q) * p.nq + head) * p.dh + col, out);
        if (col == 0) p.lse[(int64_t)(it.t0 + w.q) * p.nq + head] = pack_lse<T>(top, total);
    }
}

// ---- D = rowsum(dO * O) of every row and head -------------------------------------------------------------------------------
// LANES lanes to a row, eight elements each, four rows at a time so that their loads are under way together; rows of at most `above` keys are left out, and those
// of no sequence.  Whose plan it is shows while the keys that the first rows see are under way.
template <int DH> constexpr int dsum_lanes() { return DH <= 32 ? 4 : DH <= 64 ? 8 : 16; }
template <int LANES, typename T>
__device__ __forceinline__ void dsum_rows(const PackParams<T>& p, int wg, int wgs, int above) {
    constexpr int ROWS = 256 / LANES, AHEAD = 4;
    const int c = (threadIdx.x % LANES) * 8, mine = threadIdx.x / LANES;
    const int64_t all = (int64_t)p.M * p.nq, step = (int64_t)wgs * ROWS;
    bool ours = false;
    for (int64_t first = (int64_t)wg * ROWS; first < all; first += AHEAD * step) {
        bool wanted[AHEAD];
        float x[AHEAD][8], y[AHEAD][8];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int64_t row = first + j * step + mine;
            wanted[j] = row < all && p.plan[p.seen + (unsigned)row / (unsigned)p.nq] > above;
        }
        if (!ours && !(ours = pack_matches(reinterpret_cast<const PackHeader*>(p.plan + p.header), p))) return;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int64_t at = (first + j * step + mine) * p.dh + c;
            if (wanted[j] && c < p.dh) {
                load8(p.o + at, x[j]);
                load8(p.d_o + at, y[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (first + j * step >= all) break;                   // uniform
            float a = 0.0f;
            if (wanted[j] && c < p.dh) {
#pragma unroll
                for (int e = 0; e < 8; ++e) a = fmaf(x[j][e], y[j][e], a);
            }
#pragma unroll
            for (int off = LANES / 2; off > 0; off >>= 1) a += __shfl_xor(a, off, 64);
            if (wanted[j] && c == 0) p.dsum[first + j * step + mine] = a;
        }
    }
}
// Workgroups for that.
template <int LANES> unsigned dsum_wgs(const PackAttnArgs& a) {
    return (unsigned)std::min<int64_t>((a.M * a.nq * LANES + 255) / 256, 8 * compute_units());
}

// dQ, dK and dV of the strips that were cut: the sums of their chunks in chunk order.  dQ, then dK, then dV.
template <typename T, int DH>
__global__ __launch_bounds__(32 * JOIN_ROWS) void attn_packed_bwd_join_kernel(PackParams<T> p) {
    const PackHeader* h = reinterpret_cast<const PackHeader*>(p.plan + p.header);
    if (!pack_matches(h, p)) return;
    const int of_q = h->joins[0] * p.nkv * JOIN_WGS, of_kv = h->joins[1] * p.nkv * JOIN_WGS, col = 4 * (threadIdx.x & 31);
    for (int i = blockIdx.x; i < of_q + 2 * of_kv; i += gridDim.x) {
        const int which = i < of_q ? 0 : i < of_q + of_kv ? 1 : 2, side = which > 0, n = i - (which == 0 ? 0 : which == 1 ? of_q : of_q + of_kv);
        const int hk = n % p.nkv, rest = n / p.nkv;
        const PackItem it = pack_items(p.plan, p.joins[side])[rest / JOIN_WGS];
        const int rl = (rest % JOIN_WGS) * JOIN_ROWS + threadIdx.x / 32, r = it.first + rl;
        if (r >= (side ? it.len : it.len * p.G) || col >= p.dh) continue;
        const int PSZ = (side ? 2 : 1) * PACK_BLK * DH;
        const float* p0 = p.part[side] + ((int64_t)it.slot * p.nkv + hk) * PSZ + (which == 2 ? PACK_BLK * DH : 0) + rl * DH + col;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int c = 0; c < it.chunks; ++c) {
            const float4 x = *reinterpret_cast<const float4*>(p0 + (int64_t)c * p.nkv * PSZ);
            v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
        }
        const Row w = side ? Row{r, 0} : row_of(p, r);
        const int64_t head = side ? p.nq + (which == 2 ? p.nkv : 0) + hk : hk * p.G + w.g;
        const float f = which == 2 ? 1.0f : p.scale, out[4] = {v[0] * f, v[1] * f, v[2] * f, v[3] * f};
        join_store(p.dqkv + ((int64_t)(it.t0 + w.q) * (p.nq + 2 * p.nkv) + head) * p.dh + col, out);
    }
}

template <typename T>
PackParams<T> make_params(const PackAttnArgs& a, const PackLayout& L) {
    PackParams<T> p{};
    p.sequences = (int)a.sequences; p.M = (int)a.M; p.nq = a.nq; p.nkv = a.nkv; p.G = a.nq / a.nkv; p.dh = a.dh;
    p.mask = a.mask; p.window = a.window; p.sinks = a.sinks;
    p.div_g = 65536u / (unsigned)p.G + 1u;
    p.plan = a.plan; p.seen = L.seen; p.header = L.header;
    for (int s = 0; s < 2; ++s) { p.items[s] = L.items[s]; p.joins[s] = L.joins[s]; }
    p.qkv = (const T*)a.qkv; p.o = (T*)a.o; p.lse = a.lse;
    p.d_o = (const T*)a.d_o; p.dqkv = (T*)a.dqkv; p.dsum = a.dsum;
    p.scale = 1.0f / sqrtf((float)a.dh);
    return p;
}
PackCut cut_of(const PackAttnArgs& a) { return pack_cut(a.mask, a.window, a.sinks, a.M, a.nq, a.nkv, compute_units()); }
int padded(int dh) { return (dh + 31) / 32 * 32; }
// Sums of chunks: a cut strip of n tiles has at most 2 n / chunk of them.
struct Ws { size_t part[2], total; };
Ws ws_of(const PackAttnArgs& a, bool bwd) {
    const PackShares shares = pack_shares(a.M, a.nq, a.nkv, compute_units());
    const int DH = padded(a.dh);
    Ws w{};
    w.part[0] = (size_t)(2 * shares.of[0] * a.nkv) * PACK_BLK * (bwd ? DH : DH + 2) * sizeof(float);
    w.part[1] = bwd ? (size_t)(2 * shares.of[1] * a.nkv) * 2 * PACK_BLK * DH * sizeof(float) : 0;
    w.total = w.part[0] + w.part[1];
    return w;
}

}  // namespace
}  // namespace tpl
