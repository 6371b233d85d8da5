// What the kernels of attn_packed_bf16.hip and attn_packed_f32.hip share: parameters, a workgroup's strip, joins of chunks, row dots.
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>

#include "attn_packed.h"
#include "attn_rows.h"
#include "device_math.h"
#include "kernels.h"

namespace tpl {
namespace {

template <typename T>
struct PackParams {
    int M, nq, nkv, G, dh, causal;
    unsigned div_g;               // 65536 / G + 1: x / G = x * div_g >> 16 for x < 64 + G
    const int* plan;
    int64_t header, items[2], joins[2];
    const T* qkv; T* o; float* lse;
    const T* d_o; T* dqkv; float* dsum;
    float* part[2];               // sums of chunks: forward or dQ, dK and dV
    int kv_wgs;                   // backward: workgroups of dK/dV, before those of dQ
    float scale;
};
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
__device__ __forceinline__ bool take_strip(const PackParams<T>& p, int side, int wg, Strip<T>& s) {
    const PackHeader* h = reinterpret_cast<const PackHeader*>(p.plan + p.header);
    const int i = wg / p.nkv;
    if (!pack_matches(h, p.M, p.nq, p.nkv, p.causal) || i >= h->items[side]) return false;
    s.it = pack_items(p.plan, p.items[side])[i];
    s.hk = wg - i * p.nkv;
    s.ld = (int64_t)(p.nq + 2 * p.nkv) * p.dh;
    s.ldo = (int64_t)p.nq * p.dh;
    s.rows = s.it.len * p.G;
    s.q = p.qkv + s.it.t0 * s.ld + (int64_t)s.hk * p.G * p.dh;
    s.k = p.qkv + s.it.t0 * s.ld + (int64_t)(p.nq + s.hk) * p.dh;
    s.v = s.k + (int64_t)p.nkv * p.dh;
    s.row0 = (int64_t)s.it.t0 * p.nq + (int64_t)s.hk * p.G;
    return true;
}
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

// Joins the chunks of the strips that were cut, in chunk order: largest reference point, rescale, add.  Workgroup = (16 rows of a
// strip, key head).
constexpr int JOIN_ROWS = 16, JOIN_WGS = PACK_BLK / JOIN_ROWS;
template <typename T, int DH>
__global__ __launch_bounds__(256) void attn_packed_fwd_join_kernel(PackParams<T> p) {
    constexpr int PSZ = PACK_BLK * (DH + 2);
    const PackHeader* h = reinterpret_cast<const PackHeader*>(p.plan + p.header);
    const int hk = blockIdx.x % p.nkv, rest = blockIdx.x / p.nkv, j = rest / JOIN_WGS;
    if (!pack_matches(h, p.M, p.nq, p.nkv, p.causal) || j >= h->joins[0]) return;
    const PackItem it = pack_items(p.plan, p.joins[0])[j];
    const int rl = (rest % JOIN_WGS) * JOIN_ROWS + threadIdx.x / 16, r = it.first + rl;
    if (r >= it.len * p.G) return;
    const Row w = row_of(p, r);
    const float* p0 = p.part[0] + ((int64_t)it.slot * p.nkv + hk) * PSZ;
    const int64_t next = (int64_t)p.nkv * PSZ;
    float top = -INFINITY;
    for (int c = 0; c < it.chunks; ++c) top = fmaxf(top, p0[c * next + PACK_BLK * DH + rl]);
    const float mu = top == -INFINITY ? 0.0f : top;
    float total = 0.0f, v[DH / 16];
#pragma unroll
    for (int e = 0; e < DH / 16; ++e) v[e] = 0.0f;
    for (int c = 0; c < it.chunks; ++c) {
        const float* pc = p0 + c * next;
        const float f = pack_exp<T>(pc[PACK_BLK * DH + rl] - mu);
        if (f == 0.0f) continue;                                  // a chunk of masked keys: what it holds is not read
        total = fmaf(pc[PACK_BLK * DH + PACK_BLK + rl], f, total);
#pragma unroll
        for (int e = 0; e < DH / 16; ++e) v[e] = fmaf(pc[rl * DH + (threadIdx.x & 15) + 16 * e], f, v[e]);
    }
    const int64_t head = (int64_t)hk * p.G + w.g;
    T* op = p.o + ((int64_t)(it.t0 + w.q) * p.nq + head) * p.dh;
    const float inv = 1.0f / total;
#pragma unroll
    for (int e = 0; e < DH / 16; ++e) {
        const int d = (threadIdx.x & 15) + 16 * e;
        if (d < p.dh) op[d] = (T)(v[e] * inv);
    }
    if ((threadIdx.x & 15) == 0) p.lse[(int64_t)(it.t0 + w.q) * p.nq + head] = pack_lse<T>(top, total);
}

// ---- D = rowsum(dO * O) of every row and head -------------------------------------------------------------------------------
// A quarter wavefront to a row of 8-element chunks.
template <typename T>
__global__ __launch_bounds__(256) void attn_packed_dsum_kernel(const T* __restrict__ o, const T* __restrict__ d_o, float* __restrict__ dsum, int64_t rows, int dh) {
    const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    const int c = (threadIdx.x & 15) * 8;
    float a = 0.0f;
    if (row < rows && c < dh) {
        float x[8], y[8];
        load8(o + row * dh + c, x);
        load8(d_o + row * dh + c, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) a = fmaf(x[e], y[e], a);
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) a += __shfl_xor(a, off, 64);
    if (row < rows && c == 0) dsum[row] = a;
}

// dQ, dK and dV of the strips that were cut: the sums of their chunks in chunk order.  blockIdx.y = 0: dQ, 1: dK, 2: dV.
template <typename T, int DH>
__global__ __launch_bounds__(256) void attn_packed_bwd_join_kernel(PackParams<T> p) {
    const PackHeader* h = reinterpret_cast<const PackHeader*>(p.plan + p.header);
    const int which = blockIdx.y, side = which > 0;
    const int hk = blockIdx.x % p.nkv, rest = blockIdx.x / p.nkv, j = rest / JOIN_WGS;
    if (!pack_matches(h, p.M, p.nq, p.nkv, p.causal) || j >= h->joins[side]) return;
    const PackItem it = pack_items(p.plan, p.joins[side])[j];
    const int rl = (rest % JOIN_WGS) * JOIN_ROWS + threadIdx.x / 16, r = it.first + rl;
    if (r >= (side ? it.len : it.len * p.G)) return;
    const int PSZ = (side ? 2 : 1) * PACK_BLK * DH;
    const float* p0 = p.part[side] + ((int64_t)it.slot * p.nkv + hk) * PSZ + (which == 2 ? PACK_BLK * DH : 0) + rl * DH + (threadIdx.x & 15);
    float v[DH / 16];
#pragma unroll
    for (int e = 0; e < DH / 16; ++e) v[e] = 0.0f;
    for (int c = 0; c < it.chunks; ++c)
#pragma unroll
        for (int e = 0; e < DH / 16; ++e) v[e] += p0[(int64_t)c * p.nkv * PSZ + 16 * e];
    const Row w = side ? Row{r, 0} : row_of(p, r);
    const int64_t head = side ? p.nq + (which == 2 ? p.nkv : 0) + hk : hk * p.G + w.g;
    T* out = p.dqkv + ((int64_t)(it.t0 + w.q) * (p.nq + 2 * p.nkv) + head) * p.dh;
    const float f = which == 2 ? 1.0f : p.scale;
#pragma unroll
    for (int e = 0; e < DH / 16; ++e) {
        const int d = (threadIdx.x & 15) + 16 * e;
        if (d < p.dh) out[d] = (T)(v[e] * f);
    }
}

template <typename T>
PackParams<T> make_params(const PackAttnArgs& a, const PackLayout& L) {
    PackParams<T> p{};
    p.M = (int)a.M; p.nq = a.nq; p.nkv = a.nkv; p.G = a.nq / a.nkv; p.dh = a.dh; p.causal = a.causal;
    p.div_g = 65536u / (unsigned)p.G + 1u;
    p.plan = a.plan; p.header = L.header;
    for (int s = 0; s < 2; ++s) { p.items[s] = L.items[s]; p.joins[s] = L.joins[s]; }
    p.qkv = (const T*)a.qkv; p.o = (T*)a.o; p.lse = a.lse;
    p.d_o = (const T*)a.d_o; p.dqkv = (T*)a.dqkv; p.dsum = a.dsum;
    p.scale = 1.0f / sqrtf((float)a.dh);
    return p;
}
int padded(int dh) { return (dh + 31) / 32 * 32; }
struct Ws { int64_t slots; size_t part[2], total; };
Ws ws_of(const PackAttnArgs& a, bool bwd) {
    const int64_t slots = 2 * pack_shares(a.M, a.nq, a.nkv, compute_units()) * a.nkv;     // see pack_layout: a cut strip of n tiles has at most 2 n / chunk chunks
    const int DH = padded(a.dh);
    Ws w{slots, {0, 0}, 0};
    w.part[0] = (size_t)slots * PACK_BLK * (bwd ? DH : DH + 2) * sizeof(float);
    w.part[1] = bwd ? (size_t)slots * 2 * PACK_BLK * DH * sizeof(float) : 0;
    w.total = w.part[0] + w.part[1];
    return w;
}

}  // namespace
}  // namespace tpl
