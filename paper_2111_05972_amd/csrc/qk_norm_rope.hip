// RMS norm of every query and key head and the rotation of rope.hip in one pass over rows of (q | k | v, head, dh), for gfx950:
//   y = turn(xh gamma), xh = x rstd, rstd = 1 / sqrt(mean(x^2) + eps)            v is copied
// and backward, with g = turn back(dy) and everything worked out again from x:
//   dx = rstd (g gamma - xh mean(g gamma xh)),  dgamma = sum of g xh over rows (and heads, where one row of weights is for all)
//
// Bound by memory.  A group of 1 to 64 neighbouring lanes has a head of a row, a lane two units of 16 bytes of it: the two places of the pairs that it turns,
// or neighbours where a pair lies in one unit.  Where the halves of a rotation are not whole units, a head's values go through LDS to their partners.  Sums
// over a head take log2(lanes) steps inside the wavefront.  A group keeps its head over the rows of its workgroup, with gamma and the sums of dgamma in
// registers; angles as in rope.hip, one per (token, pair) for all heads.  dgamma: sums of a workgroup in LDS, then row_sums.h; no atomics.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_math.h"
#include "kernels.h"
#include "row_sums.h"

namespace tpl {
namespace {

constexpr int MAX_THREADS = 512;
constexpr int ANGLES = 4096;            // (token, pair) values of a workgroup at most: 32 KiB of LDS
enum Mode { HALVES = 0, NEIGHBOURS = 1, APART = 2 };     // APART: halves that are not whole units

struct NormParams {
    int64_t M, seq;
    int nq, normed, heads, row_heads, dh, rot;        // heads that are normed, of a pass over the row (without v in place), of a row
    int lanes, slots;                                 // of a head: a power of two, those with a unit
    int at_once, rows_at_once, tokens;                // heads and rows that a workgroup works on at a time, rows in all
    int angles, chunk;                                // of a token in LDS, and of how many tokens
    const double* freq;
    float factor, back, eps, inv_dh;
    const int* pos;
    int per_head;
};

template <typename T> constexpr int unit() { return 16 / sizeof(T); }
typedef unsigned raw_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void widen(const raw_t& u, float (&v)[8], int at = 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}
__device__ __forceinline__ void widen(const raw_t& u, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(u[i]);
}
__device__ __forceinline__ raw_t narrow(const float (&v)[8]) {
    raw_t u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        u[i] = (unsigned)__builtin_bit_cast(unsigned short, (bf16_t)v[2 * i]) | ((unsigned)__builtin_bit_cast(unsigned short, (bf16_t)v[2 * i + 1]) << 16);
    return u;
}
__device__ __forceinline__ raw_t narrow(const float (&v)[4]) { return raw_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}; }

// Sums over aligned groups of `lanes` lanes (a power of two), in all of them.
template <int CTRL> __device__ __forceinline__ float add_dpp(float x) { return x + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, true)); }
template <int N> __device__ __forceinline__ void group_sums(float (&v)[N], int lanes) {
    if (lanes > 1)
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = add_dpp<0xB1>(v[j]);        // lane ^ 1
    if (lanes > 2)
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = add_dpp<0x4E>(v[j]);        // lane ^ 2
    if (lanes > 4)
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = add_dpp<0x141>(v[j]);       // 7 - lane: the other four
    if (lanes > 8)
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = add_dpp<0x140>(v[j]);       // 15 - lane: the other eight
    for (int d = 16; d < lanes; d *= 2)
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] += __shfl_xor(v[j], d, 64);
}

template <typename T, int MODE, bool BWD>
__global__ __launch_bounds__(MAX_THREADS) void qk_norm_rope_kernel(NormParams p, const T* x, const T* up, T* out, const T* gamma_q, const T* gamma_k, float* part) {
    constexpr int E = unit<T>(), AHEAD = BWD ? 2 : 4;
    extern __shared__ __attribute__((aligned(16))) float2 cs[];                       // [token][angle], then floats
    const int t = threadIdx.x, threads = blockDim.x, lanes = p.lanes, group = t / lanes, slot = t & (lanes - 1);
    const int row_lane = group / p.at_once, head_lane = group - row_lane * p.at_once;
    const int half = p.rot / 2, turning = MODE == HALVES ? half / E : 0;              // slots that turn, HALVES
    const bool turned = MODE == HALVES && slot < turning;
    const int a = MODE == HALVES && !turned ? p.rot + (slot - turning) * 2 * E : slot * (turned ? E : 2 * E), b = turned ? a + half : a + E;
    const bool has_a = row_lane < p.rows_at_once && slot < p.slots, has_b = has_a && b < p.dh;
    const int64_t m0 = (int64_t)blockIdx.x * p.tokens, row = (int64_t)p.row_heads * p.dh;
    const int n = (int)(p.M - m0 < p.tokens ? p.M - m0 : p.tokens);
    float* const lds = reinterpret_cast<float*>(cs + p.chunk * p.angles);
    float* const mine = lds + group * p.dh;                                            // APART: this group's head

    raw_t xr[AHEAD][2], ur[AHEAD][2];
    const raw_t zero = {0u, 0u, 0u, 0u};
    auto request = [&](int h, int k0, int end) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int k = k0 + j * p.rows_at_once + row_lane;
            const bool in = k < end && h < p.heads;
            const int64_t at = (m0 + k) * row + (int64_t)h * p.dh;
            const bool wanted = in && (!BWD || h < p.normed);
            xr[j][0] = wanted && has_a ? *reinterpret_cast<const raw_t*>(x + at + a) : zero;
            xr[j][1] = wanted && has_b ? *reinterpret_cast<const raw_t*>(x + at + b) : zero;
            if (BWD) {
                ur[j][0] = in && has_a ? *reinterpret_cast<const raw_t*>(up + at + a) : zero;
                ur[j][1] = in && has_b ? *reinterpret_cast<const raw_t*>(up + at + b) : zero;
            }
        }
    };
    // Turns (v0, v1) of the chunk's token k.
    auto turn = [&](float (&v0)[E], float (&v1)[E], int k) __attribute__((always_inline)) {
        const float2* w = cs + k * p.angles;
        if constexpr (MODE == HALVES) {
            if (!turned) return;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float2 r = w[a + e];
                const float u = v0[e];
                v0[e] = fmaf(u, r.x, -v1[e] * r.y);
                v1[e] = fmaf(u, r.y, v1[e] * r.x);
            }
        } else if constexpr (MODE == NEIGHBOURS) {
            if (!has_a) return;
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
                const float2 r = w[a / 2 + e], s = w[b / 2 + e];
                const float u = v0[2 * e], z = v1[2 * e];
                v0[2 * e] = fmaf(u, r.x, -v0[2 * e + 1] * r.y);
                v0[2 * e + 1] = fmaf(u, r.y, v0[2 * e + 1] * r.x);
                v1[2 * e] = fmaf(z, s.x, -v1[2 * e + 1] * s.y);
                v1[2 * e + 1] = fmaf(z, s.y, v1[2 * e + 1] * s.x);
            }
        } else {
            // one wavefront writes and reads: what it has written is there once its LDS counter says so
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (has_a) mine[a + e] = v0[e];
                if (has_b) mine[b + e] = v1[e];
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            auto partner = [&](float& v, int i) {
                if (i >= p.rot) return;
                const bool first = i < half;
                const float2 r = w[first ? i : i - half];
                const float o = mine[first ? i + half : i - half];
                v = first ? fmaf(v, r.x, -o * r.y) : fmaf(o, r.y, v * r.x);
            };
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (has_a) partner(v0[e], a + e);
                if (has_b) partner(v1[e], b + e);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // read before the next row is written
        }
    };
    auto angles = [&](int k0, int end) __attribute__((always_inline)) {
        for (int i = t; i < (end - k0) * p.angles; i += threads) {
            const int k = i / p.angles, f = i - k * p.angles;
            const int64_t m = m0 + k0 + k;
            float s = 0.0f, c = 1.0f, by = 1.0f;                    // past the last pair: as it is
            if (f < half) {
                const double where = p.pos ? (double)p.pos[m] : (double)(m % p.seq);
                const double turns = where * p.freq[f] * 0.15915494309189533577;     // of a whole circle
                sincosf((float)((turns - rint(turns)) * 6.28318530717958647692), &s, &c);
                by = p.factor;
            }
            cs[i] = make_float2(c * by, s * by * p.back);
        }
    };
    request(head_lane, 0, min(n, p.chunk));
    angles(0, min(n, p.chunk));
    float* const sums = lds;                                        // [2E][threads + 1]: a workgroup's dgamma of a pass
    float* const total = sums + 2 * E * (threads + 1);              // [q, k][dh] of all passes, where weights are shared
    if (BWD && !p.per_head)
        for (int i = t; i < 2 * p.dh; i += threads) total[i] = 0.0f;
    __syncthreads();
    const int stride = threads + 1, each = p.at_once * lanes;
    for (int h0 = 0; h0 < p.heads; h0 += p.at_once) {
        const int h = h0 + head_lane;
        const bool normed = h < p.normed;
        float g0[E], g1[E], d0[E], d1[E];
#pragma unroll
        for (int e = 0; e < E; ++e) g0[e] = g1[e] = d0[e] = d1[e] = 0.0f;
        if (normed) {
            const T* w = h < p.nq ? gamma_q + (p.per_head ? (int64_t)h * p.dh : 0) : gamma_k + (p.per_head ? (int64_t)(h - p.nq) * p.dh : 0);
            if (has_a) widen(*reinterpret_cast<const raw_t*>(w + a), g0);
            if (has_b) widen(*reinterpret_cast<const raw_t*>(w + b), g1);
        }
        for (int c0 = 0; c0 < n; c0 += p.chunk) {
            const int end = min(n, c0 + p.chunk);
            if (n > p.chunk && (h0 > 0 || c0 > 0)) {                  // uniform
                __syncthreads();
                angles(c0, end);
                __syncthreads();
            }
            for (int k0 = c0; k0 < end; k0 += AHEAD * p.rows_at_once) {
                if (h0 > 0 || k0 > 0) request(h, k0, end);
                float r1[AHEAD], r2[AHEAD];
                float v0[AHEAD][E], v1[AHEAD][E];                       // backward: dy turned back
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    float x0[E], x1[E];
                    widen(xr[j][0], x0);
                    widen(xr[j][1], x1);
                    r1[j] = 0.0f;
#pragma unroll
                    for (int e = 0; e < E; ++e) r1[j] = fmaf(x0[e], x0[e], fmaf(x1[e], x1[e], r1[j]));
                    if constexpr (BWD) {
                        widen(ur[j][0], v0[j]);
                        widen(ur[j][1], v1[j]);
                        turn(v0[j], v1[j], min(k0 + j * p.rows_at_once + row_lane, end - 1) - c0);
                        r2[j] = 0.0f;
#pragma unroll
                        for (int e = 0; e < E; ++e) r2[j] = fmaf(v0[j][e] * g0[e], x0[e], fmaf(v1[j][e] * g1[e], x1[e], r2[j]));
                    }
                }
                group_sums(r1, lanes);
                if constexpr (BWD) group_sums(r2, lanes);
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    const int k = k0 + j * p.rows_at_once + row_lane;
                    const float rstd = 1.0f / sqrtf(fmaf(r1[j], p.inv_dh, p.eps));
                    float x0[E], x1[E];
                    widen(xr[j][0], x0);
                    widen(xr[j][1], x1);
                    raw_t o0, o1;
                    if constexpr (BWD) {
                        const float c = rstd * r2[j] * p.inv_dh;
                        float y0[E], y1[E];
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            const float u = x0[e] * rstd, z = x1[e] * rstd;
                            y0[e] = rstd * fmaf(v0[j][e], g0[e], -u * c);
                            y1[e] = rstd * fmaf(v1[j][e], g1[e], -z * c);
                            if (k < end && normed) {
                                d0[e] = fmaf(v0[j][e], u, d0[e]);
                                d1[e] = fmaf(v1[j][e], z, d1[e]);
                            }
                        }
                        o0 = normed ? narrow(y0) : ur[j][0];
                        o1 = normed ? narrow(y1) : ur[j][1];
                    } else {
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            x0[e] = x0[e] * rstd * g0[e];
                            x1[e] = x1[e] * rstd * g1[e];
                        }
                        turn(x0, x1, min(k, end - 1) - c0);
                        o0 = normed ? narrow(x0) : xr[j][0];
                        o1 = normed ? narrow(x1) : xr[j][1];
                    }
                    if (k < end && h < p.heads) {
                        T* to = out + (m0 + k) * row + (int64_t)h * p.dh;
                        if (has_a) __builtin_nontemporal_store(o0, reinterpret_cast<raw_t*>(to + a));
                        if (has_b) __builtin_nontemporal_store(o1, reinterpret_cast<raw_t*>(to + b));
                    }
                }
            }
        }
        if constexpr (!BWD) continue;
        if (h0 >= p.normed) continue;                               // uniform: v alone
        __syncthreads();                                            // the sums of the pass before have been read, and the heads of APART
#pragma unroll
        for (int e = 0; e < E; ++e) {
            sums[e * stride + t] = d0[e];
            sums[(E + e) * stride + t] = d1[e];
        }
        __syncthreads();
        auto place = [&](int s, int e) {                            // element of the head that is number e of slot s
            const bool tu = MODE == HALVES && s < turning;
            const int first = MODE == HALVES && !tu ? p.rot + (s - turning) * 2 * E : s * (tu ? E : 2 * E);
            return e < E ? first + e : tu ? first + half + e - E : first + e;
        };
        if (p.per_head) {
            for (int i = t; i < each * 2 * E; i += threads) {
                const int e = i % (2 * E), at = i / (2 * E), s = at & (lanes - 1), head = h0 + at / lanes, el = place(s, e);
                if (s >= p.slots || head >= p.normed || el >= p.dh) continue;
                float v = sums[e * stride + at];
                for (int r = 1; r < p.rows_at_once; ++r) v += sums[e * stride + r * each + at];
                part[((int64_t)blockIdx.x * p.normed + head) * p.dh + el] = v;
            }
        } else {
            for (int i = t; i < 2 * lanes * 2 * E; i += threads) {
                const int e = i % (2 * E), s = i / (2 * E) & (lanes - 1), side = i / (2 * E * lanes), el = place(s, e);
                if (s >= p.slots || el >= p.dh) continue;
                const int from = max(side ? p.nq - h0 : 0, 0), to = min((side ? p.normed : p.nq) - h0, p.at_once);
                float v = total[side * p.dh + el];
                for (int r = 0; r < p.rows_at_once; ++r)
                    for (int g = from; g < to; ++g) v += sums[e * stride + r * each + g * lanes + s];
                total[side * p.dh + el] = v;                        // this thread's alone
            }
        }
        if (MODE == APART) __syncthreads();                         // heads go where the sums were
    }
    if (BWD && !p.per_head) {
        __syncthreads();
        for (int i = t; i < 2 * p.dh; i += threads) part[(int64_t)blockIdx.x * 2 * p.dh + i] = total[i];
    }
}

// Workgroups of backward, each of which leaves sums: two to a compute unit at most.
int64_t tokens_each(int64_t M, bool bwd) { const int64_t groups = (bwd ? 2 : 4) * (int64_t)compute_units(); return (M + groups - 1) / groups; }

template <typename T, int MODE>
hipError_t launch(const QkNormArgs& a, NormParams& p, bool bwd) {
    constexpr int E = unit<T>();
    const int turning = MODE == HALVES ? a.rot / 2 / E : 0;
    p.slots = MODE == HALVES ? turning + ((a.dh - a.rot) / E + 1) / 2 : (a.dh + 2 * E - 1) / (2 * E);
    for (p.lanes = 1; p.lanes < p.slots; p.lanes *= 2) {}
    p.angles = MODE == NEIGHBOURS ? p.slots * E : a.rot / 2;
    // Threads, heads at a time and rows at a time that leave the fewest groups idle; fewer passes over the heads where that is alike.
    const int64_t spread = tokens_each(a.M, bwd);
    int threads = 0;
    double best = 0.0;
    for (int passes = 1; passes <= p.heads; ++passes) {
        const int at_once = (p.heads + passes - 1) / passes;
        if (passes > 1 && at_once == (p.heads + passes - 2) / (passes - 1)) continue;
        if (at_once * p.lanes > MAX_THREADS) continue;
        for (int th = 64; th <= MAX_THREADS; th += 64) {
            const int groups = th / p.lanes, rows = (int)std::min<int64_t>(groups / std::max(1, at_once), spread);
            if (rows < 1) continue;
            const double full = (double)p.heads * rows / ((double)passes * groups) * (th >= 256 ? 1.0 : 0.9) - 0.01 * passes;
            if (full > best) { best = full; threads = th; p.at_once = at_once; p.rows_at_once = rows; }
        }
        if (at_once * p.lanes <= 64) break;
    }
    const int64_t fits = std::max(1, ANGLES / p.angles), step = p.rows_at_once;
    // Backward: no more workgroups than the workspace has rows for, whose angles come in chunks.
    p.tokens = (int)((spread + step - 1) / step * step);
    p.chunk = (int)std::min<int64_t>(p.tokens, fits >= step ? fits / step * step : fits);
    if (!bwd) p.tokens = p.chunk;
    const dim3 grid((unsigned)((a.M + p.tokens - 1) / p.tokens));
    const size_t angles = (size_t)p.chunk * p.angles * sizeof(float2);
    const size_t apart = MODE == APART ? (size_t)(threads / p.lanes) * a.dh * sizeof(float) : 0;
    const size_t sums = bwd ? (size_t)(2 * E * (threads + 1) + 2 * a.dh) * sizeof(float) : 0;
    const size_t lds = angles + std::max(apart, sums);
    const T *x = (const T*)a.qkv, *up = (const T*)a.dqkv, *gq = (const T*)a.gamma_q, *gk = (const T*)a.gamma_k;
    if (!bwd) {
        hipLaunchKernelGGL((qk_norm_rope_kernel<T, MODE, false>), grid, dim3((unsigned)threads), lds, a.stream, p, x, up, (T*)a.out, gq, gk, nullptr);
        return hipGetLastError();
    }
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&qk_norm_rope_kernel<T, MODE, true>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 << 10);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL((qk_norm_rope_kernel<T, MODE, true>), grid, dim3((unsigned)threads), lds, a.stream, p, x, up, (T*)a.out, gq, gk, (float*)a.ws);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t cols = (a.per_head ? p.normed : 2) * (int64_t)a.dh;
    return row_sums<T>(grid.x, cols, (a.per_head ? a.nq : 1) * (int64_t)a.dh, (const float*)a.ws, a.dgamma_q, a.dgamma_k, a.stream);
}
template <typename T>
hipError_t run(const QkNormArgs& a, NormParams& p, bool bwd) {
    if (a.adjacent) return launch<T, NEIGHBOURS>(a, p, bwd);
    return a.rot % (2 * unit<T>()) == 0 ? launch<T, HALVES>(a, p, bwd) : launch<T, APART>(a, p, bwd);
}
}  // namespace

size_t qk_norm_rope_workspace_bytes(int64_t M, int nq, int nkv, int dh) {
    const int64_t each = tokens_each(M, true);
    return (size_t)((M + each - 1) / each) * ((size_t)nq + nkv) * dh * sizeof(float);
}
hipError_t qk_norm_rope(const QkNormArgs& a, bool bwd) {
    NormParams p{};
    p.M = a.M; p.seq = a.seq; p.nq = a.nq; p.normed = a.nq + a.nkv; p.row_heads = a.nq + 2 * a.nkv; p.dh = a.dh; p.rot = a.rot;
    p.heads = (bwd ? a.dqkv : a.qkv) == a.out ? p.normed : p.row_heads;
    p.freq = a.freq; p.factor = a.factor; p.back = bwd ? -1.0f : 1.0f; p.eps = a.eps; p.inv_dh = 1.0f / (float)a.dh; p.pos = a.positions; p.per_head = a.per_head;
    return a.dtype == BF16 ? run<bf16_t>(a, p, bwd) : run<float>(a, p, bwd);
}

}  // namespace tpl
