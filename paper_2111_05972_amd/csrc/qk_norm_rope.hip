// RMS norm of every query and key head and the rotation of rope.hip in one pass over rows of (q | k | v, head, dh), for gfx950:
//   y = turn(xh gamma), xh = x rstd, rstd = 1 / sqrt(mean(x^2) + eps)            v is copied
// and backward, with g = turn back(dy) and everything worked out again from x:
//   dx = rstd (g gamma - xh mean(g gamma xh)),  dgamma = sum of g xh over rows (and heads, where one row of weights is for all)
//
// Bound by memory, with vector work close behind (72 % of the vector units' time in bf16, 58 in float: widening, the norm and the rotation are about ten operations an element;
// reads of angles, 64 bytes from lane to lane with halves in bf16, keep LDS busy for 25 to 30 % of the cycles, 18 to 20 of them conflicts).  A
// group of 1 to 64 neighbouring lanes has a head of a row, a lane two units of it: the two places of the pairs that it turns, or any two where a pair lies in
// one unit; units of neighbouring lanes are neighbours (units of a lane side by side took 46.8 us instead of 34.1 in float).  A unit is 16 bytes, or 8 or 4 where the
// halves of a rotation are no multiple of that; where these are not even, a head's values go through LDS to their partners.  Sums over a head take log2(lanes) steps
// inside the wavefront.  Angles are one per (token, pair) for all heads, through LDS.  Backward: a group keeps its head over the rows of its workgroup, with gamma and the
// sums of dgamma in registers; a workgroup's sums are joined in LDS and left for row_sums.h: no atomics.
// 8192 tokens in bf16: 12 + 2 x 12 heads of 128, forward 151 MB in 25.6 us (5.9 TB/s), backward 201 MB in 39.7 (5.1) and 4.6 for the sums; 32 + 2 x 8 heads, weights for each head,
// neighbouring pairs, 201 MB in 32.7 (6.2) and 285 MB in 50.8 (5.6).  3001 tokens in float, 32 + 2 x 8 heads of 80: 92 MB in 18.4 us (5.0) and 130 MB in 25.4 (5.1).  64 tokens: 4 us, a launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "device_math.h"
#include "kernels.h"
#include "row_sums.h"

namespace tpl {
namespace {

constexpr int FWD_THREADS = 256, FWD_HEADS = 4;   // heads that a group of lanes takes
constexpr int MAX_THREADS = 512;
constexpr int ANGLES = 4096;            // (token, pair) values of a workgroup at most: 32 KiB of LDS
enum Mode { HALVES = 0, NEIGHBOURS = 1, APART = 2, NEIGHBOURS_SOME = 3 };     // APART: halves that are not whole units; SOME: not the whole head is turned

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

// A unit: E elements of T, 16 bytes, or 8 or 4 where the halves of a rotation are no multiple of that.
template <typename T> constexpr int unit() { return 16 / sizeof(T); }
template <int WORDS> struct RawOf { typedef unsigned type __attribute__((ext_vector_type(WORDS))); };
template <> struct RawOf<1> { typedef unsigned type; };
template <typename T, int E> using Raw = typename RawOf<E * sizeof(T) / 4>::type;
template <typename R> __device__ __forceinline__ unsigned word(const R& u, int i) {
    if constexpr (sizeof(R) == 4) return u;
    else return u[i];
}
template <typename T, int E> __device__ __forceinline__ void widen(const Raw<T, E>& u, float (&v)[E]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = __uint_as_float(word(u, i));
    } else {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) { v[2 * i] = __uint_as_float(word(u, i) << 16); v[2 * i + 1] = __uint_as_float(word(u, i) & 0xffff0000u); }
    }
}
template <typename T, int E> __device__ __forceinline__ Raw<T, E> narrow(const float (&v)[E]) {
    constexpr int WORDS = E * sizeof(T) / 4;
    unsigned w[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i)
        w[i] = sizeof(T) == 4 ? __float_as_uint(v[i])
                              : (unsigned)__builtin_bit_cast(unsigned short, (bf16_t)v[2 * i % E]) | ((unsigned)__builtin_bit_cast(unsigned short, (bf16_t)v[(2 * i + 1) % E]) << 16);
    Raw<T, E> u;
    if constexpr (WORDS == 1) u = w[0];
    else
#pragma unroll
        for (int i = 0; i < WORDS; ++i) u[i] = w[i];
    return u;
}

// The compiler is to widen again what it has widened before: 8 registers of a row kept instead of 16.
template <typename R> __device__ __forceinline__ void again(R& u) { asm volatile("" : "+v"(u)); }

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

// Sine and cosine of position * frequency, times the factor.  Whole quarters of a turn are taken off in 64 bits; what is left, an eighth at most, is an
// angle of 32 bits (off by 2^-24 of at most 0.79) for the Taylor series of both, whose first terms left out are below 2^-29 and 2^-33.
__device__ __forceinline__ float2 angle(double where, double freq, float factor, float back) {
    const double quarters = where * freq * 0.63661977236758134308, whole = rint(quarters);
    const float x = (float)((quarters - whole) * 1.57079632679489661923), z = x * x;
    const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), x);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
    const int q = (int)(whole - 4.0 * floor(whole * 0.25));       // 0 .. 3
    const float cq = q & 1 ? s : c, sq = q & 1 ? c : s;
    return make_float2((q == 1 || q == 2 ? -cq : cq) * factor, (q >= 2 ? -sq : sq) * factor * back);
}

// What a lane has of a head.
template <int MODE, int E>
struct Slot {
    int number, a, b;                                             // its two units begin at elements a and b
    bool turned, has_a, has_b;
    __device__ __forceinline__ Slot(const NormParams& p, int slot) {
        const int half = p.rot / 2, turning = MODE == HALVES ? half / E : 0;
        number = slot;
        turned = MODE == HALVES && slot < turning;
        // neighbouring lanes have neighbouring units, so that a load or store of theirs is one piece
        a = MODE == HALVES && !turned ? p.rot + (slot - turning) * E : slot * E;
        b = a + (turned ? half : (p.slots - turning) * E);
        has_a = slot < p.slots;
        has_b = has_a && b < p.dh;
    }
    // Turns (v0, v1) by the angles at w; APART: through `mine`, the head's place in LDS.
    __device__ __forceinline__ void turn(const NormParams& p, float (&v0)[E], float (&v1)[E], const float2* w, float* mine) const {
        if constexpr (MODE == HALVES) {
            if (!turned) return;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float2 r = w[a + e];
                const float u = v0[e];
                v0[e] = fmaf(u, r.x, -v1[e] * r.y);
                v1[e] = fmaf(u, r.y, v1[e] * r.x);
            }
        } else if constexpr (MODE == NEIGHBOURS || MODE == NEIGHBOURS_SOME) {
            if (!has_a) return;
            // SOME: a pair past `rot` is left alone, as an infinity turned by nothing would make NaN of its partner (8192 tokens in bf16, 32 + 2 x 8 heads of 80 by 20, both
            // directions, 67 -> 69 us; by branches instead of selections 70)
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
                const float2 r = w[a / 2 + e], s = w[b / 2 + e];
                const float u = v0[2 * e], x = v0[2 * e + 1], z = v1[2 * e], y = v1[2 * e + 1];
                const bool one = MODE == NEIGHBOURS || a + 2 * e < p.rot, two = MODE == NEIGHBOURS || b + 2 * e < p.rot;
                v0[2 * e] = one ? fmaf(u, r.x, -x * r.y) : u;
                v0[2 * e + 1] = one ? fmaf(u, r.y, x * r.x) : x;
                v1[2 * e] = two ? fmaf(z, s.x, -y * s.y) : z;
                v1[2 * e + 1] = two ? fmaf(z, s.y, y * s.x) : y;
            }
        } else {
            // one wavefront writes and reads: what it has written is there once its LDS counter says so
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (has_a) mine[a + e] = v0[e];
                if (has_b) mine[b + e] = v1[e];
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            const int half = p.rot / 2;
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
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // read before the next head is written
        }
    }
};
// The angles of tokens m0 .. m0 + n into LDS; past the last pair none that counts.
__device__ __forceinline__ void angles_of(const NormParams& p, float2* cs, int64_t m0, int n) {
    for (int i = threadIdx.x; i < n * p.angles; i += blockDim.x) {
        const int k = i / p.angles, f = i - k * p.angles;
        const int64_t m = m0 + k;
        cs[i] = f < p.rot / 2 ? angle(p.pos ? (double)p.pos[m] : (double)(m % p.seq), p.freq[f], p.factor, p.back) : make_float2(1.0f, 0.0f);
    }
}
template <typename T> __device__ __forceinline__ const T* weights_of(const NormParams& p, const T* gamma_q, const T* gamma_k, int h) {
    return h < p.nq ? gamma_q + (p.per_head ? (int64_t)h * p.dh : 0) : gamma_k + (p.per_head ? (int64_t)(h - p.nq) * p.dh : 0);
}

// Forward: a group takes every so many heads of its workgroup's rows, AHEAD of them at a time, whose loads are out before the angles are worked out.
template <typename T, int MODE, int E>
__global__ __launch_bounds__(FWD_THREADS, 4) void qk_norm_rope_fwd_kernel(NormParams p, const T* x, T* out, const T* gamma_q, const T* gamma_k) {
    using raw_t = Raw<T, E>;
    constexpr int AHEAD = 4;
    extern __shared__ __attribute__((aligned(16))) float2 cs[];                       // [token][angle], then APART: [group][dh] floats
    const int group = threadIdx.x / p.lanes, groups = FWD_THREADS / p.lanes;
    const Slot<MODE, E> s(p, threadIdx.x & (p.lanes - 1));
    const int64_t m0 = (int64_t)blockIdx.x * p.tokens, row = (int64_t)p.row_heads * p.dh;
    const int n = (int)(p.M - m0 < p.tokens ? p.M - m0 : p.tokens);
    float* const mine = reinterpret_cast<float*>(cs + p.tokens * p.angles) + group * p.dh;
    const int next_token = groups / p.heads, next_head = groups - next_token * p.heads;
    int token = group / p.heads, head = group - token * p.heads;
    int tk[AHEAD], hd[AHEAD];
    raw_t xr[AHEAD][2];
    auto request = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            tk[j] = token;
            hd[j] = head;
            const T* from = x + (m0 + token) * row + (int64_t)head * p.dh;
            xr[j][0] = xr[j][1] = raw_t{};
            if (token < n) {
                if (s.has_a) xr[j][0] = *reinterpret_cast<const raw_t*>(from + s.a);
                if (s.has_b) xr[j][1] = *reinterpret_cast<const raw_t*>(from + s.b);
            }
            token += next_token;
            head += next_head;
            if (head >= p.heads) { head -= p.heads; ++token; }
        }
    };
    request();
    angles_of(p, cs, m0, n);
    __syncthreads();
    while (true) {
        float r[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            float x0[E], x1[E];
            widen<T, E>(xr[j][0], x0);
            widen<T, E>(xr[j][1], x1);
            r[j] = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) r[j] = fmaf(x0[e], x0[e], fmaf(x1[e], x1[e], r[j]));
            again(xr[j][0]);
            again(xr[j][1]);
        }
        group_sums(r, p.lanes);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            __builtin_amdgcn_sched_barrier(0);
            if (tk[j] >= n) continue;
            raw_t o0 = xr[j][0], o1 = xr[j][1];
            if (hd[j] < p.normed) {
                const T* w = weights_of(p, gamma_q, gamma_k, hd[j]);
                const float rstd = rsqrtf(fmaf(r[j], p.inv_dh, p.eps));
                float x0[E], x1[E], g0[E], g1[E];
                widen<T, E>(s.has_a ? *reinterpret_cast<const raw_t*>(w + s.a) : raw_t{}, g0);
                widen<T, E>(s.has_b ? *reinterpret_cast<const raw_t*>(w + s.b) : raw_t{}, g1);
                widen<T, E>(xr[j][0], x0);
                widen<T, E>(xr[j][1], x1);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    x0[e] = x0[e] * rstd * g0[e];
                    x1[e] = x1[e] * rstd * g1[e];
                }
                s.turn(p, x0, x1, cs + tk[j] * p.angles, mine);
                o0 = narrow<T, E>(x0);
                o1 = narrow<T, E>(x1);
            }
            T* to = out + (m0 + tk[j]) * row + (int64_t)hd[j] * p.dh;
            if (s.has_a) __builtin_nontemporal_store(o0, reinterpret_cast<raw_t*>(to + s.a));
            if (s.has_b) __builtin_nontemporal_store(o1, reinterpret_cast<raw_t*>(to + s.b));
        }
        if (token >= n) break;
        request();
    }
}

// Backward: a group keeps its head over the rows of its workgroup, with gamma and the sums of dgamma in registers.
template <typename T, int MODE, int E>
__global__ __launch_bounds__(MAX_THREADS, 4) void qk_norm_rope_bwd_kernel(NormParams p, const T* x, const T* up, T* out, const T* gamma_q, const T* gamma_k, float* part) {
    using raw_t = Raw<T, E>;
    extern __shared__ __attribute__((aligned(16))) float2 cs[];                       // [token][angle], then floats
    const int t = threadIdx.x, threads = blockDim.x, lanes = p.lanes, group = t / lanes;
    const Slot<MODE, E> s(p, t & (lanes - 1));
    const int row_lane = group / p.at_once, head_lane = group - row_lane * p.at_once;
    const bool has_a = s.has_a && row_lane < p.rows_at_once, has_b = s.has_b && row_lane < p.rows_at_once;
    const int64_t m0 = (int64_t)blockIdx.x * p.tokens, row = (int64_t)p.row_heads * p.dh;
    const int n = (int)(p.M - m0 < p.tokens ? p.M - m0 : p.tokens);
    // sums of dgamma, [2E][threads + 1]: of a pass (per_head), or of all of them, q, then k (where APART has its heads until then)
    float* const sums = reinterpret_cast<float*>(cs + p.chunk * p.angles);
    const int stride = threads + 1, each = p.at_once * lanes;
    float* const sums_k = sums + 2 * E * stride;
    float* const mine = sums_k + group * p.dh;                                        // APART: this group's head
    struct Both { raw_t x[2], up[2]; };
    Both one;
    auto request = [&](Both& r, int h, int k, int end) __attribute__((always_inline)) {
        const bool in = k < end && h < p.heads, wanted = in && h < p.normed;
        const int64_t at = (m0 + k) * row + (int64_t)h * p.dh;
        r.x[0] = r.x[1] = r.up[0] = r.up[1] = raw_t{};
        if (wanted && has_a) r.x[0] = *reinterpret_cast<const raw_t*>(x + at + s.a);
        if (wanted && has_b) r.x[1] = *reinterpret_cast<const raw_t*>(x + at + s.b);
        if (in && has_a) r.up[0] = *reinterpret_cast<const raw_t*>(up + at + s.a);
        if (in && has_b) r.up[1] = *reinterpret_cast<const raw_t*>(up + at + s.b);
    };
    request(one, head_lane, row_lane, min(n, p.chunk));
    angles_of(p, cs, m0, min(n, p.chunk));
    // sums of dgamma: of float in 64 bits (a chain of 400 rows in 32 took them to 5.5 times one rounding's error, so 2.9 at most, most of it the terms' own), of bf16, which is off by up to 2^-8 in the end, in 32
    using sum_t = std::conditional_t<sizeof(T) == 4, double, float>;
    sum_t d0[E], d1[E];
    auto leave = [&](float* to) __attribute__((always_inline)) {    // this thread's sums, and begin again
#pragma unroll
        for (int e = 0; e < E; ++e) {
            to[e * stride + t] = (float)d0[e];
            to[(E + e) * stride + t] = (float)d1[e];
            d0[e] = d1[e] = 0;
        }
    };
#pragma unroll
    for (int e = 0; e < E; ++e) d0[e] = d1[e] = 0;
    auto place = [&](int slot, int e) {                             // element of the head that is number e of the slot
        const Slot<MODE, E> o(p, slot);
        return e < E ? o.a + e : o.b + e - E;
    };
    bool left = false;
    __syncthreads();
    for (int h0 = 0; h0 < p.heads; h0 += p.at_once) {
        const int h = h0 + head_lane;
        const bool normed = h < p.normed;
        raw_t w0{}, w1{};
        if (!p.per_head && h >= p.nq && !left) { leave(sums); left = true; }
        if (normed) {
            const T* w = weights_of(p, gamma_q, gamma_k, h);
            if (has_a) w0 = *reinterpret_cast<const raw_t*>(w + s.a);
            if (has_b) w1 = *reinterpret_cast<const raw_t*>(w + s.b);
        }
        for (int c0 = 0; c0 < n; c0 += p.chunk) {
            const int end = min(n, c0 + p.chunk);
            if (n > p.chunk && (h0 > 0 || c0 > 0)) {                // uniform
                __syncthreads();
                angles_of(p, cs, m0 + c0, end - c0);
                __syncthreads();
            }
            auto work = [&](Both& r, int k) __attribute__((always_inline)) {
                float v0[E], v1[E], sum[2] = {0.0f, 0.0f};          // dy turned back; sums of x^2 and g gamma x
                widen<T, E>(r.up[0], v0);
                widen<T, E>(r.up[1], v1);
                s.turn(p, v0, v1, cs + (min(k, end - 1) - c0) * p.angles, mine);
                auto add = [&](const raw_t& xraw, const raw_t& w, const float (&v)[E]) __attribute__((always_inline)) {
                    float x[E], g[E];
                    widen<T, E>(xraw, x);
                    widen<T, E>(w, g);
#pragma unroll
                    for (int e = 0; e < E; ++e) { sum[0] = fmaf(x[e], x[e], sum[0]); sum[1] = fmaf(v[e] * g[e], x[e], sum[1]); }
                };
                add(r.x[0], w0, v0);
                add(r.x[1], w1, v1);
                group_sums(sum, lanes);
                again(r.x[0]);
                again(r.x[1]);
                again(w0);
                again(w1);
                raw_t o0 = r.up[0], o1 = r.up[1];
                if (normed && k < end) {
                    const float rstd = rsqrtf(fmaf(sum[0], p.inv_dh, p.eps)), c = rstd * sum[1] * p.inv_dh;
                    auto finish = [&](const raw_t& xraw, const raw_t& w, const float (&v)[E], sum_t (&d)[E]) __attribute__((always_inline)) {
                        float x[E], g[E];
                        widen<T, E>(xraw, x);
                        widen<T, E>(w, g);
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            const float u = x[e] * rstd;
                            if constexpr (sizeof(T) == 4) d[e] += v[e] * u;
                            else d[e] = fmaf(v[e], u, d[e]);
                            x[e] = rstd * fmaf(v[e], g[e], -u * c);
                        }
                        return narrow<T, E>(x);
                    };
                    o0 = finish(r.x[0], w0, v0, d0);
                    o1 = finish(r.x[1], w1, v1, d1);
                }
                if (k < end && h < p.heads) {
                    T* to = out + (m0 + k) * row + (int64_t)h * p.dh;
                    if (has_a) __builtin_nontemporal_store(o0, reinterpret_cast<raw_t*>(to + s.a));
                    if (has_b) __builtin_nontemporal_store(o1, reinterpret_cast<raw_t*>(to + s.b));
                }
                __builtin_amdgcn_sched_barrier(0);
            };
            for (int k = c0 + row_lane; k - row_lane < end; k += p.rows_at_once) {     // uniform
                if (h0 > 0 || k > row_lane) request(one, h, k, end);
                work(one, k);
            }
        }
        if (!p.per_head || h0 >= p.normed) continue;                // uniform
        leave(sums);
        __syncthreads();
        for (int i = t; i < each * 2 * E; i += threads) {
            const int e = i % (2 * E), at = i / (2 * E), slot = at & (lanes - 1), head = h0 + at / lanes, el = place(slot, e);
            if (slot >= p.slots || head >= p.normed || el >= p.dh) continue;
            sum_t v = sums[e * stride + at];
            for (int r = 1; r < p.rows_at_once; ++r) v += sums[e * stride + r * each + at];
            part[((int64_t)blockIdx.x * p.normed + head) * p.dh + el] = (float)v;
        }
        __syncthreads();
    }
    if (p.per_head) return;
    if (MODE == APART) __syncthreads();                             // all heads have been read
    if (left) leave(sums_k);
    else { leave(sums); leave(sums_k); }
    __syncthreads();
    for (int i = t; i < 2 * lanes * 2 * E; i += threads) {
        const int e = i % (2 * E), slot = i / (2 * E) & (lanes - 1), side = i / (2 * E * lanes), el = place(slot, e);
        if (slot >= p.slots || el >= p.dh) continue;
        const float* from = (side ? sums_k : sums) + e * stride + slot;
        double v = 0.0;                                             // up to 512 of them, see row_sums.h
        for (int g = 0; g < p.rows_at_once * p.at_once; ++g) v += from[g * lanes];
        part[((int64_t)blockIdx.x * 2 + side) * p.dh + el] = (float)v;
    }
}

// Workgroups of backward, each of which leaves sums: two to a compute unit at most.
int64_t tokens_each(int64_t M) { const int64_t groups = 2 * (int64_t)compute_units(); return (M + groups - 1) / groups; }

template <typename T, int MODE, int E>
hipError_t launch_fwd(const QkNormArgs& a, NormParams& p) {
    // heads of a group: one batch, fewer where units would be left without rows
    const int groups = FWD_THREADS / p.lanes;
    const int64_t most = std::max(1, FWD_HEADS * groups / p.heads), spread = (a.M + 4 * compute_units() - 1) / (4 * compute_units());
    p.tokens = (int)std::min<int64_t>(std::min(most, spread), std::max(1, ANGLES / p.angles));
    const size_t lds = (size_t)p.tokens * p.angles * sizeof(float2) + (MODE == APART ? (size_t)groups * a.dh * sizeof(float) : 0);
    hipLaunchKernelGGL((qk_norm_rope_fwd_kernel<T, MODE, E>), dim3((unsigned)((a.M + p.tokens - 1) / p.tokens)), dim3(FWD_THREADS), lds, a.stream, p, (const T*)a.qkv,
                       (T*)a.out, (const T*)a.gamma_q, (const T*)a.gamma_k);
    return hipGetLastError();
}
template <typename T, int MODE, int E>
hipError_t launch_bwd(const QkNormArgs& a, NormParams& p) {
    // Threads, heads at a time and rows at a time: as many lanes at work as there may be, and few rows more than two workgroups to a unit leave each.
    // A third of the lanes idle costs 6 % (8192 tokens, 32 + 2 x 8 heads of 128: 62 -> 58 us with 512 instead of 384 threads), a quarter more rows a quarter (12 + 2 x 12 heads: 39 -> 48).
    const int64_t spread = tokens_each(a.M);
    int threads = 0;
    double best = 1e30;
    for (int passes = 1; passes <= p.heads; ++passes) {
        const int at_once = (p.heads + passes - 1) / passes;
        if (passes > 1 && at_once == (p.heads + passes - 2) / (passes - 1)) continue;
        if (at_once * p.lanes > MAX_THREADS) continue;
        const int64_t most = std::min<int64_t>(MAX_THREADS / p.lanes / at_once, spread);
        for (int64_t rows = 1; rows <= most; ++rows) {
            const double active = (double)p.heads * rows * p.lanes / passes, more = (double)((spread + rows - 1) / rows * rows) / spread;
            const double cost = more * (1.0 + 0.2 * (MAX_THREADS / active - 1.0)) + 0.01 * passes;
            if (cost < best) { best = cost; threads = (int)(at_once * rows * p.lanes + 63) / 64 * 64; p.at_once = at_once; p.rows_at_once = (int)rows; }
        }
        if (at_once * p.lanes <= 64) break;
    }
    // no more workgroups than the workspace has rows for, whose angles come in chunks
    const int64_t fits = std::max(1, ANGLES / p.angles), step = p.rows_at_once;
    p.tokens = (int)((spread + step - 1) / step * step);
    p.chunk = (int)std::min<int64_t>(p.tokens, fits >= step ? fits / step * step : fits);
    const dim3 grid((unsigned)((a.M + p.tokens - 1) / p.tokens));
    const size_t apart = MODE == APART ? (size_t)(threads / p.lanes) * a.dh * sizeof(float) : 0, sums = (size_t)(2 * E * (threads + 1)) * sizeof(float);
    const size_t lds = (size_t)p.chunk * p.angles * sizeof(float2) + sums + std::max(apart, a.per_head ? 0 : sums);
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&qk_norm_rope_bwd_kernel<T, MODE, E>), hipFuncAttributeMaxDynamicSharedMemorySize, 112 << 10);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL((qk_norm_rope_bwd_kernel<T, MODE, E>), grid, dim3((unsigned)threads), lds, a.stream, p, (const T*)a.qkv, (const T*)a.dqkv, (T*)a.out,
                       (const T*)a.gamma_q, (const T*)a.gamma_k, (float*)a.ws);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t cols = (a.per_head ? p.normed : 2) * (int64_t)a.dh;
    return row_sums<T>(grid.x, cols, (a.per_head ? a.nq : 1) * (int64_t)a.dh, (const float*)a.ws, a.dgamma_q, a.dgamma_k, a.stream);
}
template <typename T, int MODE, int E>
hipError_t launch(const QkNormArgs& a, NormParams& p, bool bwd) {
    const int turning = MODE == HALVES ? a.rot / 2 / E : 0;
    p.slots = MODE == HALVES ? turning + ((a.dh - a.rot) / E + 1) / 2 : (a.dh + 2 * E - 1) / (2 * E);
    for (p.lanes = 1; p.lanes < p.slots; p.lanes *= 2) {}
    p.angles = MODE == NEIGHBOURS || MODE == NEIGHBOURS_SOME ? p.slots * E : a.rot / 2;
    return bwd ? launch_bwd<T, MODE, E>(a, p) : launch_fwd<T, MODE, E>(a, p);
}
template <typename T>
hipError_t run(const QkNormArgs& a, NormParams& p, bool bwd) {
    constexpr int W = unit<T>();
    if (a.adjacent) return a.rot == a.dh ? launch<T, NEIGHBOURS, W>(a, p, bwd) : launch<T, NEIGHBOURS_SOME, W>(a, p, bwd);
    const int half = a.rot / 2;
    if (half % W == 0) return launch<T, HALVES, W>(a, p, bwd);
    // Smaller units as long as a wavefront has lanes enough for a head of them: bf16, 8192 tokens, 32 + 2 x 8 heads of 104 turned whole, both directions, 145 us through
    // LDS and 79 in units of 8 bytes.  Of 4 bytes: heads of 32 turned by 4 53 and 38, of 64 by 12 68 and 63, but of 80 by 20 88 and 104, of 256 by 20 191 and 260 (forward
    // 37 and 39, 77 and 66).
    if (half % (W / 2) == 0 && a.dh <= 64 * W) return launch<T, HALVES, W / 2>(a, p, bwd);
    if constexpr (W == 8)
        if (half % 2 == 0 && a.dh <= (bwd ? 64 : 256)) return launch<T, HALVES, 2>(a, p, bwd);
    return launch<T, APART, W>(a, p, bwd);
}
}  // namespace

size_t qk_norm_rope_workspace_bytes(int64_t M, int nq, int nkv, int dh) {
    const int64_t each = tokens_each(M);
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
