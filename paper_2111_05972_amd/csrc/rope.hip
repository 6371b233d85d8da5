// Rotary positions for gfx950: the first `rot` columns of every q and k head in rows of (q | k | v, head, dh) are turned, pair by
// pair, by the angle position * frequency; backward turns back.  Bound by memory: every element is read and written once.
//
// Angles are worked out here and not read from a table: one per (token, pair), shared by all heads through LDS.  position *
// frequency is a product of 64 bits whose whole turns are taken off before it is rounded to 32 (at position 1e6 a 32-bit angle
// would be off by 0.03), so there is no largest position and nothing to keep.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_math.h"
#include "kernels.h"

namespace tpl {
namespace {

constexpr int RT = 256;                 // threads
constexpr int ROPE_LDS_PAIRS = 4096;    // (token, pair) values of a workgroup at most: 32 KiB

struct RopeParams {
    int64_t M, seq;
    int heads, turned, dh, rot, adjacent, in_place, tokens;   // heads of a row, of which the first `turned` are turned; tokens of a workgroup
    const double* freq;
    float factor, back;                                       // back: -1 in backward
    const int* pos;
};

// E elements at a time, 8 (16-byte accesses) or 1.
template <typename T, int E> __device__ __forceinline__ void load_e(const T* p, float (&v)[E]) {
    if constexpr (E == 8) load8(p, v);
    else v[0] = to_f32(p[0]);
}
template <typename T, int E> __device__ __forceinline__ void store_e(T* p, const float (&v)[E]) {
    if constexpr (E == 8) store8(p, v);
    else p[0] = from_f32<T>(v[0]);
}

// A unit of a head: E pairs (their 2 E elements; E / 2 pairs where neighbours are pairs and E is 8), or E elements that are copied.
template <typename T, int E, bool ADJ>
__global__ __launch_bounds__(RT) void rope_kernel(RopeParams p, const T* in, T* out) {
    extern __shared__ float2 cs[];
    const int t = threadIdx.x, pairs = p.rot / 2;
    const int64_t m0 = (int64_t)blockIdx.x * p.tokens;
    const int tokens = (int)(p.M - m0 < p.tokens ? p.M - m0 : p.tokens);
    for (int i = t; i < tokens * pairs; i += RT) {
        const int k = i / pairs;
        const int64_t m = m0 + k;
        const double at = p.pos ? (double)p.pos[m] : (double)(m % p.seq);
        const double turns = at * p.freq[i - k * pairs] * 0.15915494309189533577;     // of a whole circle
        float s, c;
        sincosf((float)((turns - rint(turns)) * 6.28318530717958647692), &s, &c);
        cs[i] = make_float2(c * p.factor, s * p.factor * p.back);
    }
    __syncthreads();
    constexpr int STEP = ADJ && E == 1 ? 2 : E;               // elements of a turned unit in one place
    const int nturn = ADJ ? p.rot / STEP : pairs / E;         // units of a turned head, then those that are copied
    const int ncopy = p.in_place ? 0 : (p.dh - p.rot) / E, nv = p.in_place ? 0 : p.dh / E;
    const int per_turned = nturn + ncopy, per_token = p.turned * per_turned + (p.heads - p.turned) * nv;
    const int64_t row = (int64_t)p.heads * p.dh;
    for (int i = t; i < tokens * per_token; i += RT) {
        const int k = i / per_token;
        int u = i - k * per_token, h;
        int64_t at = (m0 + k) * row;
        bool copy = true;
        if (u < p.turned * per_turned) {
            h = u / per_turned;
            u -= h * per_turned;
            copy = u >= nturn;
            at += (int64_t)h * p.dh + (copy ? p.rot + (u - nturn) * E : u * STEP);
        } else {
            u -= p.turned * per_turned;
            at += (int64_t)p.turned * p.dh + (int64_t)u * E;
        }
        float a[E], b[E];
        if (copy) {
            load_e<T, E>(in + at, a);
            store_e<T, E>(out + at, a);
            continue;
        }
        const float2* w = cs + k * pairs;
        if constexpr (ADJ && E == 8) {
            load_e<T, E>(in + at, a);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 x = w[u * 4 + e];
                b[2 * e] = fmaf(a[2 * e], x.x, -a[2 * e + 1] * x.y);
                b[2 * e + 1] = fmaf(a[2 * e], x.y, a[2 * e + 1] * x.x);
            }
            store_e<T, E>(out + at, b);
        } else {
            const int64_t other = at + (ADJ ? 1 : pairs);
            load_e<T, E>(in + at, a);
            load_e<T, E>(in + other, b);
            float c[E], d[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float2 x = w[u * E + e];
                c[e] = fmaf(a[e], x.x, -b[e] * x.y);
                d[e] = fmaf(a[e], x.y, b[e] * x.x);
            }
            store_e<T, E>(out + at, c);
            store_e<T, E>(out + other, d);
        }
    }
}

template <typename T>
hipError_t launch(const RopeArgs& a, const RopeParams& p, bool wide) {
    const dim3 grid((unsigned)((a.M + p.tokens - 1) / p.tokens));
    const size_t lds = (size_t)p.tokens * (p.rot / 2) * sizeof(float2);
    const T* in = (const T*)a.in;
    T* out = (T*)a.out;
    if (wide && a.adjacent) hipLaunchKernelGGL((rope_kernel<T, 8, true>), grid, dim3(RT), lds, a.stream, p, in, out);
    else if (wide) hipLaunchKernelGGL((rope_kernel<T, 8, false>), grid, dim3(RT), lds, a.stream, p, in, out);
    else if (a.adjacent) hipLaunchKernelGGL((rope_kernel<T, 1, true>), grid, dim3(RT), lds, a.stream, p, in, out);
    else hipLaunchKernelGGL((rope_kernel<T, 1, false>), grid, dim3(RT), lds, a.stream, p, in, out);
    return hipGetLastError();
}
}  // namespace

hipError_t rope(const RopeArgs& a, bool back) {
    RopeParams p{};
    p.M = a.M; p.seq = a.seq; p.heads = a.nq + 2 * a.nkv; p.turned = a.nq + a.nkv; p.dh = a.dh; p.rot = a.rot; p.adjacent = a.adjacent;
    p.in_place = a.in == a.out;
    p.freq = a.freq; p.factor = a.factor; p.back = back ? -1.0f : 1.0f; p.pos = a.positions;
    // Tokens of a workgroup: enough for an angle to a thread, fewer where that would leave compute units without work.
    const int64_t most = std::min<int64_t>(8, ROPE_LDS_PAIRS / (a.rot / 2)), spread = (a.M + 4 * compute_units() - 1) / (4 * compute_units());
    p.tokens = (int)std::max<int64_t>(1, std::min(most, spread));
    const bool wide = a.dh % 8 == 0 && a.rot % (a.adjacent ? 8 : 16) == 0;
    return a.dtype == BF16 ? launch<bf16_t>(a, p, wide) : launch<float>(a, p, wide);
}

}  // namespace tpl
