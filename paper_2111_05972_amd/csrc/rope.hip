// Rotary positions for gfx950: the first `rot` columns of every q and k head in rows of (q | k | v, head, dh) are turned, pair by
// pair, by the angle position * frequency; backward turns back.  Bound by memory: every element is read and written once.  8192 tokens of
// 12 + 2 x 12 heads of 128 in bf16, 151 MB: 24.5 us, 6.2 TB/s (some of it out of the infinity cache; a copy of 512 MiB reaches 5.4); 3001 tokens of
// 32 + 2 x 8 heads of 80 in float, 92 MB: 16 us, 5.8 TB/s; 64 tokens 3.3 us, a launch.  That is where the two halves of a rotation (neighbouring pairs: the
// rotation) are whole 16-byte units; otherwise every element of the row moves alone: bf16, 8192 tokens, 32 + 2 x 8 heads of 104 turned whole 40.5 us (4.0 TB/s;
// neighbouring pairs 25.8), 64 + 2 x 8 of 96 turned by 24 85 us (3.0; 38.7), 32 + 2 x 8 of 80 turned by 20 47 us (2.7).
//
// Angles are worked out here and not read from a table: one per (token, pair), shared by all heads through LDS.  position *
// frequency is a product of 64 bits whose whole turns are taken off before it is rounded to 32 (at position 1e6 a 32-bit angle
// would be off by 0.03), so there is no largest position and nothing to keep.  What is left, half a circle at most, is an angle of 32 bits, off by 2^-24 of
// itself: rows of float are 1.5 times as far from 64 bits as with sine and cosine rounded once.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_math.h"
#include "kernels.h"

namespace tpl {
namespace {

constexpr int RT = 256;                 // threads
constexpr int UNITS = 6;
constexpr int ROPE_LDS_PAIRS = 4096;    // (token, pair) values of a workgroup at most: 32 KiB

struct RopeParams {
    int64_t M, seq;
    int heads, turned, dh, rot;           // heads of a row, of which the first `turned` are turned
    int tokens;                           // of a workgroup
    // Units of work, E elements or a pair of E elements: of a turned head (pairs, then what is copied), of a row.
    int turn_units, head_units, row_units;
    unsigned div_head;                    // u / head_units = u * div_head >> 31
    int next_token, next_unit;            // RT units further
    const double* freq;
    float factor, back;                   // back: -1 in backward
    const int* pos;
};

// E elements at a time: 16 bytes, or one.  Wide stores have the non-temporal hint: the lines leave as they are written, and the kernel's end does
// not wait for those that L2 holds (8192 tokens of 12 + 2 x 12 heads of 128, both directions, 70 -> 63 us; 2048 20.6 -> 15.6).
template <typename T> constexpr int wide() { return 16 / sizeof(T); }
template <typename T, int E> __device__ __forceinline__ void load_e(const T* p, float (&v)[E]) {
    if constexpr (E == 8) {
        load8(p, v);
    } else if constexpr (E == 4) {
        const float4 a = *reinterpret_cast<const float4*>(p);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    } else {
        v[0] = to_f32(p[0]);
    }
}
template <typename T, int E> __device__ __forceinline__ void store_e(T* p, const float (&v)[E]) {
    if constexpr (E == 8) {
        store8_nt(p, v);
    } else if constexpr (E == 4) {
        const u32x4_t u = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        __builtin_nontemporal_store(u, reinterpret_cast<u32x4_t*>(p));
    } else {
        p[0] = from_f32<T>(v[0]);
    }
}
// Where a unit lies: element offsets of its two places (the same where there is one), its first pair, -1: copied.
struct Place { int64_t a, b; int pair; };

// A thread takes every RT-th unit of its workgroup's tokens, AHEAD of them at a time: their loads go out before the first is used, those of
// the first ones before the angles are worked out.
template <typename T, int E, bool ADJ>
__global__ __launch_bounds__(RT) void rope_kernel(RopeParams p, const T* in, T* out) {
    extern __shared__ float2 cs[];
    constexpr int AHEAD = 4;
    constexpr int STEP = ADJ && E == 1 ? 2 : E;               // elements of a turned unit in one place
    constexpr bool TWO = !(ADJ && E > 1);                    // a turned unit lies in two places
    constexpr int PAIRS = ADJ && E > 1 ? E / 2 : E;              // of a turned unit
    const int t = threadIdx.x, pairs = p.rot / 2;
    const int64_t m0 = (int64_t)blockIdx.x * p.tokens, row = (int64_t)p.heads * p.dh;
    const int tokens = (int)(p.M - m0 < p.tokens ? p.M - m0 : p.tokens);
    int token = t / p.row_units, unit = t - token * p.row_units;
    Place at[AHEAD];
    int of[AHEAD];                                            // token, or past the last
    float x[AHEAD][E], y[AHEAD][E];
    auto request = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            of[j] = token;
            if (token < tokens) {
                const int h = (int)(((uint64_t)(unsigned)unit * p.div_head) >> 31);
                Place q;
                if (h < p.turned) {
                    const int u = unit - h * p.head_units;
                    const bool copy = u >= p.turn_units;
                    q.a = (m0 + token) * row + (int64_t)h * p.dh + (copy ? p.rot + (u - p.turn_units) * E : u * STEP);
                    q.pair = copy ? -1 : u * PAIRS;
                    q.b = q.a + (copy ? 0 : ADJ ? 1 : pairs);
                } else {
                    q.a = q.b = (m0 + token) * row + (int64_t)p.turned * p.dh + (int64_t)(unit - p.turned * p.head_units) * E;
                    q.pair = -1;
                }
                at[j] = q;
                load_e<T, E>(in + q.a, x[j]);
                if (TWO && q.pair >= 0) load_e<T, E>(in + q.b, y[j]);
            }
            token += p.next_token;
            unit += p.next_unit;
            if (unit >= p.row_units) { unit -= p.row_units; ++token; }
        }
    };
    request();
    for (int i = t; i < tokens * pairs; i += RT) {
        const int k = i / pairs;
        const int64_t m = m0 + k;
        const double where = p.pos ? (double)p.pos[m] : (double)(m % p.seq);
        const double turns = where * p.freq[i - k * pairs] * 0.15915494309189533577;     // of a whole circle
        float s, c;
        sincosf((float)((turns - rint(turns)) * 6.28318530717958647692), &s, &c);
        cs[i] = make_float2(c * p.factor, s * p.factor * p.back);
    }
    __syncthreads();
    while (true) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (of[j] >= tokens) return;
            if (at[j].pair < 0) {
                store_e<T, E>(out + at[j].a, x[j]);
                continue;
            }
            const float2* w = cs + of[j] * pairs + at[j].pair;
            float c[E], d[E];
            if constexpr (TWO) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    c[e] = fmaf(x[j][e], w[e].x, -y[j][e] * w[e].y);
                    d[e] = fmaf(x[j][e], w[e].y, y[j][e] * w[e].x);
                }
                store_e<T, E>(out + at[j].b, d);
            } else {
#pragma unroll
                for (int e = 0; e < E / 2; ++e) {
                    c[2 * e] = fmaf(x[j][2 * e], w[e].x, -x[j][2 * e + 1] * w[e].y);
                    c[2 * e + 1] = fmaf(x[j][2 * e], w[e].y, x[j][2 * e + 1] * w[e].x);
                }
            }
            store_e<T, E>(out + at[j].a, c);
        }
        request();
    }
}

template <typename T>
hipError_t launch(const RopeArgs& a, const RopeParams& p, int E) {
    const dim3 grid((unsigned)((a.M + p.tokens - 1) / p.tokens));
    const size_t lds = (size_t)p.tokens * (p.rot / 2) * sizeof(float2);
    const T* in = (const T*)a.in;
    T* out = (T*)a.out;
    if (E > 1 && a.adjacent) hipLaunchKernelGGL((rope_kernel<T, wide<T>(), true>), grid, dim3(RT), lds, a.stream, p, in, out);
    else if (E > 1) hipLaunchKernelGGL((rope_kernel<T, wide<T>(), false>), grid, dim3(RT), lds, a.stream, p, in, out);
    else if (a.adjacent) hipLaunchKernelGGL((rope_kernel<T, 1, true>), grid, dim3(RT), lds, a.stream, p, in, out);
    else hipLaunchKernelGGL((rope_kernel<T, 1, false>), grid, dim3(RT), lds, a.stream, p, in, out);
    return hipGetLastError();
}
}  // namespace

hipError_t rope(const RopeArgs& a, bool back) {
    const bool in_place = a.in == a.out;
    const int W = a.dtype == BF16 ? wide<bf16_t>() : wide<float>(), E = a.dh % W == 0 && a.rot % (a.adjacent ? W : 2 * W) == 0 ? W : 1;
    RopeParams p{};
    p.M = a.M; p.seq = a.seq; p.heads = a.nq + 2 * a.nkv; p.turned = a.nq + a.nkv; p.dh = a.dh; p.rot = a.rot;
    p.freq = a.freq; p.factor = a.factor; p.back = back ? -1.0f : 1.0f; p.pos = a.positions;
    p.turn_units = a.adjacent && E > 1 ? a.rot / E : a.rot / 2 / E;
    p.head_units = p.turn_units + (in_place ? 0 : (a.dh - a.rot) / E);
    p.row_units = p.turned * p.head_units + (in_place ? 0 : a.nkv * (a.dh / E));
    p.div_head = ((1u << 31) + p.head_units - 1) / p.head_units;       // exact for row_units * head_units < 2^31: tp_layer.cpp
    p.next_token = RT / p.row_units; p.next_unit = RT % p.row_units;
    // Tokens of a workgroup: about six units to a thread, fewer where that would leave compute units without work.
    const int64_t most = std::min(std::max(UNITS * RT / p.row_units, 1), std::max(1, ROPE_LDS_PAIRS / (a.rot / 2)));
    const int64_t spread = (a.M + 4 * compute_units() - 1) / (4 * compute_units());
    p.tokens = (int)std::max<int64_t>(1, std::min(most, spread));
    return a.dtype == BF16 ? launch<bf16_t>(a, p, E) : launch<float>(a, p, E);
}

}  // namespace tpl
