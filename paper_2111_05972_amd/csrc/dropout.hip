// Dropout for gfx950: out = keep (in + bias) / (1 - p) + resid, and backward din = keep dout / (1 - p), dbias = sum of its rows.  The mask is worked
// out where it is needed and never stored: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers, SC 2011), a block of 128 bits for
// every eight neighbouring elements of the whole tensor, 16 bits an element.  Counter: number of the eight (44 bits), site (20), step (64); key: the
// seed.  So a slice draws its part of the tensor's mask whichever rank or launch works on it.
//
// An element is kept where its 16 bits are p 65536 (rounded) or more, and what is kept is multiplied by 65536 over the number of values that keep it:
// the mean is exact, p is met to 2^-17; from 1 - 2^-17 on it is 1 - 2^-16, one value of 65536 that keeps.
//
// A workgroup has a strip of columns and some rows, a thread eight columns and every so many rows, four of them requested at once.  Sums
// of dbias stay in registers until the workgroup's rows are through, are joined in LDS and left for row_sums.h: no atomics.
// Bound by memory: 4096 rows of 12288 in bf16 with bias and residual, 302 MB in 55 us (5.5 TB/s); backward 201 MB in 40 (5.0) and 4.8 for the sums.  The generator's 20 products of
// 32 x 32 bits for eight elements are half to two thirds of the vector units' time beside that.  4001 rows of 1280 in float 41 MB in 9.2 us and 10.0; 64 x 1024 3 us, a launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "device_math.h"
#include "kernels.h"
#include "row_sums.h"

namespace tpl {
namespace {

constexpr int DT = 256;                 // threads
constexpr int STRIP = 64;               // units of eight columns to a strip at most

struct DropParams {
    int64_t M, N, first, pitch;         // number of the first eight elements, and from row to row
    int units, cu, lanes;               // eights in a row, of them in a strip, row lanes of a workgroup
    int64_t rows;                       // of a workgroup
    unsigned threshold, site;
    float scale;
    const unsigned long long* rng;      // seed, step
};

struct Words { unsigned w[4]; };
__device__ __forceinline__ Words philox(unsigned long long group, unsigned site, unsigned long long step, unsigned long long seed) {
    unsigned c0 = (unsigned)group, c1 = (unsigned)(group >> 32) | site << 12, c2 = (unsigned)step, c3 = (unsigned)(step >> 32);
    unsigned k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(b >> 32) ^ c1 ^ k0;
        c1 = (unsigned)b;
        c2 = (unsigned)(a >> 32) ^ c3 ^ k1;
        c3 = (unsigned)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words{{c0, c1, c2, c3}};
}
// v where kept, scaled, and 0 elsewhere, whatever v is there.
__device__ __forceinline__ void drop8(float (&v)[8], const Words& q, unsigned threshold, float scale) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = (q.w[i] & 0xffffu) >= threshold ? v[2 * i] * scale : 0.0f;
        v[2 * i + 1] = (q.w[i] >> 16) >= threshold ? v[2 * i + 1] * scale : 0.0f;
    }
}

// in: forward's input or dout; out: forward's output or din; part: backward's sums [gridDim.y][N], or null
template <typename T, bool BIAS, bool RESID, bool SUMS>
__global__ __launch_bounds__(DT) void dropout_kernel(DropParams p, const T* in, const T* bias, const T* resid, T* out, float* part, T* dbias) {
    constexpr int AHEAD = 4;
    // Sums over rows.  Of float: four rows in 32 bits, from there on in 64, as a chain of a thread's rows (193 for 65536 rows of 12288) took dbias to seven times the
    // error of one rounding, so 1.5.  Of bf16, which is off by up to 2^-8 of itself in the end: 32 bits.
    using sum_t = std::conditional_t<sizeof(T) == 4, double, float>;
    __shared__ sum_t red[SUMS ? DT : 1][9];
    const int t = threadIdx.x, lane = t / p.cu, c = t - lane * p.cu, unit = blockIdx.x * p.cu + c;
    const bool mine = lane < p.lanes && unit < p.units;
    const int64_t end = min(p.M, ((int64_t)blockIdx.y + 1) * p.rows);
    sum_t sum[8] = {};
    float b[8] = {};
    if (mine) {
        const unsigned long long seed = p.rng[0], step = p.rng[1];
        if (BIAS) load8(bias + 8 * unit, b);
        for (int64_t m0 = (int64_t)blockIdx.y * p.rows + lane; m0 < end; m0 += AHEAD * p.lanes) {
            float v[AHEAD][8], r[AHEAD][8], some[8] = {};
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int64_t m = m0 + j * p.lanes;
                if (m >= end) break;
                load8(in + m * p.N + 8 * unit, v[j]);
                if (RESID) load8(resid + m * p.N + 8 * unit, r[j]);
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int64_t m = m0 + j * p.lanes;
                if (m >= end) break;
                if (BIAS)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[j][e] += b[e];
                if (p.threshold) drop8(v[j], philox((unsigned long long)(p.first + m * p.pitch + unit), p.site, step, seed), p.threshold, p.scale);
                if (RESID)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[j][e] += r[j][e];
                if (SUMS)
#pragma unroll
                    for (int e = 0; e < 8; ++e) some[e] += v[j][e];
                store8_nt(out + m * p.N + 8 * unit, v[j]);
            }
            if (SUMS)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += some[e];
        }
    }
    if constexpr (SUMS) {
#pragma unroll
        for (int e = 0; e < 8; ++e) red[t][e] = sum[e];
        __syncthreads();
        for (int i = t; i < 8 * p.cu; i += DT) {
            const int u = blockIdx.x * p.cu + i / 8;
            if (u >= p.units) break;
            sum_t s = red[i / 8][i % 8];
            for (int l = 1; l < p.lanes; ++l) s += red[l * p.cu + i / 8][i % 8];
            if (gridDim.y == 1) dbias[8 * u + i % 8] = from_f32<T>((float)s);
            else part[(int64_t)blockIdx.y * p.N + 8 * u + i % 8] = (float)s;
        }
    }
}

struct DropShape { int cu, lanes; int64_t rows, strips, slabs; };
// Strips as equal as they come, rows so that eight workgroups to a unit find work, no fewer than a thread requests at once.
DropShape shape_of(int64_t M, int64_t N) {
    DropShape s;
    const int64_t units = N / 8;
    s.strips = (units + STRIP - 1) / STRIP;
    s.cu = (int)((units + s.strips - 1) / s.strips);
    s.lanes = DT / s.cu;
    const int64_t slabs = std::max<int64_t>(1, std::min<int64_t>(65535, 8 * compute_units() / s.strips));
    s.rows = (std::max<int64_t>((M + slabs - 1) / slabs, 1) + s.lanes - 1) / s.lanes * s.lanes;
    s.slabs = (M + s.rows - 1) / s.rows;
    return s;
}
template <typename T, bool BIAS, bool RESID, bool SUMS>
hipError_t launch(const DropoutArgs& a, const DropShape& s, const DropParams& p) {
    hipLaunchKernelGGL((dropout_kernel<T, BIAS, RESID, SUMS>), dim3((unsigned)s.strips, (unsigned)s.slabs), dim3(DT), 0, a.stream, p, (const T*)a.in, (const T*)a.bias,
                       (const T*)a.resid, (T*)a.out, (float*)a.ws, (T*)a.dbias);
    return hipGetLastError();
}
template <typename T>
hipError_t run(const DropoutArgs& a) {
    const DropShape s = shape_of(a.M, a.N);
    DropParams p{};
    p.M = a.M; p.N = a.N; p.pitch = a.width / 8; p.first = a.first_row * p.pitch + a.first_col / 8;
    p.units = (int)(a.N / 8); p.cu = s.cu; p.lanes = s.lanes; p.rows = s.rows;
    p.threshold = (unsigned)std::min(65535.0, a.p * 65536.0 + 0.5);
    p.scale = (float)(65536.0 / (65536 - (int)p.threshold));
    p.site = (unsigned)a.site; p.rng = (const unsigned long long*)a.rng;
    if (a.dbias) {
        const hipError_t e = launch<T, false, false, true>(a, s, p);
        return e != hipSuccess || s.slabs == 1 ? e : row_sums<T>(s.slabs, a.N, a.N, (const float*)a.ws, a.dbias, nullptr, a.stream);
    }
    if (a.bias) return a.resid ? launch<T, true, true, false>(a, s, p) : launch<T, true, false, false>(a, s, p);
    return a.resid ? launch<T, false, true, false>(a, s, p) : launch<T, false, false, false>(a, s, p);
}
}  // namespace

size_t dropout_workspace_bytes(int64_t M, int64_t N) { return (size_t)shape_of(M, N).slabs * (size_t)N * sizeof(float); }
hipError_t dropout(const DropoutArgs& a) { return a.dtype == BF16 ? run<bf16_t>(a) : run<float>(a); }

}  // namespace tpl
