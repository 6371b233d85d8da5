// Building blocks of the float attention kernels for gfx950: LDS tiles of 32 rows, products on MFMA 32x32x2 f32, rows as operands, the sum
// of four wavefronts' blocks.  Register layouts: see attn_f32.hip.
#pragma once
#include <hip/hip_runtime.h>

#include "device_math.h"
#include "lds_dma.h"

namespace tpl {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int XT = 32;                         // rows of a tile
constexpr unsigned X_OOB = 0x80000000u;
#define MFMA32(a, b, c) __builtin_amdgcn_mfma_f32_32x32x2f32((a), (b), (c), 0, 0, 0)

// Tile of 32 rows x DH floats in LDS: chunk (16 bytes) c of row r at position c ^ xswz(r) of its row.  Two kinds of read:
// 16 bytes of 16 consecutive rows at one chunk, and single floats of 32 consecutive columns of rows r and r + 4.
template <int DH> __device__ __forceinline__ int xswz(int r) {
    if ((DH / 4) % 16 == 0) return (((r >> 2) & 1) << 3) | (((r >> 3) & 1) << 2) | (r & 3);
    return (r >> 1) & 7;                        // rows of 128 or 384 bytes: neighbours already differ by half a bank line
}
template <int DH> constexpr int xtile_bytes() { return XT * DH * 4; }
template <int DH> constexpr int xloads() { return DH / 8; }           // direct loads per lane and tile (one wavefront)

template <int DH>
__device__ __forceinline__ void xoffsets(unsigned (&off)[xloads<DH>()], int64_t ld, int dh, int lane) {
    constexpr int NC = DH / 4;
#pragma unroll
    for (int i = 0; i < xloads<DH>(); ++i) {
        const int p = lane + 64 * i, r = p / NC, c = (p % NC) ^ xswz<DH>(r);
        off[i] = 4 * c < dh ? (unsigned)r * (unsigned)(ld * 4) + (unsigned)c * 16u : X_OOB;
    }
}
template <int DH>
__device__ __forceinline__ void xfetch(const i32x4& rsrc, unsigned lds, const unsigned (&off)[xloads<DH>()], int row0, int64_t ld) {
    const unsigned r0 = (unsigned)row0 * (unsigned)(ld * 4);
#pragma unroll
    for (int i = 0; i < xloads<DH>(); ++i) buffer_load_lds_b128(rsrc, lds + i * 1024, off[i] + r0);
}
template <int N> __device__ __forceinline__ void xwait() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }
// The LDS reads issued so far have delivered: their slot may be overwritten.
__device__ __forceinline__ void xreads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// acc += T[32 rows] R^T over the head dimension: rows of the LDS tile against the lane's register row
template <int DH>
__device__ __forceinline__ f32x16 xscores(const char* tile, const float (&r)[DH / 2], int lane) {
    const int row = lane & 31, half = lane >> 5, x = xswz<DH>(row);
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.0f;
#pragma unroll
    for (int g = 0; g < DH / 8; ++g) {
        const float4 a = *reinterpret_cast<const float4*>(tile + row * (DH * 4) + (((2 * g + half) ^ x) << 4));
        s = MFMA32(a.x, r[4 * g + 0], s);
        s = MFMA32(a.y, r[4 * g + 1], s);
        s = MFMA32(a.z, r[4 * g + 2], s);
        s = MFMA32(a.w, r[4 * g + 3], s);
    }
    return s;
}
// acc[d block][.] += T^T W: sum over the 32 tile rows, weights in accumulator order
template <int DH>
__device__ __forceinline__ void xaccumulate(f32x16 (&acc)[DH / 32], const char* tile, const f32x16& w, int lane) {
    const int half = lane >> 5, col = lane & 31;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int r = 8 * (v >> 2) + 4 * half + (v & 3);
#pragma unroll
        for (int d = 0; d < DH / 32; ++d) {
            const int c = (d * 32 + col) >> 2;
            const float a = *reinterpret_cast<const float*>(tile + r * (DH * 4) + ((c ^ xswz<DH>(r)) << 4) + (col & 3) * 4);
            acc[d] = MFMA32(a, w[v], acc[d]);
        }
    }
}
// The lane's row (of 32) of a row-major global matrix in operand order; zero past nrows and past dh.
template <int DH>
__device__ __forceinline__ void xrow(float (&r)[DH / 2], const float* base, int64_t ld, int row, int nrows, int dh, int lane) {
    const int half = lane >> 5;
#pragma unroll
    for (int g = 0; g < DH / 8; ++g) {
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const int d = 8 * g + 4 * half;
        if (row < nrows && d < dh) v = *reinterpret_cast<const float4*>(base + (int64_t)row * ld + d);
        r[4 * g] = v.x; r[4 * g + 1] = v.y; r[4 * g + 2] = v.z; r[4 * g + 3] = v.w;
    }
}
__device__ __forceinline__ i32x4 xrsrc(const float* base, int64_t ld, int S, int dh) {
    return make_rsrc(base, (unsigned)(((int64_t)(S - 1) * ld + dh) * 4));
}
__device__ __forceinline__ float xother(float v) { return __shfl_xor(v, 32, 64); }

// Adds the four wavefronts' blocks in wavefront order, each scaled by its f, and hands element (row 8 i + 4 half + j,
// column) to put(d block, i, four rows' values): wavefront w writes accumulator quads w of every block, rows for which
// xmine(row, w).  Returns 0, or NaN if one of the lane's values is not finite.
//
// Infinities and NaN under the causal mask.  The matrix instruction multiplies a masked weight, zero, with its row, and zero
// times infinity is NaN: in the tile that the diagonal crosses, a token would reach tokens before it.  A wavefront that ends
// with a value that is not finite therefore computes what it has written again, row by row, where a masked row is not read
// (attn_rows.h; LDS at xrows).
__device__ __forceinline__ bool xmine(int row, int wave) { return ((row >> 3) & 3) == wave; }
template <int DH, typename Put>
__device__ __forceinline__ float xcombine(char* smem, const f32x16 (&acc)[DH / 32], const float (&f)[4], int wave, int lane, Put put) {
    float* red = reinterpret_cast<float*>(smem);                  // [wavefront][block][register][lane]
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) red[((wave * (DH / 32) + d) * 16 + v) * 64 + lane] = acc[d][v];
    __syncthreads();
    float z = 0.0f;
#pragma unroll
    for (int d = 0; d < DH / 32; ++d) {
        float r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int v = wave * 4 + j;
            float s = red[(d * 16 + v) * 64 + lane] * f[0];
#pragma unroll
            for (int w = 1; w < 4; ++w) s = fmaf(red[((w * (DH / 32) + d) * 16 + v) * 64 + lane], f[w], s);
            r[j] = s;
            z = fmaf(s, 0.0f, z);
        }
        put(d, wave, r);
    }
    return z;
}

// two tiles per wavefront (also the combine area), row terms, two rows per wavefront for attn_rows.h
template <int DH> constexpr int xlds_bytes() { return 4 * 2 * xtile_bytes<DH>() + 4 * 2 * XT * 4 + 4 * 2 * DH * 4; }
template <int DH> __device__ __forceinline__ float* xrows(char* smem, int wave) {
    return reinterpret_cast<float*>(smem + 4 * 2 * xtile_bytes<DH>() + 4 * 2 * XT * 4) + wave * 2 * DH;
}

}  // namespace tpl
