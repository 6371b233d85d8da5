// Building blocks of the bf16 attention kernels for gfx950: LDS tiles and their swizzle, direct loads of a tile, matrix operands
// from LDS and memory, weights as operands, reductions.  Register layouts: see attn_bf16.hip.
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "device_math.h"
#include "lds_dma.h"

namespace tpl {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((address_space(3))) s16x4* lds_s16x4_ptr;

constexpr int TILE = 64;           // rows of the streamed operand staged in LDS per step
constexpr float LOG2E = 1.44269504088896340736f;
constexpr float LN2 = 0.69314718055994530942f;
constexpr float RESCALE_LAG = 8.0f;  // forward: how far (log2) the row maximum may run ahead of the reference point

// ---- LDS tile of TILE rows x DH bf16, 16-byte chunks XOR-swizzled by row -------------------------
// Two kinds of read hit these tiles: 16-byte reads of 16 consecutive rows at one chunk (operand with
// the head dimension as K), and transposing 8-byte reads of 4 consecutive rows at two neighbouring
// 32-byte column groups.  The XOR below makes both conflict-free over the 64 banks (256 bytes): the
// bits that separate the 4 rows of a transposing read move the 64-byte column group, the remaining
// row bits move the chunk inside it.
template <int DH> __device__ __forceinline__ int swz(int row) {
    return DH == 64    ? ((((row >> 1) & 1) << 2) | ((row >> 2) & 3))     // 128-byte rows, 8 chunks
           : DH == 128 ? (((row & 3) << 2) | ((row >> 2) & 3))            // 256-byte rows, 16 chunks
                       : ((row >> 2) & 3);    // 64- and 192-byte rows: 4 rows already start in 4 different column groups
}
template <int DH> constexpr int tile_bytes() { return TILE * DH * 2; }
template <int DH, int NT> constexpr int NCHUNKS = (TILE * DH / 8 + NT - 1) / NT;   // 16-byte chunks per thread and tile (at most)

// ---- global -> LDS without passing through registers ---------------------------------------------
// A tile is TILE rows x DH bf16 = TILE*DH/8 chunks of 16 bytes; a buffer load with the LDS flag writes the 64
// chunks of a wavefront to 64 consecutive LDS positions.  Position p = t + NT*i (row p / NC, slot p % NC) must
// hold chunk (slot ^ swz(row)) of its row, so the swizzle is applied to the global offset each lane requests.
// Offsets are relative to row 0 of this (batch, head); the descriptor ends after the head's slice of row S-1,
// which makes rows >= S read as zero.
constexpr unsigned HEAD_OOB = 0x80000000u;      // past every slice (below 2 GiB), also with a row offset added
template <int DH, int NT>
__device__ __forceinline__ void dma_offsets(unsigned (&off)[(NCHUNKS<DH, NT>)], int64_t ld, int dh, int t) {
    constexpr int NC = DH / 8;
#pragma unroll
    for (int i = 0; i < NCHUNKS<DH, NT>; ++i) {
        const int p = t + NT * i, row = p / NC, c = (p % NC) ^ swz<DH>(row);
        off[i] = c * 8 < dh ? (unsigned)row * (unsigned)(ld * 2) + (unsigned)c * 16u : HEAD_OOB;
    }
}
__device__ __forceinline__ i32x4 head_rsrc(const bf16_t* base, int64_t ld, int S, int dh) {
    return make_rsrc(base, (unsigned)(((int64_t)(S - 1) * ld + dh) * 2));
}
// rows [row0, row0 + TILE) -> LDS tile at byte address lds_tile; wave = wavefront index (uniform)
template <int DH, int NT>
__device__ __forceinline__ void tile_dma(i32x4 rsrc, unsigned lds_tile, const unsigned (&off)[(NCHUNKS<DH, NT>)],
                                         unsigned row0_bytes, int wave) {
#pragma unroll
    for (int i = 0; i < NCHUNKS<DH, NT>; ++i)
        if ((i + 1) * NT <= TILE * DH / 8 || i * NT + wave * 64 < TILE * DH / 8)   // the last round may need some wavefronts only
            buffer_load_lds_b128(rsrc, lds_tile + (unsigned)(i * NT + wave * 64) * 16u, off[i] + row0_bytes);
}
// A use of v that the compiler must order after the load that produces v: placed before a streaming loop, it
// makes the compiler wait for prologue loads there, instead of inside the loop at their first use, where the
// wait (a count of all loads in flight) would also drain the tile requested for the next step.
template <typename T> __device__ __forceinline__ void settle(const T& v) { asm volatile("" ::"v"(v)); }
// The loads above are invisible to the compiler's own wait counting: wait for all of them before the barrier
// that hands the tile to the readers.
__device__ __forceinline__ void dma_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Two kinds of read, as byte offsets inside a tile that stay in registers across the streaming loop (computed per read they are
// ~100 vector instructions per tile step, more than the softmax arithmetic itself; matrix and vector instructions do not overlap
// on a SIMD, so every one of them is matrix time lost; backward over 8192 tokens, 12 heads of 128, causal: 771 and 761 us with
// dQ's computed per read and kept).  Both are unchanged by adding a multiple of 16 to the row (the swizzle uses row bits 0..3
// only): a second block of 16 rows is the same offset plus 16 rows.
//   frag_k_off   MFMA operand with the head dimension as K: row (row_base + lane%32), dh = 16*ks + 8*(lane/32) + 0..7
//   frag_t_off   MFMA operand with the tile's ROW index as K: column (d_base + lane%32); element e = 4h + j holds row
//                r_base + 8h + 4*(lane/32) + j, which is the order accumulator registers 0..7 hold their rows
template <int DH> __device__ __forceinline__ unsigned frag_k_off(int row_base, int ks, int lane) {
    int row = row_base + (lane & 31);
    int c = 2 * ks + (lane >> 5);
    return (unsigned)(row * (DH * 2) + ((c ^ swz<DH>(row)) << 4));
}
template <int DH> __device__ __forceinline__ unsigned frag_t_off(int d_base, int r_base, int h, int lane) {
    int l16 = lane & 15;
    int d = d_base + (lane & 16) + 4 * (l16 & 3);
    int row = r_base + 8 * h + 4 * (lane >> 5) + (l16 >> 2);
    return (unsigned)(row * (DH * 2) + ((((d >> 3) ^ swz<DH>(row))) << 4) + (d & 7) * 2);
}
typedef __attribute__((address_space(3))) const bf16x8* lds_bf16x8_cptr;
// The reads themselves from a 32-bit LDS address held in a register plus a compile-time byte offset (an immediate).
template <int IMM> __device__ __forceinline__ bf16x8 lds_frag_k(unsigned addr) {
    return *reinterpret_cast<lds_bf16x8_cptr>((uintptr_t)(addr + IMM));
}
template <int IMM> __device__ __forceinline__ bf16x8 lds_frag_t(unsigned addr0, unsigned addr1) {
    s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(uintptr_t)(addr0 + IMM));
    s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(uintptr_t)(addr1 + IMM));
    bf16x4 b0 = __builtin_bit_cast(bf16x4, v0), b1 = __builtin_bit_cast(bf16x4, v1);
    bf16x8 out;
    out[0] = b0[0]; out[1] = b0[1]; out[2] = b0[2]; out[3] = b0[3];
    out[4] = b1[0]; out[5] = b1[1]; out[6] = b1[2]; out[7] = b1[3];
    return out;
}
typedef __attribute__((ext_vector_type(4))) float f32x4;
__device__ __forceinline__ f32x4 lds_f4(unsigned addr) {
    typedef __attribute__((address_space(3))) const f32x4* p_t;
    return *reinterpret_cast<p_t>((uintptr_t)addr);
}
template <typename T> __device__ __forceinline__ void keep_in_register(T& v) { asm volatile("" : "+v"(v)); }
// The same operand straight from global memory (loop-invariant fragments kept in registers).
__device__ __forceinline__ bf16x8 frag_k_global(const bf16_t* base, int64_t ld, int row, int nrows, int dh,
                                                int ks, int lane) {
    bf16x8 z;
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = (bf16_t)0.0f;
    if (row >= nrows || 16 * ks + 8 * (lane >> 5) >= dh) return z;
    return *reinterpret_cast<const bf16x8*>(base + (int64_t)row * ld + 16 * ks + 8 * (lane >> 5));
}
// The sum of the products of two runs of eight elements (float accumulation).  Runs are added to each other in pairs: one after another the
// sums of 64 lost a tenth more to rounding than the row-dot kernel's.
__device__ __forceinline__ float dot8(const bf16x8& x, const bf16x8& y) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    float c = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        bf16x2 u, v;
        u[0] = x[e]; u[1] = x[e + 1];
        v[0] = y[e]; v[1] = y[e + 1];
        c = __builtin_amdgcn_fdot2_f32_bf16(u, v, c, false);
    }
    return c;
}
// The sum of v over each aligned group of eight lanes, in all of them.
__device__ __forceinline__ float sum_of_8_lanes(float v) {
    auto step = [](float x, auto ctrl) { return x + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true)); };
    v = step(v, std::integral_constant<int, 0xB1>{});      // lane ^ 1
    v = step(v, std::integral_constant<int, 0x4E>{});      // lane ^ 2
    return step(v, std::integral_constant<int, 0x141>{});  // 7 - lane: the other four
}
#define MFMA(a, b, c) __builtin_amdgcn_mfma_f32_32x32x16_bf16((a), (b), (c), 0, 0, 0)
__device__ __forceinline__ bf16x8 pack_regs(const f32x16& a, int first) {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (bf16_t)a[first + e];
    return o;
}
// The weights of a second product (probabilities or dS, accumulator order) as matrix operands: terms g[0] + g[1] + ...
// of rows 0..15 (g[.][0]) and 16..31 (g[.][1]).  FLOATW: a float's 24 significant bits are cut into three runs of 8, which
// are bf16 exactly, so the products and their float sums are those of float weights (results that differ from the
// correctly rounded bf16 one at head size 80: 0.05 % of dV, as with float arithmetic; 42 % with rounded weights).  The
// upper halves are taken by truncation: one lane permute per pair, and an infinity stays one.
template <bool FLOATW> constexpr int weight_terms() { return FLOATW ? 3 : 1; }
template <bool FLOATW>
__device__ __forceinline__ void split_terms(f32x16 w, bf16x8 (&g)[weight_terms<FLOATW>()][2]) {
    if constexpr (!FLOATW) {
        g[0][0] = pack_regs(w, 0);
        g[0][1] = pack_regs(w, 8);
    } else {
#pragma unroll
        for (int n = 0; n < 3; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                unsigned u[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    u[e] = __builtin_amdgcn_perm(__float_as_uint(w[8 * h + 2 * e + 1]), __float_as_uint(w[8 * h + 2 * e]), 0x07060302u);
                g[n][h] = __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3]));
                if (n == 2) continue;
#pragma unroll
                for (int e = 8 * h; e < 8 * h + 8; ++e) {
                    const float top = __uint_as_float(__float_as_uint(w[e]) & 0xffff0000u);
                    w[e] = top == w[e] ? 0.0f : w[e] - top;      // not inf - inf
                }
            }
    }
}
// acc += F W for the weight rows 16 h ... of F's columns
template <bool FLOATW>
__device__ __forceinline__ f32x16 mfma_terms(const bf16x8& f, const bf16x8 (&g)[weight_terms<FLOATW>()][2], int h, f32x16 acc) {
#pragma unroll
    for (int n = 0; n < weight_terms<FLOATW>(); ++n) acc = MFMA(f, g[n][h], acc);
    return acc;
}
__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int v = 0; v < 16; ++v) z[v] = 0.0f;
    return z;
}
__device__ __forceinline__ void store4(bf16_t* p, float a, float b, float c, float d) {
    bf16x4 o;
    o[0] = (bf16_t)a; o[1] = (bf16_t)b; o[2] = (bf16_t)c; o[3] = (bf16_t)d;
    *reinterpret_cast<bf16x4*>(p) = o;
}
__device__ __forceinline__ void store_f4(float* p, float a, float b, float c, float d) {
    *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}
// max(v[l], v[l ^ 32]) in every lane by one lane-swap instruction (no trip through the LDS crossbar, whose latency would
// sit in the middle of the softmax chain): swapping the upper half of a with the lower half of b, for a = b = v, leaves
// (v.lo, v.lo) and (v.hi, v.hi).
__device__ __forceinline__ float cross_half_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// z stays 0 while the values are finite, and becomes NaN otherwise.
__device__ __forceinline__ void note4(float& z, const float (&r)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) z = fmaf(r[j], 0.0f, z);
}
__device__ __forceinline__ bool any_nonfinite(float z) { return __any(z != 0.0f); }
// 2^x on the hardware transcendental unit (arguments here are <= ~0; results below 2^-126 flush to 0).
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Log-sum-exp of a row from its reference point (log2) and sum.
template <bool FLOATW> __device__ __forceinline__ float strip_lse(float m, float l) {
    return FLOATW ? fmaf(m, LN2, logf(l)) : (m + log2f(l)) * LN2;
}

}  // namespace tpl
