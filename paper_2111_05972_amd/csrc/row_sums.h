// Sums over the rows of a float matrix [rows, cols] that workgroups have left, in a fixed order: the last step of gradients that belong to columns.
// 32 columns to a workgroup, 32 row lanes that add every 32nd row one after another, eight requested at once, and are joined in lane order, in 64 bits: the sums are near their
// final size here, and 48 additions of 32 bits took gradients of float to three times the distance from 64 bits that one rounding has.  A launch and two
// round trips to memory: 4.0 to 4.7 us for 79 to 512 rows of 160 to 12288 columns, 16 to 64 lanes and 8 to 32 columns no less.
#pragma once
#include <hip/hip_runtime.h>

#include "device_math.h"

namespace tpl {
namespace {

constexpr int RS_COLS = 32, RS_LANES = 32;
// Columns from `split` on go to out1 (split = cols: there is one output).
template <typename T>
__global__ __launch_bounds__(RS_COLS * RS_LANES) void row_sums_kernel(int rows, int64_t cols, int64_t split, const float* __restrict__ part, T* __restrict__ out0,
                                                                      T* __restrict__ out1) {
    __shared__ double red[RS_LANES][RS_COLS + 1];
    const int c = threadIdx.x % RS_COLS, lane = threadIdx.x / RS_COLS;
    const int64_t n = (int64_t)blockIdx.x * RS_COLS + c;
    double s = 0.0;
    if (n < cols) {
        const float* src = part + n;
        int i = lane;
        for (; i + 7 * RS_LANES < rows; i += 8 * RS_LANES) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = src[(int64_t)(i + j * RS_LANES) * cols];
#pragma unroll
            for (int j = 0; j < 8; ++j) s += v[j];
        }
        for (; i < rows; i += RS_LANES) s += src[(int64_t)i * cols];
    }
    red[lane][c] = s;
    __syncthreads();
    if (lane != 0 || n >= cols) return;
    double total = red[0][c];
#pragma unroll
    for (int j = 1; j < RS_LANES; ++j) total += red[j][c];
    (n < split ? out0[n] : out1[n - split]) = from_f32<T>((float)total);
}
template <typename T>
hipError_t row_sums(int64_t rows, int64_t cols, int64_t split, const float* part, void* out0, void* out1, hipStream_t s) {
    hipLaunchKernelGGL(row_sums_kernel<T>, dim3((unsigned)((cols + RS_COLS - 1) / RS_COLS)), dim3(RS_COLS * RS_LANES), 0, s, (int)rows, cols, split, part, (T*)out0, (T*)out1);
    return hipGetLastError();
}

}  // namespace
}  // namespace tpl
