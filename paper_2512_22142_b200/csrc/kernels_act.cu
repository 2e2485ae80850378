// Backward pass of the product's epilogue (see cleave.h): dz, the multiplier's gradient, the bias gradient.
#include "ops.cuh"

namespace cleave {

constexpr uint32_t kActCols = 32, kActWarps = 8;
constexpr uint32_t kActMaxParts = 128;

// rows of partial bias gradients: one per band of rows
uint32_t act_backward_parts(uint64_t rows, uint32_t cols) {
    (void)cols;
    const uint64_t bands = (rows + 63) / 64;
    return (uint32_t)(bands < kActMaxParts ? bands : kActMaxParts);
}

// CTA (x, y): 32 columns, a band of rows; lane = column, warp w takes the rows w, w + 8, ... of the band.
__global__ void __launch_bounds__(32 * kActWarps) act_backward_any_kernel(const __grid_constant__ cleave_act_backward_t d, float* __restrict__ ws) {
    __shared__ float s[kActWarps][32];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint64_t j = (uint64_t)blockIdx.x * kActCols + lane;
    const uint64_t band = (d.rows + gridDim.y - 1) / gridDim.y, r0 = blockIdx.y * band, r1 = r0 + band < d.rows ? r0 + band : d.rows;
    float sum = 0.f;
    if (j < d.cols)
        for (uint64_t i = r0 + warp; i < r1; i += kActWarps) {
            const float dy = load_as(d.dy, d.dy_type, i * d.lddy + j);
            const float2 f = act_value_slope(d.z ? load_as(d.z, d.z_type, i * d.ldz + j) : 0.f, d.act);
            const float mul = d.mul ? load_as(d.mul, d.mul_type, i * d.ldmul + j) : 1.f;
            const float dz = dy * f.y * mul;
            if (d.dmul) store_as(d.dmul, d.dmul_type, i * d.lddmul + j, dy * f.x);
            if (d.dz) store_as(d.dz, d.dz_type, i * d.lddz + j, dz);
            sum += dz;
        }
    if (!d.dbias) return;
    s[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && j < d.cols) {
#pragma unroll
        for (int w = 1; w < (int)kActWarps; ++w) sum += s[w][lane];
        ws[(uint64_t)blockIdx.y * d.cols + j] = sum;
    }
}

cudaError_t launch_act_backward(const cleave_act_backward_t& d, float* ws, cudaStream_t st) {
    if (!d.cols) return cudaSuccess;
    const uint32_t parts = act_backward_parts(d.rows, d.cols);
    if (parts) act_backward_any_kernel<<<dim3((d.cols + kActCols - 1) / kActCols, parts), 32 * kActWarps, 0, st>>>(d, ws);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !d.dbias) return e;
    return launch_sum_parts(ws, parts, d.cols, d.dbias, st);
}

}  // namespace cleave
