// Root-mean-square norm with the residual's addition, its backward pass, and rows in 8 bits (see cleave.h).
#include "ops.cuh"

namespace cleave {

constexpr uint32_t kRowThreads = 256;

// Sum / NaN-keeping maximum over the CTA; every thread receives it.  `buf` holds one value per warp and may be
// reused after the call (it ends with a barrier).
__device__ __forceinline__ float cta_sum(float v, float* buf) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if ((threadIdx.x & 31u) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.f;
    for (uint32_t w = 0; w < blockDim.x / 32; ++w) s += buf[w];
    __syncthreads();
    return s;
}
__device__ __forceinline__ float cta_max_nan(float v, float* buf) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    if ((threadIdx.x & 31u) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = buf[0];
    for (uint32_t w = 1; w < blockDim.x / 32; ++w) s = max_nan(s, buf[w]);
    __syncthreads();
    return s;
}
// scale of a row whose largest magnitude is `top`, and its reciprocal (0 for a row of zeros or of values so small
// that the reciprocal would overflow)
__device__ __forceinline__ float2 row_scale(float top) {
    const float s = top * (1.f / kE4M3Max);
    return make_float2(s, s < 0x1p-120f ? 0.f : 1.f / s);
}

// One CTA per row, any types, sizes and alignments: the row is read again in each pass (it stays in L1 / L2).
template <bool NORM>
__global__ void __launch_bounds__(kRowThreads) row_any_kernel(const __grid_constant__ cleave_rmsnorm_t d) {
    __shared__ float buf[32];
    const uint64_t row = blockIdx.x;
    const uint64_t ox = row * d.ldx, orr = row * d.ldr, oh = row * d.ldh, oy = row * d.ldy;
    // (h may be r's buffer: it is written in the last pass only, each element by the thread that has just read it)
    auto sum_at = [&](uint32_t j) { return load_as(d.x, d.x_type, ox + j) + (d.r ? load_as(d.r, d.r_type, orr + j) : 0.f); };
    float rstd = 1.f;
    if (NORM) {
        float ss = 0.f;
        for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) { const float h = sum_at(j); ss = fmaf(h, h, ss); }
        rstd = rsqrtf(cta_sum(ss, buf) / (float)d.cols + d.eps);
        if (d.rstd && threadIdx.x == 0) d.rstd[row] = rstd;
    }
    float inv = 1.f;
    if (d.y_type == CLEAVE_T_E4M3) {
        float top = 0.f;
        for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) {
            const float y = sum_at(j) * rstd * (d.w ? load_as(d.w, d.w_type, j) : 1.f);
            top = max_nan(top, fabsf(y));
        }
        const float2 s = row_scale(cta_max_nan(top, buf));
        inv = s.y;
        if (threadIdx.x == 0) d.scale[row] = s.x;
    }
    for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) {
        const float h = sum_at(j);
        if (NORM && d.h) store_as(d.h, d.r_type, oh + j, h);
        const float y = h * rstd * (d.w ? load_as(d.w, d.w_type, j) : 1.f);
        if (d.y_type == CLEAVE_T_E4M3) static_cast<uint8_t*>(d.y)[oy + j] = e4m3_nearest(y * inv);
        else store_as(d.y, d.y_type, oy + j, y);
    }
}

cudaError_t launch_rmsnorm(const cleave_rmsnorm_t& d, bool norm, cudaStream_t st) {
    if (!d.rows || !d.cols) return cudaSuccess;
    if (norm) row_any_kernel<true><<<(unsigned)d.rows, kRowThreads, 0, st>>>(d);
    else      row_any_kernel<false><<<(unsigned)d.rows, kRowThreads, 0, st>>>(d);
    return cudaGetLastError();
}

// ---- backward ----------------------------------------------------------------------------------------
// A CTA takes the rows part, part + parts, ...; its share of dw goes to row `part` of the workspace (fp32
// [parts x cols]; each element belongs to one thread), and sum_parts_kernel adds the parts in order.
constexpr uint32_t kMaxParts = 2 * 148;
uint32_t rmsnorm_backward_parts(uint64_t rows, uint32_t cols) {
    (void)cols;
    return (uint32_t)(rows < kMaxParts ? rows : kMaxParts);
}

__global__ void __launch_bounds__(kRowThreads) rmsnorm_backward_any_kernel(const __grid_constant__ cleave_rmsnorm_backward_t d, float* __restrict__ ws) {
    __shared__ float buf[32];
    float* dw = ws + (uint64_t)blockIdx.x * d.cols;
    if (d.dw) for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) dw[j] = 0.f;
    for (uint64_t row = blockIdx.x; row < d.rows; row += gridDim.x) {
        const uint64_t ody = row * d.lddy, oh = row * d.ldh, ors = row * d.lddres, odx = row * d.lddx;
        const float rstd = d.rstd[row];
        float dot = 0.f;
        for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) {
            const float dy = load_as(d.dy, d.dy_type, ody + j), xh = load_as(d.h, d.h_type, oh + j) * rstd;
            dot = fmaf(dy * (d.w ? load_as(d.w, d.w_type, j) : 1.f), xh, dot);
        }
        const float mean = cta_sum(dot, buf) / (float)d.cols;
        for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) {
            const float dy = load_as(d.dy, d.dy_type, ody + j), xh = load_as(d.h, d.h_type, oh + j) * rstd;
            float dx = rstd * (dy * (d.w ? load_as(d.w, d.w_type, j) : 1.f) - xh * mean);
            if (d.dres) dx += load_as(d.dres, d.h_type, ors + j);
            store_as(d.dx, d.h_type, odx + j, dx);
            if (d.dw) dw[j] = fmaf(dy, xh, dw[j]);
        }
    }
}

// out[j] = sum over the parts of ws[part][j], in a fixed order.  32 columns per CTA; warp w adds the parts
// w, w + 8, ... and the eight sums are added in warp order.
__global__ void __launch_bounds__(256) sum_parts_kernel(const float* __restrict__ ws, uint32_t parts, uint32_t cols, float* __restrict__ out) {
    __shared__ float s[8][32];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, j = blockIdx.x * 32u + lane;
    float v = 0.f;
    if (j < cols) for (uint32_t p = warp; p < parts; p += 8) v += ws[(uint64_t)p * cols + j];
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && j < cols) {
#pragma unroll
        for (int w = 1; w < 8; ++w) v += s[w][lane];
        out[j] = v;
    }
}
cudaError_t launch_sum_parts(const float* ws, uint32_t parts, uint32_t cols, float* out, cudaStream_t st) {
    sum_parts_kernel<<<(cols + 31) / 32, 256, 0, st>>>(ws, parts, cols, out);
    return cudaGetLastError();
}

cudaError_t launch_rmsnorm_backward(const cleave_rmsnorm_backward_t& d, float* ws, cudaStream_t st) {
    if (!d.cols) return cudaSuccess;
    const uint32_t parts = rmsnorm_backward_parts(d.rows, d.cols);
    if (parts) rmsnorm_backward_any_kernel<<<parts, kRowThreads, 0, st>>>(d, ws);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !d.dw) return e;
    return launch_sum_parts(ws, parts, d.cols, d.dw, st);
}

}  // namespace cleave
