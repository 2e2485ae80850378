// Layer norm with the residual's addition, and its backward pass (see cleave.h).
#include <algorithm>

#include "rows.cuh"
#include "tokens.cuh"

namespace cleave {

// ---- forward, any shape ------------------------------------------------------------------------------
__global__ void __launch_bounds__(kRowThreads) layernorm_any_kernel(const __grid_constant__ cleave_layernorm_t d) {
    __shared__ float buf[32];
    begin_chained();
    const uint64_t row = blockIdx.x;
    const uint64_t ox = row * d.ldx, orr = row * d.ldr, oh = row * d.ldh, oy = row * d.ldy;
    // (h may be r's buffer: it is written in the last pass only, each element by the thread that has just read it)
    auto sum_at = [&](uint32_t j) { return load_as(d.x, d.x_type, ox + j) + (d.r ? load_as(d.r, d.r_type, orr + j) : 0.f); };
    auto result = [&](float c, uint32_t j) { return fmaf(c, d.w ? load_as(d.w, d.w_type, j) : 1.f, d.b ? load_as(d.b, d.b_type, j) : 0.f); };
    float s = 0.f;
    for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) s += sum_at(j);
    const float mean = cta_sum(s, buf) / (float)d.cols;
    float ss = 0.f;
    for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) { const float c = sum_at(j) - mean; ss = fmaf(c, c, ss); }
    const float rstd = rsqrtf(cta_sum(ss, buf) / (float)d.cols + d.eps);
    if (threadIdx.x == 0) {
        if (d.mean) d.mean[row] = mean;
        if (d.rstd) d.rstd[row] = rstd;
    }
    float inv = 1.f;
    if (d.y_type == CLEAVE_T_E4M3) {
        float top = 0.f;
        for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) top = max_nan(top, fabsf(result((sum_at(j) - mean) * rstd, j)));
        const float2 sc = row_scale(cta_max_nan(top, buf));
        inv = sc.y;
        if (threadIdx.x == 0) d.scale[row] = sc.x;
    }
    for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) {
        const float h = sum_at(j), y = result((h - mean) * rstd, j);
        if (d.h) store_as(d.h, d.r_type, oh + j, h);
        if (d.y_type == CLEAVE_T_E4M3) static_cast<uint8_t*>(d.y)[oy + j] = e4m3_nearest(y * inv);
        else store_as(d.y, d.y_type, oy + j, y);
    }
}
cudaError_t launch_layernorm(const cleave_layernorm_t& d, int, cudaStream_t st) {
    return launch_chained(layernorm_any_kernel, (unsigned)d.rows, kRowThreads, 0, st, d);
}

// ---- backward ----------------------------------------------------------------------------------------
// A CTA takes the rows part, part + parts, ...; its shares of dw and db go to row `part` of the workspace (fp32
// [parts x 2 cols], dw's columns first), and sum_parts_kernel adds the parts in order.
uint32_t layernorm_backward_parts(uint64_t rows, uint32_t) { return (uint32_t)std::min<uint64_t>(rows, 2 * kPartSms); }

__global__ void __launch_bounds__(kRowThreads) layernorm_backward_any_kernel(const __grid_constant__ cleave_layernorm_backward_t d, float* __restrict__ ws) {
    __shared__ float buf[32];
    begin_chained();
    const bool sums = d.dw || d.db;
    float* dw = ws + (uint64_t)blockIdx.x * 2 * d.cols;
    float* db = dw + d.cols;
    if (sums) for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) dw[j] = db[j] = 0.f;
    for (uint64_t row = blockIdx.x; row < d.rows; row += gridDim.x) {
        const uint64_t ody = row * d.lddy, oh = row * d.ldh, ors = row * d.lddres, odx = row * d.lddx;
        const float rstd = d.rstd[row], mean = d.mean[row];
        auto xh_at = [&](uint32_t j) { return (load_as(d.h, d.h_type, oh + j) - mean) * rstd; };
        float dot = 0.f, sum = 0.f;
        for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) {
            const float q = load_as(d.dy, d.dy_type, ody + j) * (d.w ? load_as(d.w, d.w_type, j) : 1.f);
            sum += q;
            dot = fmaf(q, xh_at(j), dot);
        }
        const float along = cta_sum(dot, buf) / (float)d.cols, shift = cta_sum(sum, buf) / (float)d.cols;
        for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) {
            const float dy = load_as(d.dy, d.dy_type, ody + j), xh = xh_at(j);
            float dx = rstd * (dy * (d.w ? load_as(d.w, d.w_type, j) : 1.f) - shift - xh * along);
            if (d.dres) dx += load_as(d.dres, d.h_type, ors + j);
            store_as(d.dx, d.h_type, odx + j, dx);
            if (sums) { dw[j] = fmaf(dy, xh, dw[j]); db[j] += dy; }
        }
    }
}
// out[j] = sum over the parts of ws[part][j], 0 <= j < cols for dw and behind them for db, each in a fixed order: 32 columns
// per CTA; warp w adds the parts w, w + 32, ... and the 32 sums are added by a shuffle tree.
__global__ void __launch_bounds__(1024) layernorm_sum_parts_kernel(const float* ws, uint32_t parts, uint32_t cols, float* dw, float* db) {
    __shared__ float s[32][33];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, j = blockIdx.x * 32u + lane;
    float* out = blockIdx.y ? db : dw;
    wait_for_primary();
    if (!out) return;
    float v = 0.f;
    if (j < cols) {
#pragma unroll 8
        for (uint32_t p = warp; p < parts; p += 32) v += __ldcs(ws + ((uint64_t)p * 2 + blockIdx.y) * cols + j);
    }
    s[warp][lane] = v;
    __syncthreads();
    v = warp_sum(s[lane][warp]);
    if (lane == 0 && blockIdx.x * 32u + warp < cols) out[blockIdx.x * 32u + warp] = v;
}

cudaError_t launch_layernorm_backward(const cleave_layernorm_backward_t& d, float* ws, cudaStream_t st) {
    const uint32_t parts = layernorm_backward_parts(d.rows, d.cols);
    cudaError_t e = cudaSuccess;
    if (parts) e = launch_chained(layernorm_backward_any_kernel, parts, kRowThreads, 0, st, d, ws);
    if (e != cudaSuccess || (!d.dw && !d.db)) return e;
    return launch_chained(layernorm_sum_parts_kernel, dim3((d.cols + 31) / 32, 2), 1024, 0, st, ws, parts, d.cols, d.dw, d.db);
}

}  // namespace cleave
