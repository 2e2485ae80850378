// Backward pass of the product's epilogue (see cleave.h): dz, the multiplier's gradient, the bias gradient.
//
// Bound by the HBM's bandwidth (dy, z, mul read once; dz, dmul written once).  A warp takes U columns a lane (8
// where rows are whole 16-byte groups, else 1: any size, stride or alignment) and, with the seven other warps of
// its CTA, the rows of a band; several rows of each operand are asked for before the first is used.  The bias
// gradient stays in registers over the band's rows, the CTA's warps are joined in shared memory, and a band's sums
// are one row of the workspace, added in order by sum_parts_kernel.
#include "ops.cuh"

namespace cleave {

constexpr uint32_t kActWarps = 8;
constexpr uint32_t kActMaxParts = 256;

// rows of partial bias gradients: one per band of rows (bands of 64 rows, longer when that would make too many)
uint32_t act_backward_parts(uint64_t rows, uint32_t cols) {
    (void)cols;
    const uint64_t bands = (rows + 63) / 64;
    return (uint32_t)(bands < kActMaxParts ? bands : kActMaxParts);
}

// U elements of an operand whose type is a launch-time constant (a uniform branch)
template <int U>
__device__ __forceinline__ void load_cells(const void* p, uint32_t type, uint64_t at, float (&x)[U]) {
    if constexpr (U == 1) x[0] = load_as(p, type, at);
    else if (type == CLEAVE_T_F32) unpack8(load_raw8(static_cast<const float*>(p) + at), x);
    else unpack8(load_raw8(static_cast<const __nv_bfloat16*>(p) + at), x);
}
template <int U>
__device__ __forceinline__ void store_cells(void* p, uint32_t type, uint64_t at, const float (&x)[U]) {
    if constexpr (U == 1) store_as(p, type, at, x[0]);
    else if (type == CLEAVE_T_F32) store8(static_cast<float*>(p) + at, x);
    else store8(static_cast<__nv_bfloat16*>(p) + at, x);
}

template <int U, uint32_t ACT>
__global__ void __launch_bounds__(32 * kActWarps) act_backward_kernel(const __grid_constant__ cleave_act_backward_t d, float* __restrict__ ws) {
    __shared__ float s[kActWarps][32 * U];
    constexpr int ROWS = U == 1 ? 4 : 2;                 // rows in flight per warp
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint64_t j = ((uint64_t)blockIdx.x * 32u + lane) * U;
    const uint64_t band = (d.rows + gridDim.y - 1) / gridDim.y, r0 = blockIdx.y * band, r1 = r0 + band < d.rows ? r0 + band : d.rows;
    float sum[U];
#pragma unroll
    for (int i = 0; i < U; ++i) sum[i] = 0.f;
    if (j < d.cols)
        for (uint64_t row = r0 + warp; row < r1; row += kActWarps * ROWS) {
            float dy[ROWS][U], z[ROWS][U], mul[ROWS][U];
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                const uint64_t i = row + k * kActWarps;
                if (i >= r1) break;
                load_cells<U>(d.dy, d.dy_type, i * d.lddy + j, dy[k]);
                if (d.z) load_cells<U>(d.z, d.z_type, i * d.ldz + j, z[k]);
                if (d.mul) load_cells<U>(d.mul, d.mul_type, i * d.ldmul + j, mul[k]);
            }
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                const uint64_t i = row + k * kActWarps;
                if (i >= r1) break;
                float dz[U], dm[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float2 f = act_value_slope(d.z ? z[k][u] : 0.f, ACT);
                    dm[u] = dy[k][u] * f.x;
                    dz[u] = dy[k][u] * f.y;
                    if (d.mul) dz[u] *= mul[k][u];
                    sum[u] += dz[u];
                }
                if (d.dmul) store_cells<U>(d.dmul, d.dmul_type, i * d.lddmul + j, dm);
                if (d.dz) store_cells<U>(d.dz, d.dz_type, i * d.lddz + j, dz);
            }
        }
    if (!d.dbias) return;
#pragma unroll
    for (int u = 0; u < U; ++u) s[warp][u * 32 + lane] = sum[u];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < 32u * U; c += 32 * kActWarps) {         // column c of the CTA: lane c / U, cell c % U
        const uint32_t at = (c % U) * 32u + c / U;
        const uint64_t col = (uint64_t)blockIdx.x * 32u * U + c;
        if (col >= d.cols) continue;
        float t = s[0][at];
#pragma unroll
        for (int w = 1; w < (int)kActWarps; ++w) t += s[w][at];
        ws[(uint64_t)blockIdx.y * d.cols + col] = t;
    }
}

template <int U>
void launch_act(const cleave_act_backward_t& d, float* ws, uint32_t parts, cudaStream_t st) {
    const dim3 grid((d.cols + 32 * U - 1) / (32 * U), parts), block(32 * kActWarps);
    switch (d.act) {
        case CLEAVE_ACT_RELU: act_backward_kernel<U, CLEAVE_ACT_RELU><<<grid, block, 0, st>>>(d, ws); break;
        case CLEAVE_ACT_GELU: act_backward_kernel<U, CLEAVE_ACT_GELU><<<grid, block, 0, st>>>(d, ws); break;
        case CLEAVE_ACT_GELU_TANH: act_backward_kernel<U, CLEAVE_ACT_GELU_TANH><<<grid, block, 0, st>>>(d, ws); break;
        case CLEAVE_ACT_SILU: act_backward_kernel<U, CLEAVE_ACT_SILU><<<grid, block, 0, st>>>(d, ws); break;
        default: act_backward_kernel<U, CLEAVE_ACT_NONE><<<grid, block, 0, st>>>(d, ws); break;
    }
}

cudaError_t launch_act_backward(const cleave_act_backward_t& d, float* ws, cudaStream_t st) {
    if (!d.cols) return cudaSuccess;
    const uint32_t parts = act_backward_parts(d.rows, d.cols);
    const bool wide = d.cols % 8 == 0 && rows_wide(d.dy, d.lddy, d.dy_type) && (!d.z || rows_wide(d.z, d.ldz, d.z_type)) &&
                      (!d.mul || rows_wide(d.mul, d.ldmul, d.mul_type)) && (!d.dz || rows_wide(d.dz, d.lddz, d.dz_type)) &&
                      (!d.dmul || rows_wide(d.dmul, d.lddmul, d.dmul_type));
    if (parts) { if (wide) launch_act<8>(d, ws, parts, st); else launch_act<1>(d, ws, parts, st); }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !d.dbias) return e;
    return launch_sum_parts(ws, parts, d.cols, d.dbias, st);
}

}  // namespace cleave
