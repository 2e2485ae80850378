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

// Rows of partial bias gradients: one per band of rows.  As many bands as give each SM three CTAs of 256 columns
// (the wide form's), so that a CTA's warps stream over many rows and the sums are joined once.
uint32_t act_backward_parts(uint64_t rows, uint32_t cols) {
    const uint64_t tiles = (cols + 255) / 256, most = (rows + 2 * kActWarps - 1) / (2 * kActWarps);
    const uint64_t bands = tiles < 444 ? 444 / tiles : 1;
    return (uint32_t)(bands < most ? bands : most);
}

// U elements of an operand: raw (what stays in flight) and as fp32.  The wide form is typed; U = 1 takes the type
// from the launch (a uniform branch).
template <int U, typename T> struct Cells { Raw8<T> raw; };
template <typename T> struct Cells<1, T> { float raw; };
template <int U, typename T>
__device__ __forceinline__ void load_cells(Cells<U, T>& c, const void* p, uint32_t type, uint64_t at) {
    if constexpr (U == 1) c.raw = load_as(p, type, at);
    else c.raw = load_raw8(static_cast<const T*>(p) + at);
}
template <int U, typename T>
__device__ __forceinline__ void unpack_cells(const Cells<U, T>& c, float (&x)[U]) {
    if constexpr (U == 1) x[0] = c.raw;
    else unpack8(c.raw, x);
}
template <int U, typename T>
__device__ __forceinline__ void store_cells(void* p, uint32_t type, uint64_t at, const float (&x)[U]) {
    if constexpr (U == 1) store_as(p, type, at, x[0]);
    else store8(static_cast<T*>(p) + at, x);
}

// D: type of dy; T: type of z, mul, dz and dmul (wide form: one type).  Rows in flight per warp and operand: two
// batches of ROWS.
template <int U, typename D, typename T, uint32_t ACT, bool MUL>
__global__ void __launch_bounds__(32 * kActWarps, MUL ? 2 : 3) act_backward_kernel(const __grid_constant__ cleave_act_backward_t d, float* __restrict__ ws) {
    __shared__ float s[kActWarps][32 * U];
    constexpr int ROWS = U > 1 && sizeof(T) == 4 ? 1 : 2;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint64_t j = ((uint64_t)blockIdx.x * 32u + lane) * U;
    const uint64_t band = (d.rows + gridDim.y - 1) / gridDim.y, r0 = blockIdx.y * band, r1 = r0 + band < d.rows ? r0 + band : d.rows;
    const bool has_z = ACT != CLEAVE_ACT_NONE || d.z;
    float sum[U];
#pragma unroll
    for (int i = 0; i < U; ++i) sum[i] = 0.f;
    // two batches of ROWS rows: the next one is asked for before the first is used
    Cells<U, D> cdy[2][ROWS];
    Cells<U, T> cz[2][ROWS], cm[2][ROWS];
    auto fetch = [&](uint64_t row, int b) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const uint64_t i = row + k * kActWarps;
            if (i >= r1) break;
            load_cells(cdy[b][k], d.dy, d.dy_type, i * d.lddy + j);
            if (has_z) load_cells(cz[b][k], d.z, d.z_type, i * d.ldz + j);
            if constexpr (MUL) load_cells(cm[b][k], d.mul, d.mul_type, i * d.ldmul + j);
        }
    };
    auto use = [&](uint64_t row, int b) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const uint64_t i = row + k * kActWarps;
            if (i >= r1) break;
            float dy[U], z[U], mul[U], dz[U], dm[U];
            unpack_cells(cdy[b][k], dy);
            if (has_z) unpack_cells(cz[b][k], z);
            if constexpr (MUL) unpack_cells(cm[b][k], mul);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float2 f = act_value_slope(has_z ? z[u] : 0.f, ACT);
                // (rounded one by one: the sums' bits do not depend on which outputs are wanted)
                dm[u] = __fmul_rn(dy[u], f.x);
                dz[u] = __fmul_rn(dy[u], f.y);
                if constexpr (MUL) dz[u] = __fmul_rn(dz[u], mul[u]);
                sum[u] = __fadd_rn(sum[u], dz[u]);
            }
            if (d.dmul) store_cells<U, T>(d.dmul, d.dmul_type, i * d.lddmul + j, dm);
            if (d.dz) store_cells<U, T>(d.dz, d.dz_type, i * d.lddz + j, dz);
        }
    };
    constexpr uint32_t kStep = kActWarps * ROWS;
    if (j < d.cols) {
        fetch(r0 + warp, 0);
        for (uint64_t row = r0 + warp; row < r1; row += 2 * kStep) {
            fetch(row + kStep, 1);
            use(row, 0);
            fetch(row + 2 * kStep, 0);
            use(row + kStep, 1);
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

template <int U, typename D, typename T, bool MUL>
void launch_act(const cleave_act_backward_t& d, float* ws, uint32_t parts, cudaStream_t st) {
    const dim3 grid((d.cols + 32 * U - 1) / (32 * U), parts), block(32 * kActWarps);
    switch (d.act) {
        case CLEAVE_ACT_RELU: act_backward_kernel<U, D, T, CLEAVE_ACT_RELU, MUL><<<grid, block, 0, st>>>(d, ws); break;
        case CLEAVE_ACT_GELU: act_backward_kernel<U, D, T, CLEAVE_ACT_GELU, MUL><<<grid, block, 0, st>>>(d, ws); break;
        case CLEAVE_ACT_GELU_TANH: act_backward_kernel<U, D, T, CLEAVE_ACT_GELU_TANH, MUL><<<grid, block, 0, st>>>(d, ws); break;
        case CLEAVE_ACT_SILU: act_backward_kernel<U, D, T, CLEAVE_ACT_SILU, MUL><<<grid, block, 0, st>>>(d, ws); break;
        default: act_backward_kernel<U, D, T, CLEAVE_ACT_NONE, MUL><<<grid, block, 0, st>>>(d, ws); break;
    }
}
template <int U, typename D, typename T>
void launch_act(const cleave_act_backward_t& d, float* ws, uint32_t parts, cudaStream_t st) {
    if (d.mul) launch_act<U, D, T, true>(d, ws, parts, st);
    else launch_act<U, D, T, false>(d, ws, parts, st);
}

cudaError_t launch_act_backward(const cleave_act_backward_t& d, float* ws, cudaStream_t st) {
    if (!d.cols) return cudaSuccess;
    const uint32_t parts = act_backward_parts(d.rows, d.cols);
    // the wide form: whole aligned groups of 8 columns, and one type for z, mul, dz and dmul
    uint32_t type = d.z ? d.z_type : (d.dz ? d.dz_type : d.dy_type);
    auto fits = [&](const void* p, uint32_t t, uint64_t ld) { return !p || (t == type && rows_wide(p, ld, t)); };
    const bool wide = d.cols % 8 == 0 && rows_wide(d.dy, d.lddy, d.dy_type) && fits(d.z, d.z_type, d.ldz) && fits(d.mul, d.mul_type, d.ldmul) &&
                      fits(d.dz, d.dz_type, d.lddz) && fits(d.dmul, d.dmul_type, d.lddmul);
    if (!parts) { }
    else if (!wide) launch_act<1, float, float>(d, ws, parts, st);
    else if (d.dy_type == CLEAVE_T_F32) { if (type == CLEAVE_T_F32) launch_act<8, float, float>(d, ws, parts, st); else launch_act<8, float, __nv_bfloat16>(d, ws, parts, st); }
    else { if (type == CLEAVE_T_F32) launch_act<8, __nv_bfloat16, float>(d, ws, parts, st); else launch_act<8, __nv_bfloat16, __nv_bfloat16>(d, ws, parts, st); }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !d.dbias) return e;
    return launch_sum_parts(ws, parts, d.cols, d.dbias, st);
}

}  // namespace cleave
