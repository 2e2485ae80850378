// Backward pass of the product's epilogue (see cleave.h): dz, the multiplier's gradient, the bias gradient.
//
// Bound by the HBM's bandwidth (dy, z, mul read once; dz, dmul written once).  A warp takes 8 columns a lane (where
// rows are whole 16-byte groups, else one) and, with the seven other warps of its CTA, the rows of a band.  In the
// wide form the operands' next rows are on their way to shared memory while a row is used -- each thread copies and
// reads its own groups only, so there is no barrier, and the bytes in flight do not cost registers.  The bias
// gradient stays in registers over the band's rows, the CTA's warps are joined in shared memory, and a band's sums
// are one row of the workspace, added in order by sum_parts_kernel.  Few rows (join_rows) make at most eight bands, a
// cluster, whose sums are added in order through distributed shared memory: one launch.
// Measured: 8192 x 3072 with GELU and the bias gradient 28 us (5.4 TB/s; the gate's arithmetic issues in 75 % of the
// cycles), 8192 x 11008 with SwiGLU's two gradients 153 us (5.9 TB/s of 6.5).
#include <algorithm>

#include "ops.cuh"
#include "ptx.cuh"

namespace cleave {

constexpr uint32_t kActWarps = 8;
constexpr uint32_t kJoinBands = 8;
// Rows up to which the bands are one cluster.  A call is a launch shorter (plain column sums of 656 x 237 5.7 against 7.5 us,
// 1024 x 3072 6.7 against 7.5); beyond, eight bands are too few CTAs (2048 x 3072: 10.5 against 8.2), sooner so where an
// activation is computed (kernels alone, with GELU: 256 x 768 3.8 against 3.7, 512 x 768 5.0 against 3.8).
inline uint64_t join_rows(uint32_t act) { return act == CLEAVE_ACT_NONE ? 1024 : 256; }

// Rows of partial bias gradients: one per band of rows.  As many bands as give each SM three CTAs of 256 columns
// (the wide form's), so that a CTA's warps stream over many rows and the sums are joined once.
uint32_t act_backward_parts(uint64_t rows, uint32_t cols) {
    const uint64_t tiles = (cols + 255) / 256, most = (rows + 2 * kActWarps - 1) / (2 * kActWarps);
    const uint64_t bands = tiles < 3 * kPartSms ? 3 * kPartSms / tiles : 1;
    return (uint32_t)(bands < most ? bands : most);
}

// Column sums of a CTA's warps, joined in warp order into the band's row of `out`; `joined`: the bands of these columns
// are one cluster, and `out` receives their sum in band order.
template <int U>
__device__ __forceinline__ void join_sums(const float (&sum)[U], float (*s)[32 * U], float* __restrict__ out, uint64_t cols, bool joined) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
#pragma unroll
    for (int u = 0; u < U; ++u) s[warp][u * 32 + lane] = sum[u];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < 32u * U; c += 32 * kActWarps) {         // column c of the CTA: lane c / U, cell c % U
        const uint32_t at = (c % U) * 32u + c / U;
        const uint64_t col = (uint64_t)blockIdx.x * 32u * U + c;
        if (col >= cols) continue;
        float t = s[0][at];
#pragma unroll
        for (int w = 1; w < (int)kActWarps; ++w) t += s[w][at];
        if (joined) s[0][at] = t;
        else out[(uint64_t)blockIdx.y * cols + col] = t;
    }
    if (!joined) return;
    cluster_arrive_wait();
    const uint32_t first = (uint32_t)__cvta_generic_to_shared(&s[0][0]);
    for (uint32_t c = blockIdx.y + gridDim.y * threadIdx.x; c < 32u * U; c += gridDim.y * 32 * kActWarps) {        // (rank in the cluster: blockIdx.y)
        const uint32_t at = first + ((c % U) * 32u + c / U) * 4u;
        const uint64_t col = (uint64_t)blockIdx.x * 32u * U + c;
        if (col >= cols) continue;
        float x[kJoinBands], t = 0.f;
#pragma unroll
        for (uint32_t b = 0; b < kJoinBands; ++b) x[b] = b < gridDim.y ? ld_dsmem(mapa_shared(at, b)) : 0.f;
#pragma unroll
        for (uint32_t b = 0; b < kJoinBands; ++b) if (b < gridDim.y) t += x[b];
        out[col] = t;
    }
    cluster_arrive_wait();                                  // no CTA leaves while another reads its sums
}
// dz and dmul of one element (rounded one by one: the sums' bits do not depend on which outputs are wanted)
template <uint32_t ACT, bool MUL>
__device__ __forceinline__ void act_cell(float dy, float z, float mul, float& dz, float& dm, float& sum) {
    const float2 f = act_value_slope(z, ACT);
    dm = __fmul_rn(dy, f.x);
    dz = __fmul_rn(dy, f.y);
    if constexpr (MUL) dz = __fmul_rn(dz, mul);
    sum = __fadd_rn(sum, dz);
}
struct Band { uint32_t r0, r1; };                     // (at most 2^31 - 1 rows)
__device__ __forceinline__ Band this_band(uint64_t rows) {
    const uint32_t n = (uint32_t)rows, band = (n + gridDim.y - 1) / gridDim.y, r0 = min(blockIdx.y * band, n);
    return Band{r0, min(r0 + band, n)};
}

// Any size, stride and alignment: a lane's column, four rows asked for at a time.
template <uint32_t ACT, bool MUL>
__global__ void __launch_bounds__(32 * kActWarps) act_backward_any_kernel(const __grid_constant__ cleave_act_backward_t d, float* __restrict__ sums, uint32_t joined) {
    __shared__ float s[kActWarps][32];
    begin_chained();
    constexpr int ROWS = 4;
    const uint64_t j = (uint64_t)blockIdx.x * 32u + (threadIdx.x & 31u);
    const Band b = this_band(d.rows);
    const bool has_z = ACT != CLEAVE_ACT_NONE || d.z;
    float sum[1] = {0.f};
    if (j < d.cols)
        for (uint32_t row = b.r0 + (threadIdx.x >> 5); row < b.r1; row += kActWarps * ROWS) {
            float dy[ROWS], z[ROWS], mul[ROWS];
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                const uint64_t i = row + k * kActWarps;
                if (i >= b.r1) break;
                dy[k] = load_as(d.dy, d.dy_type, i * d.lddy + j);
                z[k] = has_z ? load_as(d.z, d.z_type, i * d.ldz + j) : 0.f;
                mul[k] = MUL ? load_as(d.mul, d.mul_type, i * d.ldmul + j) : 1.f;
            }
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                const uint64_t i = row + k * kActWarps;
                if (i >= b.r1) break;
                float dz, dm;
                act_cell<ACT, MUL>(dy[k], z[k], mul[k], dz, dm, sum[0]);
                if (d.dmul) store_as(d.dmul, d.dmul_type, i * d.lddmul + j, dm);
                if (d.dz) store_as(d.dz, d.dz_type, i * d.lddz + j, dz);
            }
        }
    if (d.dbias) join_sums<1>(sum, s, sums, d.cols, joined != 0);
}

// Rows of whole 16-byte groups: a lane's 8 columns; STAGES rows of each operand on their way to shared memory.
// D: type of dy; T: the one type of z, mul, dz and dmul.
template <typename D, typename T, uint32_t ACT, bool MUL, int STAGES>
__global__ void __launch_bounds__(32 * kActWarps, 3) act_backward_wide_kernel(const __grid_constant__ cleave_act_backward_t d, float* __restrict__ sums, uint32_t joined) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float s[kActWarps][32 * 8];
    begin_chained();
    constexpr uint32_t BD = sizeof(D) * 8, BT = sizeof(T) * 8, NT = MUL ? 2 : 1, STAGE = 32 * (BD + NT * BT);
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint64_t j = ((uint64_t)blockIdx.x * 32u + lane) * 8u;
    const Band b = this_band(d.rows);
    const bool has_z = ACT != CLEAVE_ACT_NONE || d.z;
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    if (j < d.cols) {
        const uint32_t first = b.r0 + warp;
        const uint8_t* pd = reinterpret_cast<const uint8_t*>(static_cast<const D*>(d.dy) + first * d.lddy + j);
        const uint8_t* pz = has_z ? reinterpret_cast<const uint8_t*>(static_cast<const T*>(d.z) + first * d.ldz + j) : nullptr;
        const uint8_t* pm = MUL ? reinterpret_cast<const uint8_t*>(static_cast<const T*>(d.mul) + first * d.ldmul + j) : nullptr;
        T* odz = d.dz ? static_cast<T*>(d.dz) + first * d.lddz + j : nullptr;
        T* odm = d.dmul ? static_cast<T*>(d.dmul) + first * d.lddmul + j : nullptr;
        uint8_t* mine = ring + warp * (STAGES * STAGE);
        const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
        uint32_t ahead = first;
        auto fetch = [&](uint32_t at) {
            if (ahead < b.r1) {
#pragma unroll
                for (uint32_t x = 0; x < BD; x += 16) cp_async<16>(mine_at + at + lane * BD + x, pd + x);
#pragma unroll
                for (uint32_t x = 0; x < BT; x += 16) {
                    if (has_z) cp_async<16>(mine_at + at + 32 * BD + lane * BT + x, pz + x);
                    if constexpr (MUL) cp_async<16>(mine_at + at + 32 * (BD + BT) + lane * BT + x, pm + x);
                }
                ahead += kActWarps;
                pd += kActWarps * sizeof(D) * d.lddy;
                if (has_z) pz += kActWarps * sizeof(T) * d.ldz;
                if constexpr (MUL) pm += kActWarps * sizeof(T) * d.ldmul;
            }
            cp_async_commit();
        };
#pragma unroll
        for (int k = 0; k < STAGES; ++k) fetch(k * STAGE);
        for (uint32_t row = first; row < b.r1;) {
#pragma unroll
            for (int k = 0; k < STAGES; ++k, row += kActWarps) {      // once round the ring: stages at constant places
                if (row >= b.r1) break;
                const uint8_t* stage = mine + k * STAGE;
                cp_async_wait<STAGES - 1>();
                float dy[8], z[8], mul[8], dz[8], dm[8];
                unpack8(*reinterpret_cast<const Raw8<D>*>(stage + lane * BD), dy);
                if (has_z) unpack8(*reinterpret_cast<const Raw8<T>*>(stage + 32 * BD + lane * BT), z);
                if constexpr (MUL) unpack8(*reinterpret_cast<const Raw8<T>*>(stage + 32 * (BD + BT) + lane * BT), mul);
#pragma unroll
                for (int u = 0; u < 8; ++u) act_cell<ACT, MUL>(dy[u], has_z ? z[u] : 0.f, MUL ? mul[u] : 1.f, dz[u], dm[u], sum[u]);
                fetch(k * STAGE);                                    // the stage's values have been used
                if (odm) { store8(odm, dm); odm += kActWarps * d.lddmul; }
                if (odz) { store8(odz, dz); odz += kActWarps * d.lddz; }
            }
        }
    }
    if (d.dbias) join_sums<8>(sum, s, sums, d.cols, joined != 0);
}

struct Sums { float* out; uint32_t bands, joined; };       // where the bands' sums go; joined: the bands are one cluster
template <typename D, typename T, uint32_t ACT, bool MUL>
cudaError_t launch_act_wide(const cleave_act_backward_t& d, const Sums& b, cudaStream_t st) {
    // 32 to 60 KB a CTA: three or four CTAs an SM
    constexpr uint32_t stage = 32 * (sizeof(D) * 8 + (MUL ? 2 : 1) * sizeof(T) * 8);
    constexpr int STAGES = stage >= 2560 ? 3 : 4;
    auto kernel = act_backward_wide_kernel<D, T, ACT, MUL, STAGES>;
    constexpr uint32_t smem = kActWarps * STAGES * stage;
    static SmemLimit limit;
    const cudaError_t e = limit.raise(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return e;
    return launch_chained_clusters(kernel, dim3(1, b.joined ? b.bands : 1), dim3((d.cols + 255) / 256, b.bands), 32 * kActWarps, smem, st, d, b.out, b.joined);
}
template <uint32_t ACT, bool MUL>
cudaError_t launch_act(const cleave_act_backward_t& d, const Sums& b, bool wide, uint32_t type, cudaStream_t st) {
    if (!wide)
        return launch_chained_clusters(act_backward_any_kernel<ACT, MUL>, dim3(1, b.joined ? b.bands : 1), dim3((d.cols + 31) / 32, b.bands), 32 * kActWarps, 0, st, d,
                                       b.out, b.joined);
    if (d.dy_type == CLEAVE_T_F32)
        return type == CLEAVE_T_F32 ? launch_act_wide<float, float, ACT, MUL>(d, b, st) : launch_act_wide<float, __nv_bfloat16, ACT, MUL>(d, b, st);
    return type == CLEAVE_T_F32 ? launch_act_wide<__nv_bfloat16, float, ACT, MUL>(d, b, st) : launch_act_wide<__nv_bfloat16, __nv_bfloat16, ACT, MUL>(d, b, st);
}
template <bool MUL>
cudaError_t launch_act(const cleave_act_backward_t& d, const Sums& b, bool wide, uint32_t type, cudaStream_t st) {
    switch (d.act) {
        case CLEAVE_ACT_RELU: return launch_act<CLEAVE_ACT_RELU, MUL>(d, b, wide, type, st);
        case CLEAVE_ACT_GELU: return launch_act<CLEAVE_ACT_GELU, MUL>(d, b, wide, type, st);
        case CLEAVE_ACT_GELU_TANH: return launch_act<CLEAVE_ACT_GELU_TANH, MUL>(d, b, wide, type, st);
        case CLEAVE_ACT_SILU: return launch_act<CLEAVE_ACT_SILU, MUL>(d, b, wide, type, st);
        default: return launch_act<CLEAVE_ACT_NONE, MUL>(d, b, wide, type, st);
    }
}

cudaError_t launch_act_backward(const cleave_act_backward_t& d, float* ws, cudaStream_t st) {
    if (!d.cols) return cudaSuccess;
    const uint32_t parts = act_backward_parts(d.rows, d.cols);
    // the wide form: whole aligned groups of 8 columns, and one type for z, mul, dz and dmul
    uint32_t type = d.z ? d.z_type : (d.dz ? d.dz_type : d.dy_type);
    auto fits = [&](const void* p, uint32_t t, uint64_t ld) { return !p || (t == type && rows_wide(p, ld, t)); };
    const bool wide = d.cols % 8 == 0 && rows_wide(d.dy, d.lddy, d.dy_type) && fits(d.z, d.z_type, d.ldz) && fits(d.mul, d.mul_type, d.ldmul) &&
                      fits(d.dz, d.dz_type, d.lddz) && fits(d.dmul, d.dmul_type, d.lddmul);
    Sums b = {ws, parts, 0u};
    const bool one_launch = d.dbias && parts && (d.rows <= join_rows(d.act) || parts == 1);
    if (one_launch) {
        b.bands = std::min(parts, kJoinBands);
        b.joined = b.bands > 1;
        b.out = d.dbias;
    }
    cudaError_t e = cudaSuccess;
    if (parts) e = d.mul ? launch_act<true>(d, b, wide, type, st) : launch_act<false>(d, b, wide, type, st);
    if (e != cudaSuccess || !d.dbias || one_launch) return e;
    return launch_sum_parts(ws, parts, d.cols, d.dbias, st);
}

}  // namespace cleave
