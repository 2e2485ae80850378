// Pieces that the row-wise operators share: sums over a CTA, a row's columns in registers, rows in 8 bits (internal).
#pragma once

#include "ops.cuh"

namespace cleave {

constexpr uint32_t kRowThreads = 256;           // of the forms for any shape

// Sum / NaN-keeping maximum over the CTA; every thread receives it.  `buf` holds one value per warp and may be
// reused after the call (it ends with a barrier).
__device__ __forceinline__ float cta_sum(float v, float* buf) {
    v = warp_sum(v);
    if ((threadIdx.x & 31u) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.f;
    for (uint32_t w = 0; w < blockDim.x / 32; ++w) s += buf[w];
    __syncthreads();
    return s;
}
__device__ __forceinline__ float cta_max_nan(float v, float* buf) {
    v = warp_abs_max(v);
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

// ---- a row held by its CTA, any alignment, up to 8192 columns ---------------------------------------------
// A thread owns the columns tid, tid + T, ...: kOwn of them stay in registers, and the next row's are asked for before
// this row's sums are joined.
constexpr uint32_t kOwn = 8, kOwnCols = kOwn * 1024;

// Raw words (a bf16's bits below), so that nothing waits for a load before all of them are on their way; columns that do
// not exist repeat the last one and are cleared by own_values.
__device__ __forceinline__ void load_own(const void* p, uint32_t type, uint64_t at, uint32_t cols, uint32_t (&x)[kOwn]) {
    if (type == CLEAVE_T_F32) {
        const uint32_t* s = static_cast<const uint32_t*>(p) + at;
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) x[k] = s[min(threadIdx.x + k * blockDim.x, cols - 1)];
    } else {
        const uint16_t* s = static_cast<const uint16_t*>(p) + at;
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) x[k] = s[min(threadIdx.x + k * blockDim.x, cols - 1)];
    }
}
__device__ __forceinline__ void own_values(const uint32_t (&raw)[kOwn], uint32_t type, uint32_t cols, float (&x)[kOwn]) {
    const uint32_t shift = type == CLEAVE_T_F32 ? 0u : 16u;
#pragma unroll
    for (uint32_t k = 0; k < kOwn; ++k) x[k] = threadIdx.x + k * blockDim.x < cols ? __uint_as_float(raw[k] << shift) : 0.f;
}
__device__ __forceinline__ void store_own(void* p, uint32_t type, uint64_t at, uint32_t cols, const float (&x)[kOwn]) {
    if (type == CLEAVE_T_F32) {
        float* s = static_cast<float*>(p) + at;
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) { const uint32_t j = threadIdx.x + k * blockDim.x; if (j < cols) s[j] = x[k]; }
    } else if (type == CLEAVE_T_BF16) {
        __nv_bfloat16* s = static_cast<__nv_bfloat16*>(p) + at;
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) { const uint32_t j = threadIdx.x + k * blockDim.x; if (j < cols) s[j] = __float2bfloat16_rn(x[k]); }
    } else {
        uint8_t* s = static_cast<uint8_t*>(p) + at;
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) { const uint32_t j = threadIdx.x + k * blockDim.x; if (j < cols) s[j] = e4m3_nearest(x[k]); }
    }
}
// sum and NaN-keeping maximum over the CTA with one barrier; the buffers take turns
__device__ __forceinline__ float2 cta_join(float sum, float top, float2* p) {
    sum = warp_sum(sum);
    top = warp_abs_max(top);
    if (blockDim.x == 32) return make_float2(sum, top);
    if ((threadIdx.x & 31u) == 0) p[threadIdx.x >> 5] = make_float2(sum, top);
    __syncthreads();
    const float2 q = (threadIdx.x & 31u) < blockDim.x / 32 ? p[threadIdx.x & 31u] : make_float2(0.f, 0.f);
    return make_float2(warp_sum(q.x), warp_abs_max(q.y));
}

inline uint32_t own_threads(uint32_t cols) { return (cols + 32 * kOwn - 1) / (32 * kOwn) * 32; }

// ---- 8 columns at a time ----------------------------------------------------------------------------------
struct NoRes {};                    // no residual operand
template <typename T> struct Bytes8 { static constexpr uint32_t value = sizeof(T) * 8; };
template <> struct Bytes8<NoRes> { static constexpr uint32_t value = 0; };

template <typename Desc>
__device__ __forceinline__ void load_weight8(const Desc& d, uint32_t col, F2 (&w)[4]) {      // (the same for every row: L1)
    if (d.w_type == CLEAVE_T_F32) {
        Raw8<float> r;
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(d.w) + col);
        r.w[0] = p[0]; r.w[1] = p[1];
        unpack8(r, w);
    } else if (d.w_type == CLEAVE_T_BF16) {
        Raw8<__nv_bfloat16> r;
        r.w[0] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(d.w) + col);
        unpack8(r, w);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = f2(1.f, 1.f);
    }
}
// largest magnitude of a pair and `top`; a NaN stays
__device__ __forceinline__ float top2(float top, F2 a) {
    const float2 h = halves(a);
    return max_nan(max_nan(top, fabsf(h.x)), fabsf(h.y));
}

}  // namespace cleave
