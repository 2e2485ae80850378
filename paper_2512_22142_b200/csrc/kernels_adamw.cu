// adamw_kernel: one optimizer step over the elements of many tensors (see cleave.h for the formula and the
// 8-bit states).
//
// One warp per block of 256 elements, a CTA of 8 warps per chunk of up to 32 neighbouring blocks of one tensor.  The
// work list (tensor, first block) is made once per handle, so tensors of any number and size share one launch.  Lane l owns the elements 4 l .. 4 l + 3 of both
// halves of the block: every fp32 access of a warp is 512 consecutive bytes, and a block's largest magnitude is
// a shuffle reduction inside its warp, so an 8-bit state needs no second pass.
// Bound by the HBM's bandwidth: 30 bytes an element with fp32 states (gradient 4, weight 8, states 16, copy 2),
// 18 with 8-bit ones.
#include <cuda_fp16.h>

#include "ops.cuh"

namespace cleave {

// SplitMix64's output function
__device__ __forceinline__ uint64_t mix64(uint64_t x) {
    x += 0x9E3779B97F4A7C15ull;
    x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
    x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
    return x ^ (x >> 31);
}

// E4M3 magnitude code of |q| <= 448 (rounding of the scale may leave it a unit above), away from zero with the
// probability of what is cut off (u: 16 random bits).  From 2^-6 on three mantissa bits stay, so the random bits are
// added right below them and the rest is cut; below (a few elements in ten thousand), codes are multiples of 2^-9.
__device__ __forceinline__ uint32_t stochastic_code(float q, uint32_t u) {
    const float a = fabsf(q);
    uint32_t code = ((__float_as_uint(a) + (u << 4)) >> 20) - 960u;                 // exponent bias 127 - 7, 3 mantissa bits
    if (a < 0.015625f) code = (uint32_t)floorf(__fadd_rn(__fmul_rn(a, 512.f), __fmul_rn((float)u, 1.f / 65536.f)));
    return min(code, 0x7Eu);
}

template <bool WIDE, typename T>
__device__ __forceinline__ void load4(const T* src, uint64_t e, uint64_t n, float (&x)[4]) {
    if constexpr (WIDE) {
        if constexpr (sizeof(T) == 4) {
            const float4 v = *reinterpret_cast<const float4*>(src + e);
            x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2*>(src + e);
            const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.x)), b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.y));
            x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = e + i < n ? to_f32<T>(src[e + i]) : 0.f;
    }
}
template <bool WIDE>
__device__ __forceinline__ void load4_codes(const uint8_t* src, uint64_t e, uint64_t n, float (&x)[4]) {
    if constexpr (WIDE) {
        const uint32_t c = *reinterpret_cast<const uint32_t*>(src + e);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(h ? c >> 16 : c & 0xFFFFu), __NV_E4M3);
            const float2 f = __half22float2(__half2(r));
            x[2 * h] = f.x; x[2 * h + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = e + i < n ? e4m3_value(src[e + i]) : 0.f;
    }
}
template <bool WIDE>
__device__ __forceinline__ void store4(float* dst, uint64_t e, uint64_t n, const float (&x)[4]) {
    if constexpr (WIDE) *reinterpret_cast<float4*>(dst + e) = make_float4(x[0], x[1], x[2], x[3]);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) if (e + i < n) dst[e + i] = x[i];
}
template <bool WIDE>
__device__ __forceinline__ void store4(__nv_bfloat16* dst, uint64_t e, uint64_t n, const float (&x)[4]) {
    if constexpr (WIDE) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
        *reinterpret_cast<uint2*>(dst + e) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    } else
#pragma unroll
        for (int i = 0; i < 4; ++i) if (e + i < n) dst[e + i] = __float2bfloat16_rn(x[i]);
}
template <bool WIDE>                       // codes in the top bytes of c
__device__ __forceinline__ void store4_codes(uint8_t* dst, uint64_t e, uint64_t n, const uint32_t (&c)[4]) {
    if constexpr (WIDE)
        *reinterpret_cast<uint32_t*>(dst + e) = __byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) if (e + i < n) dst[e + i] = (uint8_t)(c[i] >> 24);
}

// largest magnitude of the warp's values; a NaN stays
__device__ __forceinline__ float warp_abs_max(float v) {
    float r;
    asm volatile("redux.sync.max.abs.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
// scale of a block whose largest magnitude is `top`, and its reciprocal (both 0 when there is nothing to scale)
__device__ __forceinline__ float2 block_scale(float top) {
    const float s = top < 0x1p-100f ? 0.f : __fmul_rn(top, 1.f / kE4M3Max);
    return make_float2(s, s == 0.f ? 0.f : __frcp_rn(s));
}

// What an element's code needs besides its value: 16 random bits of `word` moved to where the 20 cut bits begin.
__device__ __forceinline__ uint32_t bits_low(uint32_t w) { return (w << 4) & 0xFFFF0u; }
__device__ __forceinline__ uint32_t bits_high(uint32_t w) { return (w >> 12) & 0xFFFF0u; }

// One block of 256 elements; WIDE: the block is whole and its buffers are aligned.
template <bool STATE8, typename G, bool WIDE>
__device__ __forceinline__ void adamw_block(const AdamTensor& t, float decay, uint64_t key, uint64_t block, const AdamStep& s, uint32_t lane) {
    const uint64_t n = t.numel, e0 = block * kStateBlock + lane * 4u;
    float m[2][4], r[2][4], p[2][4], g[2][4];
    float sm = 0.f, sv = 0.f;
    if constexpr (STATE8) { sm = t.m_scale[block]; sv = t.v_scale[block]; }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint64_t e = e0 + j * 128u;
        load4<WIDE>(static_cast<const G*>(t.g), e, n, g[j]);
        load4<WIDE>(t.p, e, n, p[j]);
        if constexpr (STATE8) { load4_codes<WIDE>(static_cast<const uint8_t*>(t.m), e, n, m[j]); load4_codes<WIDE>(static_cast<const uint8_t*>(t.v), e, n, r[j]); }
        else                  { load4<WIDE>(static_cast<const float*>(t.m), e, n, m[j]); load4<WIDE>(static_cast<const float*>(t.v), e, n, r[j]); }
    }
    float top_m = 0.f, top_r = 0.f;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float gr = __fmul_rn(g[j][i], s.grad_scale);
            float mo = m[j][i], vo = r[j][i];
            if constexpr (STATE8) {
                mo = __fmul_rn(mo, sm);
                const float root = __fmul_rn(vo, sv);
                vo = __fmul_rn(root, root);
            }
            mo = __fadd_rn(__fmul_rn(mo, s.beta1), __fmul_rn(gr, s.omb1));
            vo = __fadd_rn(__fmul_rn(vo, s.beta2), __fmul_rn(__fmul_rn(gr, gr), s.omb2));
            const float root = __fsqrt_rn(vo);
            const float den = __fadd_rn(__fmul_rn(root, s.root), s.eps);
            p[j][i] = __fsub_rn(__fmul_rn(p[j][i], decay), __fmul_rn(__fdiv_rn(mo, den), s.step_size));
            m[j][i] = mo;
            if constexpr (STATE8) { r[j][i] = root; top_m = max_nan(top_m, fabsf(mo)); top_r = max_nan(top_r, root); }
            else r[j][i] = vo;
        }
        const uint64_t e = e0 + j * 128u;
        store4<WIDE>(t.p, e, n, p[j]);
        if (t.w) store4<WIDE>(t.w, e, n, p[j]);
        if constexpr (!STATE8) { store4<WIDE>(static_cast<float*>(t.m), e, n, m[j]); store4<WIDE>(static_cast<float*>(t.v), e, n, r[j]); }
    }
    if constexpr (STATE8) {
        top_m = warp_abs_max(top_m);
        top_r = warp_abs_max(top_r);
        const float2 bm = block_scale(top_m), bv = block_scale(top_r);
        const bool odd = !(top_m < INFINITY) || !(top_r < INFINITY);       // NaN or infinity: some codes have to be NaN
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint64_t e = e0 + j * 128u;
            float qm[4], qv[4];
            uint32_t w[4], cm[4], cv[4];                                    // w: the element's 32 random bits
            float least = INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                qm[i] = __fmul_rn(m[j][i], bm.y);
                qv[i] = __fmul_rn(r[j][i], bv.y);
                least = fminf(fminf(least, fabsf(qm[i])), qv[i]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint64_t word = mix64(key + (e >> 1) + h);
                w[2 * h] = (uint32_t)word; w[2 * h + 1] = (uint32_t)(word >> 32);
            }
            if (least >= 0.015625f && !odd) {
                // every value has three mantissa bits left: the code is bits 20-26 of its magnitude plus the random
                // bits, less 960 << 20 (exponent bias 127 - 7).  448 and a few units above it stay below the next code.
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    cm[i] = (((__float_as_uint(qm[i]) & 0x7FFFFFFFu) + bits_low(w[i]) - (960u << 20)) << 4 & 0x7F000000u) | (__float_as_uint(qm[i]) & 0x80000000u);
                    cv[i] = (__float_as_uint(qv[i]) + bits_high(w[i]) - (960u << 20)) << 4;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t a = stochastic_code(qm[i], w[i] & 0xFFFFu), b = stochastic_code(qv[i], w[i] >> 16);
                    if (qm[i] < 0.f) a |= 0x80u;
                    if (qv[i] > 0.f) b = max(b, 1u);
                    if (qm[i] != qm[i]) a = 0x7Fu;
                    if (qv[i] != qv[i]) b = 0x7Fu;
                    cm[i] = a << 24; cv[i] = b << 24;
                }
            }
            store4_codes<WIDE>(static_cast<uint8_t*>(t.m), e, n, cm);
            store4_codes<WIDE>(static_cast<uint8_t*>(t.v), e, n, cv);
        }
        if (lane == 0) { t.m_scale[block] = bm.x; t.v_scale[block] = bv.x; }
    }
}

template <bool STATE8, typename G>
__global__ void __launch_bounds__(32 * kChunkWarps, 3)
adamw_kernel(const AdamTensor* __restrict__ tensors, const AdamChunk* __restrict__ chunks, uint32_t chunk_blocks, const __grid_constant__ AdamStep s) {
    const AdamChunk c = chunks[blockIdx.x];
    const AdamTensor t = tensors[c.tensor];
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t key = STATE8 ? mix64(mix64(s.base + c.tensor)) : 0ull;
    const float decay = (float)__dadd_rn(1.0, -__dmul_rn(s.lr, t.weight_decay));
    for (uint32_t k = threadIdx.x >> 5; k < chunk_blocks; k += kChunkWarps) {
        const uint64_t block = (uint64_t)c.block0 + k;
        if (block * kStateBlock >= t.numel) return;
        if (t.wide && (block + 1) * kStateBlock <= t.numel) adamw_block<STATE8, G, true>(t, decay, key, block, s, lane);
        else adamw_block<STATE8, G, false>(t, decay, key, block, s, lane);
    }
}

cudaError_t launch_adamw(const AdamTensor* tensors, const AdamChunk* chunks, uint32_t n_chunks, uint32_t chunk_blocks, const AdamStep& s,
                         bool state8, bool g_bf16, cudaStream_t st) {
    if (!n_chunks) return cudaSuccess;
    const dim3 block(32 * kChunkWarps);
    if (state8) {
        if (g_bf16) adamw_kernel<true, __nv_bfloat16><<<n_chunks, block, 0, st>>>(tensors, chunks, chunk_blocks, s);
        else        adamw_kernel<true, float><<<n_chunks, block, 0, st>>>(tensors, chunks, chunk_blocks, s);
    } else {
        if (g_bf16) adamw_kernel<false, __nv_bfloat16><<<n_chunks, block, 0, st>>>(tensors, chunks, chunk_blocks, s);
        else        adamw_kernel<false, float><<<n_chunks, block, 0, st>>>(tensors, chunks, chunk_blocks, s);
    }
    return cudaGetLastError();
}

}  // namespace cleave
