// adamw_kernel: one optimizer step over the elements of many tensors (see cleave.h for the formula and the
// 8-bit states).
//
// One warp per block of 256 elements, a CTA of 8 warps per chunk of up to 256 neighbouring blocks of one tensor.  The
// work list (tensor, first block) is made once per handle, so tensors of any number and size share one launch.  Lane l
// owns the elements 4 l .. 4 l + 3 of both halves of the block: every fp32 access of a warp is 512 consecutive bytes, and
// a block's largest magnitude is a reduction inside its warp, so an 8-bit state needs no second pass.  A warp's next
// blocks are on their way to shared memory (three stages of its own, no barrier) while one is used.
// Bytes an element: 30 with fp32 states (gradient 4, weight 8, states 16, copy 2; 28 with bf16 gradients), 18 with 8-bit
// ones.  fp32 states are bound by the HBM (a layer of width 768, 7.1 M elements: 35 us, 5.7 TB/s).  8-bit states are bound
// by instruction issue (73 % of the cycles issue, 64 % of the HBM's): two roundings with random bits, a division and a
// root an element; 202 M elements take 691 us a step of one optimizer after another (5.3 TB/s), 720 with three in turn.
#include <cuda_fp16.h>

#include <type_traits>

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

// Four consecutive elements of a lane.  `whole`: all four exist and the buffer allows one wide access.
template <typename T>
__device__ __forceinline__ void unpack4(const T* p, float (&x)[4]) {
    if constexpr (sizeof(T) == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else if constexpr (sizeof(T) == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xFFFF0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xFFFF0000u);
    } else {                                                          // E4M3 codes
        const uint32_t c = *reinterpret_cast<const uint32_t*>(p);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(h ? c >> 16 : c & 0xFFFFu), __NV_E4M3);
            const float2 f = __half22float2(__half2(r));
            x[2 * h] = f.x; x[2 * h + 1] = f.y;
        }
    }
}
__device__ __forceinline__ float element(const float* p) { return *p; }
__device__ __forceinline__ float element(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float element(const uint8_t* p) { return e4m3_value(*p); }
template <typename T>
__device__ __forceinline__ void load4(const T* src, uint64_t e, uint64_t n, bool whole, float (&x)[4]) {
    if (whole) unpack4(src + e, x);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = e + i < n ? element(src + e + i) : 0.f;
}
__device__ __forceinline__ void store4(float* dst, uint64_t e, uint64_t n, bool whole, const float (&x)[4]) {
    if (whole) *reinterpret_cast<float4*>(dst + e) = make_float4(x[0], x[1], x[2], x[3]);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) if (e + i < n) dst[e + i] = x[i];
}
__device__ __forceinline__ void store4(__nv_bfloat16* dst, uint64_t e, uint64_t n, bool whole, const float (&x)[4]) {
    if (whole) *reinterpret_cast<uint2*>(dst + e) = make_uint2(bf16x2(x[0], x[1]), bf16x2(x[2], x[3]));
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) if (e + i < n) dst[e + i] = __float2bfloat16_rn(x[i]);
}
// codes in the top bytes of c
__device__ __forceinline__ void store4(uint8_t* dst, uint64_t e, uint64_t n, bool whole, const uint32_t (&c)[4]) {
    if (whole) *reinterpret_cast<uint32_t*>(dst + e) = __byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) if (e + i < n) dst[e + i] = (uint8_t)(c[i] >> 24);
}

// scale of a block whose largest magnitude is `top`, and its reciprocal (both 0 when there is nothing to scale)
__device__ __forceinline__ float2 block_scale(float top) {
    const float s = top < 0x1p-100f ? 0.f : __fmul_rn(top, 1.f / kE4M3Max);
    return make_float2(s, s == 0.f ? 0.f : __frcp_rn(s));
}

// three-input forms (one instruction)
__device__ __forceinline__ float abs_max3(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float abs_min3(float a, float b, float c) {
    float r;
    asm("min.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// The update of one block of 256 elements whose values the warp holds (lane: elements 4 lane .. + 3 of both halves),
// and its stores.  WHOLE: the block is complete and its buffers are aligned.
template <bool STATE8, bool WHOLE>
__device__ __forceinline__ void adamw_block(const AdamTensor& t, float decay, uint64_t key, uint64_t block, const AdamStep& s, uint32_t lane,
                                            float (&g)[2][4], float (&p)[2][4], float (&m)[2][4], float (&r)[2][4], float sm, float sv) {
    const uint64_t n = t.numel, e0 = block * kStateBlock + lane * 4u;
    const bool whole[2] = {WHOLE || (t.wide && e0 + 4 <= n), WHOLE || (t.wide && e0 + 132 <= n)};
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
            r[j][i] = STATE8 ? root : vo;
        }
        if constexpr (STATE8) {
            top_m = abs_max3(abs_max3(top_m, m[j][0], m[j][1]), m[j][2], m[j][3]);
            top_r = abs_max3(abs_max3(top_r, r[j][0], r[j][1]), r[j][2], r[j][3]);
        }
        const uint64_t e = e0 + j * 128u;
        store4(t.p, e, n, whole[j], p[j]);
        if (t.w) store4(t.w, e, n, whole[j], p[j]);
        if constexpr (!STATE8) { store4(static_cast<float*>(t.m), e, n, whole[j], m[j]); store4(static_cast<float*>(t.v), e, n, whole[j], r[j]); }
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
                least = abs_min3(least, qm[i], qv[i]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint64_t word = mix64(key + (e >> 1) + h);
                w[2 * h] = (uint32_t)word; w[2 * h + 1] = (uint32_t)(word >> 32);
            }
            if (least >= 0.015625f && !odd) {
                // Every value has three mantissa bits left: the code is bits 20-26 of its magnitude plus the random bits
                // (moved to where the 20 cut bits begin), less 960 << 20 (exponent bias 127 - 7).  448 and a few units
                // above it stay below the next code.  Written as products, sixteenfold, so that the code ends in the
                // top byte: the integer multiply-add has a pipe of its own, shifts and masks share the busy one.
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t um = __byte_perm(w[i], 0, 0x4410), uv = __byte_perm(w[i], 0, 0x4432);
                    const uint32_t am = (__float_as_uint(qm[i]) & 0x7FFFFFFFu) * 16u + (0u - (960u << 24)), av = __float_as_uint(qv[i]) * 16u + (0u - (960u << 24));
                    cm[i] = ((um * 256u + am) & 0x7F000000u) | (__float_as_uint(qm[i]) & 0x80000000u);
                    cv[i] = uv * 256u + av;
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
            store4(static_cast<uint8_t*>(t.m), e, n, whole[j], cm);
            store4(static_cast<uint8_t*>(t.v), e, n, whole[j], cv);
        }
        if (lane == 0) { t.m_scale[block] = bm.x; t.v_scale[block] = bv.x; }
    }
}

// A warp's ring of blocks on their way to shared memory: each lane copies and reads its own elements only.
template <bool STATE8, typename G> struct AdamStage {
    using S = typename std::conditional<STATE8, uint8_t, float>::type;
    static constexpr uint32_t g = 256 * 4, m = g + 256 * sizeof(G), v = m + 256 * sizeof(S), scales = v + 256 * sizeof(S);
    static constexpr uint32_t bytes = scales + (STATE8 ? 2 * 32 * 4 : 0);
    static constexpr int stages = 3;
};

template <bool STATE8, typename G>
__global__ void __launch_bounds__(32 * kChunkWarps, 3)
adamw_kernel(const AdamTensor* tensors, const AdamChunk* chunks, uint32_t chunk_blocks, const __grid_constant__ AdamStep s) {
    using Stage = AdamStage<STATE8, G>;
    using S = typename Stage::S;
    extern __shared__ __align__(16) uint8_t ring[];
    begin_chained();
    const AdamChunk c = chunks[blockIdx.x];
    const AdamTensor t = tensors[c.tensor];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint64_t key = STATE8 ? mix64(mix64(s.base + c.tensor)) : 0ull;
    const float decay = (float)__dadd_rn(1.0, -__dmul_rn(s.lr, t.weight_decay));
    const uint64_t all = (t.numel + kStateBlock - 1) / kStateBlock;
    const uint64_t end = min(all, (uint64_t)c.block0 + chunk_blocks);
    const uint64_t whole_end = t.wide ? min(end, t.numel / kStateBlock) : c.block0;        // blocks below it go through the ring
    uint64_t block = (uint64_t)c.block0 + warp, ahead = block;
    const G* const tg = static_cast<const G*>(t.g);
    const S* const tm = static_cast<const S*>(t.m);
    const S* const tv = static_cast<const S*>(t.v);
    uint8_t* const mine = ring + warp * (Stage::stages * Stage::bytes);
    const uint32_t mine_at = (uint32_t)__cvta_generic_to_shared(mine);
    auto fetch = [&](uint32_t at) {
        if (ahead < whole_end) {
            const uint64_t e = ahead * kStateBlock + lane * 4u;
            const uint32_t to = mine_at + at;
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j) {
                const uint32_t o = lane * 4u + j * 128u;
                cp_async<16>(to + o * 4u, t.p + e + j * 128u);
                cp_async<4 * sizeof(G)>(to + Stage::g + o * (uint32_t)sizeof(G), tg + e + j * 128u);
                cp_async<4 * sizeof(S)>(to + Stage::m + o * (uint32_t)sizeof(S), tm + e + j * 128u);
                cp_async<4 * sizeof(S)>(to + Stage::v + o * (uint32_t)sizeof(S), tv + e + j * 128u);
            }
            if constexpr (STATE8) {
                cp_async<4>(to + Stage::scales + lane * 4u, t.m_scale + ahead);
                cp_async<4>(to + Stage::scales + 128u + lane * 4u, t.v_scale + ahead);
            }
            ahead += kChunkWarps;
        }
        cp_async_commit();
    };
#pragma unroll
    for (int k = 0; k < Stage::stages; ++k) fetch(k * Stage::bytes);
    uint32_t at = 0;
    float g[2][4], p[2][4], m[2][4], r[2][4], sm = 0.f, sv = 0.f;
    for (; block < whole_end; block += kChunkWarps) {
        cp_async_wait<Stage::stages - 1>();
        const uint8_t* stage = mine + at;
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) {
            const uint32_t o = lane * 4u + j * 128u;
            unpack4(reinterpret_cast<const float*>(stage) + o, p[j]);
            unpack4(reinterpret_cast<const G*>(stage + Stage::g) + o, g[j]);
            unpack4(reinterpret_cast<const S*>(stage + Stage::m) + o, m[j]);
            unpack4(reinterpret_cast<const S*>(stage + Stage::v) + o, r[j]);
        }
        if constexpr (STATE8) {
            sm = *reinterpret_cast<const float*>(stage + Stage::scales + lane * 4u);
            sv = *reinterpret_cast<const float*>(stage + Stage::scales + 128u + lane * 4u);
        }
        adamw_block<STATE8, true>(t, decay, key, block, s, lane, g, p, m, r, sm, sv);
        __syncwarp();
        fetch(at);                                                    // the stage's values have been used
        at = at + Stage::bytes == Stage::stages * Stage::bytes ? 0 : at + Stage::bytes;
    }
    // a block that is not whole, or buffers that are not aligned: straight from global memory
    for (; block < end; block += kChunkWarps) {
        if constexpr (STATE8) { sm = t.m_scale[block]; sv = t.v_scale[block]; }
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) {
            const uint64_t e = block * kStateBlock + lane * 4u + j * 128u;
            const bool whole = t.wide && e + 4 <= t.numel;
            load4(tg, e, t.numel, whole, g[j]);
            load4(const_cast<const float*>(t.p), e, t.numel, whole, p[j]);
            load4(tm, e, t.numel, whole, m[j]);
            load4(tv, e, t.numel, whole, r[j]);
        }
        adamw_block<STATE8, false>(t, decay, key, block, s, lane, g, p, m, r, sm, sv);
    }
}

template <bool STATE8, typename G>
cudaError_t launch_adamw_as(const AdamTensor* tensors, const AdamChunk* chunks, uint32_t n_chunks, uint32_t chunk_blocks, const AdamStep& s, cudaStream_t st) {
    using Stage = AdamStage<STATE8, G>;
    constexpr uint32_t smem = kChunkWarps * Stage::stages * Stage::bytes;
    auto kernel = adamw_kernel<STATE8, G>;
    static SmemLimit limit;
    const cudaError_t e = limit.raise(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return e;
    return launch_chained(kernel, n_chunks, 32 * kChunkWarps, smem, st, tensors, chunks, chunk_blocks, s);
}

cudaError_t launch_adamw(const AdamTensor* tensors, const AdamChunk* chunks, uint32_t n_chunks, uint32_t chunk_blocks, const AdamStep& s,
                         bool state8, bool g_bf16, cudaStream_t st) {
    if (!n_chunks) return cudaSuccess;
    if (state8) return g_bf16 ? launch_adamw_as<true, __nv_bfloat16>(tensors, chunks, n_chunks, chunk_blocks, s, st)
                              : launch_adamw_as<true, float>(tensors, chunks, n_chunks, chunk_blocks, s, st);
    return g_bf16 ? launch_adamw_as<false, __nv_bfloat16>(tensors, chunks, n_chunks, chunk_blocks, s, st)
                  : launch_adamw_as<false, float>(tensors, chunks, n_chunks, chunk_blocks, s, st);
}

}  // namespace cleave
