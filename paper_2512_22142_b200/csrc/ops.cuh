// Shared pieces of the operators around the GEMMs: element types, activations, 8-bit codes, launcher
// declarations (internal).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "cleave.h"

namespace cleave {

constexpr float kE4M3Max = 448.f;
constexpr uint32_t kStateBlock = 256;            // elements that share a scale in an 8-bit optimizer state

inline uint32_t type_bytes(uint32_t t) { return t == CLEAVE_T_F32 ? 4u : (t == CLEAVE_T_BF16 ? 2u : (t == CLEAVE_T_E4M3 ? 1u : 0u)); }

// The operators' kernels are launched so that a kernel may start while the one before it in the stream still runs: the
// first lets its dependents start at its beginning, the second sets itself up and then waits until the first has
// ended and its results are visible, before it touches any memory.  Stream order is what it always is; a launch's
// own latency (2 to 3 us) passes beside the kernel before it.  No load here goes by the read-only path (ld.global.nc):
// the memory may still change after the kernel has begun, before its wait ends.
__device__ __forceinline__ void let_dependents_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_primary() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void begin_chained() { let_dependents_start(); wait_for_primary(); }
template <typename... P, typename... A>
cudaError_t launch_chained_clusters(void (*kernel)(P...), dim3 cluster, dim3 grid, dim3 block, uint32_t smem, cudaStream_t st, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster.x; attr[1].val.clusterDim.y = cluster.y; attr[1].val.clusterDim.z = cluster.z;
    cfg.attrs = attr;
    cfg.numAttrs = cluster.x * cluster.y * cluster.z > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}
template <typename... P, typename... A>
cudaError_t launch_chained(void (*kernel)(P...), dim3 grid, dim3 block, uint32_t smem, cudaStream_t st, const A&... args) {
    return launch_chained_clusters(kernel, dim3(1), grid, block, smem, st, args...);
}

// Raises a kernel's dynamic shared memory limit, once per device.
struct SmemLimit {
    std::atomic<uint64_t> devices{0};
    cudaError_t raise(const void* kernel, int bytes) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const uint64_t bit = dev < 64 ? 1ull << dev : 0ull;
        if (devices.load(std::memory_order_relaxed) & bit) return cudaSuccess;
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == cudaSuccess) devices.fetch_or(bit, std::memory_order_relaxed);
        return e;
    }
};

// ---- elements ----------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// element `i` of an operand whose type is only known at run time (edges; the wide paths are typed)
__device__ __forceinline__ float load_as(const void* p, uint32_t type, uint64_t i) {
    return type == CLEAVE_T_F32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
__device__ __forceinline__ void store_as(void* p, uint32_t type, uint64_t i, float v) {
    if (type == CLEAVE_T_F32) static_cast<float*>(p)[i] = v;
    else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}

// largest of two values; a NaN in either stays (fmaxf would drop it)
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ uint8_t e4m3_nearest(float v) { return (uint8_t)__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ float e4m3_value(uint8_t code) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3)));
}

// ---- 8 consecutive elements: 16 bytes of bf16 or 32 of fp32, as raw words and as fp32 -----------------------
template <typename T> struct Raw8;
template <> struct Raw8<float> { uint4 w[2]; };
template <> struct Raw8<__nv_bfloat16> { uint4 w[1]; };
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw8(const T* p) {           // read once: the line need not stay in L1
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r.w) / 16); ++i) r.w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    return r;
}
__device__ __forceinline__ void unpack8(const Raw8<float>& r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[4 * i] = __uint_as_float(r.w[i].x); x[4 * i + 1] = __uint_as_float(r.w[i].y);
        x[4 * i + 2] = __uint_as_float(r.w[i].z); x[4 * i + 3] = __uint_as_float(r.w[i].w);
    }
}
__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16>& r, float (&x)[8]) {
    const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(bf16x2(x[0], x[1]), bf16x2(x[2], x[3]), bf16x2(x[4], x[5]), bf16x2(x[6], x[7]));
}
// eight E4M3 codes (to nearest even, magnitudes above 448 become 448)
__device__ __forceinline__ void store8(uint8_t* p, const float (&x)[8]) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(x[4 * i], x[4 * i + 1]), __NV_SATFINITE, __NV_E4M3) |
               ((uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(x[4 * i + 2], x[4 * i + 3]), __NV_SATFINITE, __NV_E4M3) << 16);
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}
// the wide accesses apply: base and rows 16-byte aligned (8 bytes for rows of codes), whole groups of 8 columns
inline bool rows_wide(const void* p, uint64_t ld, uint32_t type) {
    const uint64_t unit = type == CLEAVE_T_E4M3 ? 8 : 16;
    return (uintptr_t)p % unit == 0 && (ld * type_bytes(type)) % unit == 0;
}

// ---- two fp32 values in one register pair --------------------------------------------------------------------------
// (A product and a sum of pairs may be contracted: not for what is defined to the bit.)
typedef unsigned long long F2;
__device__ __forceinline__ F2 f2(float lo, float hi) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 halves(F2 a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a));
    return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ void unpack8(const Raw8<float>& r, F2 (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[2 * i] = f2(__uint_as_float(r.w[i].x), __uint_as_float(r.w[i].y));
        x[2 * i + 1] = f2(__uint_as_float(r.w[i].z), __uint_as_float(r.w[i].w));
    }
}
__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16>& r, F2 (&x)[4]) {
    const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const F2 (&x)[4]) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 h = halves(x[i]); y[2 * i] = h.x; y[2 * i + 1] = h.y; }
    store8(p, y);
}

// ---- asynchronous copies into shared memory, and warp reductions ----------------------------------------
// A thread copies only what it reads itself, so a ring of such copies needs no barrier: the thread's own group count
// says when a stage has landed.
template <int BYTES>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
// largest magnitude of the warp's values; a NaN stays
__device__ __forceinline__ float warp_abs_max(float v) {
    float r;
    asm volatile("redux.sync.max.abs.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// ---- activations ----------------------------------------------------------------------------------
// The two forms with an exponential are z g with g = 1 / (1 + e), e = exp(-t): one exponential (base 2, the factor
// log2(e) in the argument's constants) and one reciprocal of a value of at least 1, both the hardware's
// approximations (a few units in the last place; what they flush to zero is below 2^-126).  Where e overflows g is 0
// (the limit); no 1 - tanh cancellation on the negative side.  In the slopes 1 - g loses relative accuracy only
// where g is close to 1 and the term it belongs to vanishes against g.
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float rcp_fast(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// 1 / (1 + exp(-2 sqrt(2/pi) (z + 0.044715 z^3))) and 1 / (1 + exp(-z))
__device__ __forceinline__ float gelu_tanh_gate(float z) {
    return rcp_fast(1.f + exp2_fast(-z * fmaf(0.1029432407f, z * z, 2.3022081983f)));
}
__device__ __forceinline__ float silu_gate(float z) { return rcp_fast(1.f + exp2_fast(-1.4426950409f * z)); }
// Phi(z), the normal distribution, and exp(-z^2 / 2), with one reciprocal and one exponential (8192 x 768 x 3072 with z takes
// 48.3 us, with the tanh form 43.4; erfcf takes far longer: 84 against 24 us where an earlier polynomial of degree 4
// stood in the write-out of 39 M elements).  On the negative side Phi(z) = t P(t) exp(-z^2 / 2) with
// t = 1 / (1 + 0.30405593 |z|): 0.5 erfcx(|z| / sqrt(2)) / t is smooth in t, and P is its polynomial of degree 7 with the
// smallest largest relative error over |z| <= 13.3 (8.4e-8; fitted by reweighted least squares on Chebyshev points).
// In fp32 Phi's relative error is at most 16 (1 + z^2) 2^-24, tail included (the exponent's rounding grows with z^2, as
// does what half a unit of z itself makes); where exp underflows, below z = -13.2, Phi is 0.
__device__ __forceinline__ float2 normal_cdf(float z) {
    const float a = fabsf(z), t = rcp_fast(fmaf(0.30405593f, a, 1.f));
    float p = fmaf(0.036853947f, t, -0.15518661f);
    p = fmaf(p, t, 0.19185269f);
    p = fmaf(p, t, -0.042862743f);
    p = fmaf(p, t, 0.12342216f);
    p = fmaf(p, t, 0.10247557f);
    p = fmaf(p, t, 0.122187726f);
    p = fmaf(p, t, 0.12125731f);
    const float e = exp2_fast(-0.72134752f * a * a), tail = p * t * e;
    return make_float2(z > 0.f ? 1.f - tail : tail, e);
}
__device__ __forceinline__ float act_value(float z, uint32_t act) {
    switch (act) {
        case CLEAVE_ACT_RELU: return z > 0.f ? z : (z != z ? z : 0.f);
        case CLEAVE_ACT_GELU: return z * normal_cdf(z).x;
        case CLEAVE_ACT_GELU_TANH: return z * gelu_tanh_gate(z);
        case CLEAVE_ACT_SILU: return z * silu_gate(z);
        default: return z;
    }
}
// value and slope at once
__device__ __forceinline__ float2 act_value_slope(float z, uint32_t act) {
    switch (act) {
        case CLEAVE_ACT_RELU: return make_float2(z > 0.f ? z : (z != z ? z : 0.f), z > 0.f ? 1.f : 0.f);
        case CLEAVE_ACT_GELU: {
            const float2 n = normal_cdf(z);
            return make_float2(z * n.x, fmaf(z * n.y, 0.3989422804014327f, n.x));
        }
        case CLEAVE_ACT_GELU_TANH: {
            const float g = gelu_tanh_gate(z), zg = z * g;
            const float du = fmaf(0.21406444881780074f, fminf(z * z, 1e30f), 1.5957691216057308f);      // finite: 0 * du is 0 far out
            return make_float2(zg, fmaf(zg * (1.f - g), du, g));
        }
        case CLEAVE_ACT_SILU: {
            const float g = silu_gate(z), zg = z * g;
            return make_float2(zg, fmaf(zg, 1.f - g, g));
        }
        default: return make_float2(z, 1.f);
    }
}

// ---- AdamW -----------------------------------------------------------------------------------------
struct AdamTensor {                 // device record of one tensor
    uint64_t numel;
    float* p;
    __nv_bfloat16* w;
    const void* g;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    double weight_decay;
    uint32_t wide;                  // every buffer allows the wide accesses
    uint32_t pad;
};
struct AdamStep {
    float beta1, omb1, beta2, omb2; // omb = 1 - beta, formed in 64 bits
    float step_size, root, eps, grad_scale;
    double lr;
    uint64_t base;                  // seed + (step << 32)
};
struct AdamChunk { uint32_t tensor, block0; };   // a CTA's blocks of 256 elements, from block0 on
constexpr uint32_t kChunkWarps = 8, kChunkMost = 32;     // warps of a CTA; blocks a warp takes at most
cudaError_t launch_adamw(const AdamTensor* tensors, const AdamChunk* chunks, uint32_t n_chunks, uint32_t chunk_blocks, const AdamStep& s,
                         bool state8, bool g_bf16, cudaStream_t st);

// ---- norm, rows in 8 bits, epilogue backward ---------------------------------------------------------
cudaError_t launch_rmsnorm(const cleave_rmsnorm_t& d, bool norm, int sms, cudaStream_t st);   // sms: the device's SM count
// Rows of partial sums in the workspace: as many as keep kPartSms SMs busy.  A constant, a B200's number of SMs, because the
// workspace queries ask no device; on another number of SMs the sums only spread a little worse.
constexpr uint32_t kPartSms = 148;
uint32_t rmsnorm_backward_parts(uint64_t rows, uint32_t cols);
cudaError_t launch_rmsnorm_backward(const cleave_rmsnorm_backward_t& d, float* ws, cudaStream_t st);
uint32_t act_backward_parts(uint64_t rows, uint32_t cols);
cudaError_t launch_act_backward(const cleave_act_backward_t& d, float* ws, cudaStream_t st);
cudaError_t launch_sum_parts(const float* ws, uint32_t parts, uint32_t cols, float* out, cudaStream_t st);

// ---- product with an epilogue --------------------------------------------------------------------------
int launch_linear(const cleave_linear_t& d, int sms, cudaStream_t st);           // CLEAVE_* code
int linear_status(cudaStream_t st);
void linear_set_wait_limit_ns(uint64_t ns);

}  // namespace cleave
