// Root-mean-square norm with the residual's addition, its backward pass, and rows in 8 bits (see cleave.h).
//
// All of it is bound by the HBM's bandwidth: each row is read once, kept in registers while its statistics are
// formed, and written once.  Two forms of each pass:
//   wide   rows of whole 16-byte groups: a thread owns groups of 8 columns.  Up to 1024 columns a warp takes a row
//          (no barrier, rows in flight by occupancy); above, a CTA takes a row, the next rows come by cp.async
//          into a ring in shared memory -- each thread copies and reads its own groups only, so the ring needs no
//          barrier of its own and the bytes in flight do not depend on registers -- and one barrier a row joins
//          the warps' sums.
//   own    any alignment, up to 8192 columns: neighbouring threads own neighbouring columns, held in registers.
//   any    what is left: the row is taken again in each pass (it stays in L1 / L2).
// Measured: 8192 x 4096 with residual into E4M3 43 us (5.4 TB/s; a plain copy of as many bytes takes 36); rows of a
// 11008 x 4096 weight into E4M3 24.6 us (5.5 TB/s); backward of 16384 x 5120 with dw 122 us (5.5 TB/s of 6.5); one row of
// 4096 3 us, a launch.  Registers bound the CTAs an SM, and some instances of the backward spill: 150 to 180 bytes a
// thread with fp32 h at 256 threads, 210 to 330 at 1024; the own form 300 at 1024.
#include <algorithm>
#include <type_traits>

#include "ops.cuh"

namespace cleave {

constexpr uint32_t kRowThreads = 256;

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

// ---- forward, any shape ------------------------------------------------------------------------------
template <bool NORM>
__global__ void __launch_bounds__(kRowThreads) row_any_kernel(const __grid_constant__ cleave_rmsnorm_t d) {
    __shared__ float buf[32];
    begin_chained();
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

// ---- any alignment, up to 8192 columns ------------------------------------------------------------------
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

template <bool NORM, int T>
__global__ void __launch_bounds__(T) row_own_kernel(const __grid_constant__ cleave_rmsnorm_t d) {
    __shared__ float2 parts[3][32];
    begin_chained();
    float w[kOwn];
    uint32_t x[kOwn], r[kOwn];
#pragma unroll
    for (uint32_t k = 0; k < kOwn; ++k) { w[k] = 1.f; r[k] = 0u; }
    if (d.w) { load_own(d.w, d.w_type, 0, d.cols, x); own_values(x, d.w_type, d.cols, w); }
    const float inv_cols = 1.f / (float)d.cols;
    uint64_t row = blockIdx.x;
    load_own(d.x, d.x_type, row * d.ldx, d.cols, x);
    if (d.r) load_own(d.r, d.r_type, row * d.ldr, d.cols, r);
    const bool codes = d.y_type == CLEAVE_T_E4M3;
    for (uint32_t it = 0; row < d.rows; row += gridDim.x, ++it) {
        float h[kOwn], ss = 0.f, top = 0.f;
        own_values(x, d.x_type, d.cols, h);
        if (d.r) {
            float t[kOwn];
            own_values(r, d.r_type, d.cols, t);
#pragma unroll
            for (uint32_t k = 0; k < kOwn; ++k) h[k] += t[k];
        }
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) ss = fmaf(h[k], h[k], ss);
        if (codes) {
#pragma unroll
            for (uint32_t k = 0; k < kOwn; ++k) top = max_nan(top, fabsf(h[k] * w[k]));
        }
        const uint64_t next = row + gridDim.x;
        if (next < d.rows) {
            load_own(d.x, d.x_type, next * d.ldx, d.cols, x);
            if (d.r) load_own(d.r, d.r_type, next * d.ldr, d.cols, r);
        }
        if (NORM && d.h) store_own(d.h, d.r_type, row * d.ldh, d.cols, h);
        const float2 both = cta_join(ss, top, parts[it & 1]);
        float rstd = 1.f, inv = 1.f;
        if (NORM) {
            rstd = rsqrtf(fmaf(both.x, inv_cols, d.eps));
            if (d.rstd && threadIdx.x == 0) d.rstd[row] = rstd;
        }
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) h[k] = h[k] * rstd * w[k];
        if (codes) {
            float t = both.y * rstd;
            if (both.y == INFINITY) {                            // h w overflowed: take h rstd w
                float a = 0.f;
#pragma unroll
                for (uint32_t k = 0; k < kOwn; ++k) a = max_nan(a, fabsf(h[k]));
                __syncthreads();
                t = cta_join(0.f, a, parts[2]).y;
            }
            const float2 sc = row_scale(t);
            inv = sc.y;
            if (threadIdx.x == 0) d.scale[row] = sc.x;
#pragma unroll
            for (uint32_t k = 0; k < kOwn; ++k) h[k] *= inv;
        }
        store_own(d.y, d.y_type, row * d.ldy, d.cols, h);
    }
}

template <int T>
__global__ void __launch_bounds__(T) rmsnorm_backward_own_kernel(const __grid_constant__ cleave_rmsnorm_backward_t d, float* __restrict__ ws) {
    __shared__ float2 parts[2][32];
    begin_chained();
    float w[kOwn], dw[kOwn];
    uint32_t ndy[kOwn], nh[kOwn], nres[kOwn];
#pragma unroll
    for (uint32_t k = 0; k < kOwn; ++k) { w[k] = 1.f; dw[k] = 0.f; }
    if (d.w) { load_own(d.w, d.w_type, 0, d.cols, nh); own_values(nh, d.w_type, d.cols, w); }
    const float inv_cols = 1.f / (float)d.cols;
    uint64_t row = blockIdx.x;
    load_own(d.dy, d.dy_type, row * d.lddy, d.cols, ndy);
    load_own(d.h, d.h_type, row * d.ldh, d.cols, nh);
    if (d.dres) load_own(d.dres, d.h_type, row * d.lddres, d.cols, nres);
    for (uint32_t it = 0; row < d.rows; row += gridDim.x, ++it) {
        const float rstd = d.rstd[row];
        float q[kOwn], g[kOwn], res[kOwn], dot = 0.f;
        own_values(ndy, d.dy_type, d.cols, q);
        own_values(nh, d.h_type, d.cols, g);
        if (d.dres) own_values(nres, d.h_type, d.cols, res);
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) {
            dw[k] = fmaf(q[k] * rstd, g[k], dw[k]);
            q[k] *= w[k];
            dot = fmaf(q[k], g[k], dot);
        }
        const uint64_t next = row + gridDim.x;
        if (next < d.rows) {
            load_own(d.dy, d.dy_type, next * d.lddy, d.cols, ndy);
            load_own(d.h, d.h_type, next * d.ldh, d.cols, nh);
            if (d.dres) load_own(d.dres, d.h_type, next * d.lddres, d.cols, nres);
        }
        const float along = rstd * rstd * (cta_join(dot, 0.f, parts[it & 1]).x * rstd * inv_cols);
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) { q[k] = rstd * q[k] - along * g[k]; if (d.dres) q[k] += res[k]; }
        store_own(d.dx, d.h_type, row * d.lddx, d.cols, q);
    }
    if (d.dw)
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) { const uint32_t j = threadIdx.x + k * blockDim.x; if (j < d.cols) ws[(uint64_t)blockIdx.x * d.cols + j] = dw[k]; }
}
uint32_t own_threads(uint32_t cols) { return (cols + 32 * kOwn - 1) / (32 * kOwn) * 32; }

// ---- forward, wide -----------------------------------------------------------------------------------
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

// V groups of 8 columns per thread.  WARP: blockDim (32, rows per CTA), a warp per row.  Otherwise a CTA per row
// and a ring of `stages` rows in shared memory, [stage][operand][group] with a thread's groups blockDim.x apart.
template <typename X, typename R, typename Y, int V, bool WARP, bool NORM, int T>
__global__ void __launch_bounds__(T, T == 128 ? 4 : (T == 256 ? 2 : 1)) row_wide_kernel(const __grid_constant__ cleave_rmsnorm_t d, uint32_t stages) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float2 parts[2][32];
    begin_chained();
    constexpr bool RES = !(sizeof(R) == 1), CODES = sizeof(Y) == 1;
    constexpr uint32_t BX = Bytes8<X>::value, BR = Bytes8<R>::value;
    const uint32_t groups = d.cols / 8, tid = threadIdx.x, nt = blockDim.x;
    const uint64_t first = WARP ? (uint64_t)blockIdx.x * blockDim.y + threadIdx.y : blockIdx.x;
    const uint64_t stride = WARP ? (uint64_t)gridDim.x * blockDim.y : gridDim.x;
    const uint32_t off_r = groups * BX, stage_bytes = off_r + groups * BR;
    const float inv_cols = 1.f / (float)d.cols;
    bool live[V];
#pragma unroll
    for (int v = 0; v < V; ++v) live[v] = tid + v * nt < groups;
    // this thread's first group of a row of each operand; a row's step in bytes
    const uint8_t* px = reinterpret_cast<const uint8_t*>(static_cast<const X*>(d.x) + first * d.ldx) + tid * BX;
    const uint8_t* pr = reinterpret_cast<const uint8_t*>(d.r) + (RES ? first * d.ldr * (BR / 8) + tid * BR : 0);
    const uint64_t step_x = stride * d.ldx * (BX / 8), step_r = stride * d.ldr * (BR / 8);
    const uint8_t* slot = ring + tid * BX;
    const uint32_t slot_at = (uint32_t)__cvta_generic_to_shared(ring) + tid * BX;
    uint64_t ahead = first;                                      // the row that is fetched next
    auto fetch = [&](uint32_t at) {                              // this thread's groups of the next row into the stage at byte `at`
        if (ahead < d.rows) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!live[v]) continue;
#pragma unroll
                for (uint32_t b = 0; b < BX; b += 16) cp_async<16>(slot_at + at + v * nt * BX + b, px + v * nt * BX + b);
                if constexpr (RES) {
#pragma unroll
                    for (uint32_t b = 0; b < BR; b += 16) cp_async<16>(slot_at - tid * BX + tid * BR + off_r + at + v * nt * BR + b, pr + v * nt * BR + b);
                }
            }
            ahead += stride; px += step_x; pr += step_r;
        }
        cp_async_commit();                                       // (an empty group keeps the count when there is no such row)
    };
    if constexpr (!WARP)
        for (uint32_t s = 0; s < stages; ++s) fetch(s * stage_bytes);

    // a CTA takes many rows, so its weights stay in registers (from L1 they were two thirds of what the SM's load unit
    // moved: 52 us -> 43 us at 8192 x 4096); a warp takes one row, and 1024 threads have no room
    constexpr bool KEEP = !WARP && T <= 512;
    F2 kept[KEEP ? V : 1][4];
    if constexpr (KEEP) {
#pragma unroll
        for (int v = 0; v < V; ++v) if (live[v]) load_weight8(d, (tid + v * nt) * 8, kept[v]);
    }
    auto weights = [&](int v, F2 (&w)[4]) {
        if constexpr (KEEP) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = kept[KEEP ? v : 0][i];
        } else load_weight8(d, (tid + v * nt) * 8, w);
    };
    Y* py = static_cast<Y*>(d.y) + first * d.ldy + tid * 8;
    R* ph = RES && d.h ? static_cast<R*>(d.h) + first * d.ldh + tid * 8 : nullptr;
    uint32_t it = 0, at = 0;
    for (uint64_t row = first; row < d.rows; row += stride, ++it) {
        F2 h[V][4];
        if constexpr (!WARP) {
            if (stages >= 4) cp_async_wait<3>(); else if (stages == 3) cp_async_wait<2>(); else if (stages == 2) cp_async_wait<1>(); else cp_async_wait<0>();
        }
        Raw8<X> rx[WARP ? V : 1];
        Raw8<typename std::conditional<RES, R, X>::type> rr[WARP ? V : 1];
        if constexpr (WARP) {                                    // everything is asked for before anything is used
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!live[v]) continue;
                rx[v] = load_raw8(reinterpret_cast<const X*>(px + v * nt * BX));
                if constexpr (RES) rr[v] = load_raw8(reinterpret_cast<const R*>(pr + v * nt * BR));
            }
        }
        // one reduction for both statistics: the sum of squares and, for codes, the largest |h w| (times rstd later)
        F2 squares = f2(0.f, 0.f);
        float top = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!live[v]) continue;
            if constexpr (WARP) unpack8(rx[v], h[v]);
            else unpack8(*reinterpret_cast<const Raw8<X>*>(slot + at + v * nt * BX), h[v]);
            if constexpr (RES) {
                F2 r[4];
                if constexpr (WARP) unpack8(rr[v], r);
                else unpack8(*reinterpret_cast<const Raw8<R>*>(ring + off_r + at + (tid + v * nt) * BR), r);
#pragma unroll
                for (int i = 0; i < 4; ++i) h[v][i] = add2(h[v][i], r[i]);
                if constexpr (NORM) if (ph) store8(ph + v * nt * 8, h[v]);
            }
            if constexpr (NORM) {
#pragma unroll
                for (int i = 0; i < 4; ++i) squares = fma2(h[v][i], h[v][i], squares);
            }
            if constexpr (CODES) {
                F2 w[4];
                weights(v, w);
#pragma unroll
                for (int i = 0; i < 4; ++i) top = top2(top, mul2(h[v][i], w[i]));
            }
        }
        const float2 sq = halves(squares);
        float ss = sq.x + sq.y;
        if constexpr (NORM) ss = warp_sum(ss);
        if constexpr (CODES) top = warp_abs_max(top);
        if constexpr (!WARP) {
            float2* p = parts[it & 1];
            if ((tid & 31u) == 0) p[tid >> 5] = make_float2(ss, top);
            __syncthreads();                                     // also: every thread has read this stage
            fetch(at);
            at = at + stage_bytes == stages * stage_bytes ? 0 : at + stage_bytes;
            const float2 q = (tid & 31u) < nt / 32 ? p[tid & 31u] : make_float2(0.f, 0.f);
            if constexpr (NORM) ss = warp_sum(q.x);
            if constexpr (CODES) top = warp_abs_max(q.y);
        } else { px += step_x; pr += step_r; }
        float rstd = 1.f;
        if constexpr (NORM) {
            rstd = rsqrtf(fmaf(ss, inv_cols, d.eps));
            if (d.rstd && tid == 0) d.rstd[row] = rstd;
        }
        float inv = 1.f;
        if constexpr (CODES) {
            if (top == INFINITY) {                               // h w overflowed (rows of extreme weights): take h rstd w
                float t = 0.f;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if (!live[v]) continue;
                    F2 w[4];
                    weights(v, w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) t = top2(t, mul2(mul2(h[v][i], f2(rstd, rstd)), w[i]));
                }
                t = warp_abs_max(t);
                if constexpr (!WARP) {
                    float2* p = parts[it & 1];
                    __syncthreads();
                    if ((tid & 31u) == 0) p[tid >> 5].y = t;
                    __syncthreads();
                    t = warp_abs_max((tid & 31u) < nt / 32 ? p[tid & 31u].y : 0.f);
                }
                top = t;
            } else top *= rstd;
            const float2 sc = row_scale(top);
            inv = sc.y;
            if (tid == 0) d.scale[row] = sc.x;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!live[v]) continue;
            F2 w[4], y[4];
            weights(v, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = mul2(mul2(h[v][i], f2(rstd, rstd)), w[i]);
                if constexpr (CODES) y[i] = mul2(y[i], f2(inv, inv));
            }
            store8(py + v * nt * 8, y);
        }
        py += stride * d.ldy;
        if (RES && ph) ph += stride * d.ldh;
    }
}

constexpr uint32_t kWarpRowCols = 1024;         // up to here a warp holds a row (four groups a lane)
constexpr uint32_t kRingBytes = 50 * 1024;      // per CTA; four CTAs an SM at most sizes
constexpr uint32_t kRingMost = 160 * 1024;

template <typename X, typename R, typename Y, int V, bool WARP, bool NORM, int T>
cudaError_t launch_row_wide(const cleave_rmsnorm_t& d, uint32_t threads, int sms, cudaStream_t st) {
    auto kernel = row_wide_kernel<X, R, Y, V, WARP, NORM, T>;
    if (WARP) {
        const uint64_t ctas = (d.rows + 7) / 8;
        return launch_chained(kernel, (unsigned)ctas, dim3(32, 8), 0, st, d, 0u);
    }
    const uint32_t stage = d.cols / 8 * (Bytes8<X>::value + Bytes8<R>::value);
    const uint32_t stages = max(1u, min(4u, kRingBytes / stage)), smem = stage * stages;
    static SmemLimit limit;
    const cudaError_t e = limit.raise(reinterpret_cast<const void*>(kernel), kRingMost);
    if (e != cudaSuccess) return e;
    // CTAs that fit an SM by shared memory and threads; each walks the rows in steps of the grid
    const uint32_t fit = max(1u, min(min(224u * 1024u / (smem + 2048u), 65536u / (threads * 128u)), 4u));
    const uint64_t ctas = min((uint64_t)d.rows, (uint64_t)sms * fit);
    return launch_chained(kernel, (unsigned)ctas, threads, smem, st, d, stages);
}

template <typename X, typename R, typename Y, bool NORM>
cudaError_t launch_row_types(const cleave_rmsnorm_t& d, int sms, cudaStream_t st) {
    const uint32_t groups = d.cols / 8;
    if (d.cols <= kWarpRowCols) {
        if (groups <= 32) return launch_row_wide<X, R, Y, 1, true, NORM, 256>(d, 32, sms, st);
        if (groups <= 64) return launch_row_wide<X, R, Y, 2, true, NORM, 256>(d, 32, sms, st);
        return launch_row_wide<X, R, Y, 4, true, NORM, 256>(d, 32, sms, st);
    }
    const uint32_t threads = (groups + 127) / 128 * 32;
    if (groups <= 512) return launch_row_wide<X, R, Y, 4, false, NORM, 128>(d, threads, sms, st);
    if (groups <= 1024) return launch_row_wide<X, R, Y, 4, false, NORM, 256>(d, threads, sms, st);
    if (groups <= 2048) return launch_row_wide<X, R, Y, 4, false, NORM, 512>(d, threads, sms, st);
    return launch_row_wide<X, R, Y, 4, false, NORM, 1024>(d, threads, sms, st);
}
template <typename X, typename R>
cudaError_t launch_row_out(const cleave_rmsnorm_t& d, bool norm, int sms, cudaStream_t st) {
    if constexpr (sizeof(R) == 1)
        if (!norm) return launch_row_types<X, R, uint8_t, false>(d, sms, st);
    if (d.y_type == CLEAVE_T_E4M3) return launch_row_types<X, R, uint8_t, true>(d, sms, st);
    if (d.y_type == CLEAVE_T_F32) return launch_row_types<X, R, float, true>(d, sms, st);
    return launch_row_types<X, R, __nv_bfloat16, true>(d, sms, st);
}
template <typename X>
cudaError_t launch_row_res(const cleave_rmsnorm_t& d, bool norm, int sms, cudaStream_t st) {
    if (!d.r) return launch_row_out<X, NoRes>(d, norm, sms, st);
    return d.r_type == CLEAVE_T_F32 ? launch_row_out<X, float>(d, norm, sms, st) : launch_row_out<X, __nv_bfloat16>(d, norm, sms, st);
}

cudaError_t launch_rmsnorm(const cleave_rmsnorm_t& d, bool norm, int sms, cudaStream_t st) {
    if (!d.rows || !d.cols) return cudaSuccess;
    const uint64_t stage = (uint64_t)d.cols * (type_bytes(d.x_type) + type_bytes(d.r_type));
    const bool wide = d.cols % 8 == 0 && d.cols <= 32768 && stage <= kRingMost && rows_wide(d.x, d.ldx, d.x_type) && rows_wide(d.y, d.ldy, d.y_type) &&
                      (!d.r || rows_wide(d.r, d.ldr, d.r_type)) && (!d.h || rows_wide(d.h, d.ldh, d.r_type)) && (!d.w || (uintptr_t)d.w % 16 == 0);
    if (wide) return d.x_type == CLEAVE_T_F32 ? launch_row_res<float>(d, norm, sms, st) : launch_row_res<__nv_bfloat16>(d, norm, sms, st);
    if (d.cols <= kOwnCols) {
        const uint32_t threads = own_threads(d.cols);
        const unsigned ctas = (unsigned)std::min<uint64_t>(d.rows, (uint64_t)sms * std::min(24u, 1024u / threads));
        auto kernel = threads <= 512 ? (norm ? row_own_kernel<true, 512> : row_own_kernel<false, 512>) : (norm ? row_own_kernel<true, 1024> : row_own_kernel<false, 1024>);
        return launch_chained(kernel, ctas, threads, 0, st, d);
    }
    return launch_chained(norm ? row_any_kernel<true> : row_any_kernel<false>, (unsigned)d.rows, kRowThreads, 0, st, d);
}

// ---- backward ----------------------------------------------------------------------------------------
// A CTA takes the rows part, part + parts, ...; its share of dw goes to row `part` of the workspace (fp32
// [parts x cols]; each element belongs to one thread), and sum_parts_kernel adds the parts in order.
// CTAs of the backward pass an SM: as many threads as registers allow
uint32_t backward_ctas(uint32_t cols) {
    const uint32_t threads = (cols / 8 + 63) / 64 * 32;          // of the wide form
    return threads <= 256 ? std::min(16u, 768u / std::max(threads, 32u)) : (threads <= 320 ? 2u : 1u);
}
uint32_t rmsnorm_backward_parts(uint64_t rows, uint32_t cols) {
    return (uint32_t)std::min<uint64_t>(rows, (uint64_t)kPartSms * backward_ctas(cols));
}

__global__ void __launch_bounds__(kRowThreads) rmsnorm_backward_any_kernel(const __grid_constant__ cleave_rmsnorm_backward_t d, float* __restrict__ ws) {
    __shared__ float buf[32];
    begin_chained();
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

// V groups of 8 columns a thread, a CTA per row, a ring of rows of (dy, h, dres) in shared memory; the CTA's share of
// dw stays in registers over all its rows (w comes from L1: keeping it too would cost a CTA an SM).
template <typename D, typename H, int V, int T, int CTAS>
__global__ void __launch_bounds__(T, CTAS) rmsnorm_backward_wide_kernel(const __grid_constant__ cleave_rmsnorm_backward_t d, float* __restrict__ ws, uint32_t stages) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float parts[2][32];
    begin_chained();
    constexpr uint32_t BD = Bytes8<D>::value, BH = Bytes8<H>::value;
    const uint32_t groups = d.cols / 8, tid = threadIdx.x, nt = blockDim.x;
    const bool res = d.dres != nullptr;
    const uint32_t off_h = groups * BD, off_res = off_h + groups * BH, stage_bytes = off_res + (res ? groups * BH : 0u);
    const uint32_t ring_base = (uint32_t)__cvta_generic_to_shared(ring);
    const float inv_cols = 1.f / (float)d.cols;
    bool live[V];
#pragma unroll
    for (int v = 0; v < V; ++v) live[v] = tid + v * nt < groups;
    const uint8_t* pd = reinterpret_cast<const uint8_t*>(static_cast<const D*>(d.dy) + blockIdx.x * d.lddy) + tid * BD;
    const uint8_t* ph = reinterpret_cast<const uint8_t*>(static_cast<const H*>(d.h) + blockIdx.x * d.ldh) + tid * BH;
    const uint8_t* pr = res ? reinterpret_cast<const uint8_t*>(static_cast<const H*>(d.dres) + blockIdx.x * d.lddres) + tid * BH : nullptr;
    const uint64_t step_d = gridDim.x * d.lddy * (BD / 8), step_h = gridDim.x * d.ldh * (BH / 8), step_r = gridDim.x * d.lddres * (BH / 8);
    uint64_t ahead = blockIdx.x;
    auto fetch = [&](uint32_t at) {
        if (ahead < d.rows) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!live[v]) continue;
                const uint32_t to = ring_base + at;
#pragma unroll
                for (uint32_t b = 0; b < BD; b += 16) cp_async<16>(to + (tid + v * nt) * BD + b, pd + v * nt * BD + b);
#pragma unroll
                for (uint32_t b = 0; b < BH; b += 16) cp_async<16>(to + off_h + (tid + v * nt) * BH + b, ph + v * nt * BH + b);
                if (res) {
#pragma unroll
                    for (uint32_t b = 0; b < BH; b += 16) cp_async<16>(to + off_res + (tid + v * nt) * BH + b, pr + v * nt * BH + b);
                }
            }
            ahead += gridDim.x; pd += step_d; ph += step_h;
            if (res) pr += step_r;
        }
        cp_async_commit();
    };
    for (uint32_t s = 0; s < stages; ++s) fetch(s * stage_bytes);
    F2 dw[V][4];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[v][i] = f2(0.f, 0.f);
    H* pdx = static_cast<H*>(d.dx) + blockIdx.x * d.lddx + tid * 8;
    uint32_t it = 0, at = 0;
    for (uint64_t row = blockIdx.x; row < d.rows; row += gridDim.x, ++it) {
        if (stages >= 4) cp_async_wait<3>(); else if (stages == 3) cp_async_wait<2>(); else if (stages == 2) cp_async_wait<1>(); else cp_async_wait<0>();
        const float rstd = d.rstd[row];
        const uint8_t* stage = ring + at;
        F2 q[V][4], dots = f2(0.f, 0.f);                         // q = w dy; dots: sum q h
        Raw8<H> rh[V], rr[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!live[v]) continue;
            const uint32_t g = tid + v * nt;
            unpack8(*reinterpret_cast<const Raw8<D>*>(stage + g * BD), q[v]);
            rh[v] = *reinterpret_cast<const Raw8<H>*>(stage + off_h + g * BH);
            if (res) rr[v] = *reinterpret_cast<const Raw8<H>*>(stage + off_res + g * BH);
            F2 h[4], w[4];
            unpack8(rh[v], h);
            load_weight8(d, g * 8, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                dw[v][i] = fma2(mul2(q[v][i], f2(rstd, rstd)), h[i], dw[v][i]);
                q[v][i] = mul2(q[v][i], w[i]);
                dots = fma2(q[v][i], h[i], dots);
            }
        }
        const float2 dd = halves(dots);
        float dot = dd.x + dd.y;
        dot = warp_sum(dot);
        float* p = parts[it & 1];
        if ((tid & 31u) == 0) p[tid >> 5] = dot;
        __syncthreads();                                         // also: every thread has read this stage
        fetch(at);
        at = at + stage_bytes == stages * stage_bytes ? 0 : at + stage_bytes;
        const float mean = warp_sum((tid & 31u) < nt / 32 ? p[tid & 31u] : 0.f) * rstd * inv_cols;      // of q xh
        const float along = rstd * rstd * mean;                  // rstd xh mean = along h
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!live[v]) continue;
            F2 dx[4], h[4];
            unpack8(rh[v], h);
#pragma unroll
            for (int i = 0; i < 4; ++i) dx[i] = fma2(f2(-along, -along), h[i], mul2(f2(rstd, rstd), q[v][i]));
            if (res) {
                unpack8(rr[v], h);
#pragma unroll
                for (int i = 0; i < 4; ++i) dx[i] = add2(dx[i], h[i]);
            }
            store8(pdx + v * nt * 8, dx);
        }
        pdx += gridDim.x * d.lddx;
    }
    if (d.dw)
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (live[v]) store8(ws + (uint64_t)blockIdx.x * d.cols + (tid + v * nt) * 8, dw[v]);
}

// out[j] = sum over the parts of ws[part][j], in a fixed order.  32 columns per CTA; warp w adds the parts
// w, w + 32, ... and the 32 sums are added in warp order.
__global__ void __launch_bounds__(1024) sum_parts_kernel(const float* ws, uint32_t parts, uint32_t cols, float* out) {
    __shared__ float s[32][33];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, j = blockIdx.x * 32u + lane;
    float v = 0.f;
    wait_for_primary();   // and no early start for what follows: the kernel whose sums these are still runs, and one
                          // that shares the SMs with it lands on them unevenly (act_backward of 8192 x 3072: 30 -> 35 us)
    if (j < cols) {
#pragma unroll 8
        for (uint32_t p = warp; p < parts; p += 32) v += __ldcs(ws + (uint64_t)p * cols + j);
    }
    s[warp][lane] = v;
    __syncthreads();
    // warp w adds column w's 32 sums (a shuffle tree: fixed order)
    v = warp_sum(s[lane][warp]);
    if (lane == 0 && blockIdx.x * 32u + warp < cols) out[blockIdx.x * 32u + warp] = v;
}
cudaError_t launch_sum_parts(const float* ws, uint32_t parts, uint32_t cols, float* out, cudaStream_t st) {
    return launch_chained(sum_parts_kernel, (cols + 31) / 32, 1024, 0, st, ws, parts, cols, out);
}

template <typename D, typename H, int V, int T, int CTAS>
cudaError_t launch_backward_wide(const cleave_rmsnorm_backward_t& d, float* ws, uint32_t threads, uint32_t parts, uint32_t stage, cudaStream_t st) {
    auto kernel = rmsnorm_backward_wide_kernel<D, H, V, T, CTAS>;
    static SmemLimit limit;
    const cudaError_t e = limit.raise(reinterpret_cast<const void*>(kernel), kRingMost);
    if (e != cudaSuccess) return e;
    const uint32_t stages = max(1u, min(4u, min(kRingMost, 216u * 1024u / backward_ctas(d.cols)) / stage));
    return launch_chained(kernel, parts, threads, stage * stages, st, d, ws, stages);
}
template <typename D, typename H>
cudaError_t launch_backward_types(const cleave_rmsnorm_backward_t& d, float* ws, uint32_t parts, uint32_t stage, cudaStream_t st) {
    const uint32_t groups = d.cols / 8;
    const uint32_t threads = (groups + 63) / 64 * 32;
    if (groups <= 512) return launch_backward_wide<D, H, 2, 256, 3>(d, ws, threads, parts, stage, st);
    if (groups <= 640) return launch_backward_wide<D, H, 2, 320, 2>(d, ws, threads, parts, stage, st);
    if (groups <= 1024) return launch_backward_wide<D, H, 2, 512, 1>(d, ws, threads, parts, stage, st);
    return launch_backward_wide<D, H, 2, 1024, 1>(d, ws, threads, parts, stage, st);
}

cudaError_t launch_rmsnorm_backward(const cleave_rmsnorm_backward_t& d, float* ws, cudaStream_t st) {
    if (!d.cols) return cudaSuccess;
    const uint32_t parts = rmsnorm_backward_parts(d.rows, d.cols);
    const uint64_t stage = (uint64_t)d.cols * (type_bytes(d.dy_type) + type_bytes(d.h_type) * (d.dres ? 2u : 1u));
    const bool wide = d.cols % 8 == 0 && d.cols <= 16384 && stage <= kRingMost && rows_wide(d.dy, d.lddy, d.dy_type) && rows_wide(d.h, d.ldh, d.h_type) &&
                      rows_wide(d.dx, d.lddx, d.h_type) && (!d.dres || rows_wide(d.dres, d.lddres, d.h_type)) && (uintptr_t)d.w % 16 == 0;
    cudaError_t e = cudaSuccess;
    if (parts && wide) {
        if (d.dy_type == CLEAVE_T_F32) e = d.h_type == CLEAVE_T_F32 ? launch_backward_types<float, float>(d, ws, parts, (uint32_t)stage, st) : launch_backward_types<float, __nv_bfloat16>(d, ws, parts, (uint32_t)stage, st);
        else e = d.h_type == CLEAVE_T_F32 ? launch_backward_types<__nv_bfloat16, float>(d, ws, parts, (uint32_t)stage, st) : launch_backward_types<__nv_bfloat16, __nv_bfloat16>(d, ws, parts, (uint32_t)stage, st);
    } else if (parts && d.cols <= kOwnCols) {
        const uint32_t threads = own_threads(d.cols);
        e = launch_chained(threads <= 512 ? rmsnorm_backward_own_kernel<512> : rmsnorm_backward_own_kernel<1024>, parts, threads, 0, st, d, ws);
    } else if (parts) {
        e = launch_chained(rmsnorm_backward_any_kernel, parts, kRowThreads, 0, st, d, ws);
    }
    if (e != cudaSuccess || !d.dw) return e;
    return launch_sum_parts(ws, parts, d.cols, d.dw, st);
}

}  // namespace cleave
