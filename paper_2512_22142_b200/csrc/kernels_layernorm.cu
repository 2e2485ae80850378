// Layer norm with the residual's addition, and its backward pass (see cleave.h).
//
// Bound by the HBM's bandwidth: each row is read once, kept in registers while its mean and then its variance (the sum of the
// squared differences to that mean) are formed, and written once.  Forms as in the root-mean-square norm:
//   wide   rows whose 16-byte lines begin at the same columns in all operands: a thread owns groups of 8 columns.  Up to 1024 columns a warp takes a row; above, a CTA
//          takes a row.  The next rows come by cp.async into a ring in shared memory: each thread copies and reads its own groups
//          only, so the ring needs no barrier of its own and the bytes in flight do not depend on registers.
//   own    operands that disagree, and short rows, up to 8192 columns: neighbouring threads own neighbouring columns, held in registers.
//   any    what is left: the row is taken again in each pass (it stays in L1 / L2).
// Measured: 8192 x 768 with an fp32 residual 15.4 us (4.9 TB/s: 75 MB are read and written in the time of few rows a warp), 8192 x 8192 with a bf16 residual
// into E4M3 81 to 87 us (5.4 to 5.8 TB/s), one row of 4096 a launch, 4.4 us with the call; backward of 16384 x 5120 with dw and db 123 to 130 us
// (5.2 to 5.4 TB/s, the sums of the CTAs' shares among them), with an fp32 h and bf16 dy 282 us (4.2 TB/s).  Rows of odd length: 1899 x 8962 fp32 with a residual
// 64 us (4.2 TB/s), backward of 12216 x 3349 bf16 90 us (3.6 TB/s).
#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "rows.cuh"
#include "tokens.cuh"

namespace cleave {

// 8 of a vector of weights or biases of columns, or `fill` where there is none
__device__ __forceinline__ void load_vector8(const void* p, uint32_t type, uint32_t col, float fill, F2 (&v)[4]) {
    if (type != CLEAVE_T_NONE && (((uintptr_t)p + (uint64_t)col * (type == CLEAVE_T_F32 ? 4 : 2)) & 15u)) {       // not on 16 bytes
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = f2(load_as(p, type, col + 2 * i), load_as(p, type, col + 2 * i + 1));
    } else if (type == CLEAVE_T_F32) {
        Raw8<float> r;
        const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + col);
        r.w[0] = q[0]; r.w[1] = q[1];
        unpack8(r, v);
    } else if (type == CLEAVE_T_BF16) {
        Raw8<__nv_bfloat16> r;
        r.w[0] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + col);
        unpack8(r, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = f2(fill, fill);
    }
}
// the same of all of a thread's groups, at the columns col, col + step, ...: every load is asked for before any is unpacked
// (a choice of type group by group let each group's loads wait for the one's before: 8192 x 768 17.2 us in place of 15.4)
template <int V>
__device__ __forceinline__ void load_vectors8(const void* p, uint32_t type, uint32_t col, uint32_t step, const bool (&live)[V], float fill, F2 (&x)[V][4]) {
    if (type == CLEAVE_T_NONE) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[v][i] = f2(fill, fill);
    } else if (((uintptr_t)p + (uint64_t)col * (type == CLEAVE_T_F32 ? 4 : 2)) & 15u) {
#pragma unroll
        for (int v = 0; v < V; ++v) if (live[v]) load_vector8(p, type, col + v * step, fill, x[v]);
    } else if (type == CLEAVE_T_F32) {
        Raw8<float> r[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (live[v]) { const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + col + v * step); r[v].w[0] = q[0]; r[v].w[1] = q[1]; }
#pragma unroll
        for (int v = 0; v < V; ++v) unpack8(r[v], x[v]);
    } else {
        Raw8<__nv_bfloat16> r[V];
#pragma unroll
        for (int v = 0; v < V; ++v) if (live[v]) r[v].w[0] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + col + v * step);
#pragma unroll
        for (int v = 0; v < V; ++v) unpack8(r[v], x[v]);
    }
}
__device__ __forceinline__ float sum_of(F2 a) { const float2 h = halves(a); return h.x + h.y; }

// 1 / n in two parts: the mean of n values is sum first + sum rest, rounded once.  (With the first part alone a row of ones would not have the mean 1
// for one length in seven, and a constant row y = bias; a division's branch costs more: backward of 16384 x 5120 126 -> 132 us, 1899 x 8962 fp32 65 -> 69.)
struct Reciprocal {
    float first, rest;
    __device__ __forceinline__ explicit Reciprocal(uint32_t n) : first(1.f / (float)n), rest(fmaf(-first, (float)n, 1.f) * first) {}
    __device__ __forceinline__ float mean(float sum) const {
        const float plain = sum * first;
        return fabsf(sum) < INFINITY ? fmaf(sum, first, sum * rest) : plain;
    }
};

// Where the 16-byte lines of a row begin: column (unit - (at + row step) % unit) % unit, alike in all operands.  Rows of one length that
// lie side by side (or at one distance) in all of them agree whatever that length is; what is before the first line and behind the
// last whole group of 8 columns, less than 8 each, goes to single threads.
struct Lines {
    uint32_t at, step, unit;
    __device__ __forceinline__ uint32_t head(uint64_t row, uint32_t cols) const { return min(cols, (unit - (at + (uint32_t)(row % unit) * step) % unit) % unit); }
};
struct Operand { const void* p; uint64_t ld; uint32_t type; };
static bool lines_agree(std::initializer_list<Operand> operands, Lines& lines) {
    lines = {0, 0, 0};
    for (const bool narrow : {true, false})                      // operands of 1 or 2 bytes say more than those of 4
        for (const Operand& o : operands)
            if (o.p && !lines.unit && narrow == (o.type != CLEAVE_T_F32)) {
                lines.unit = narrow ? 8 : 4;
                lines.at = (uint32_t)((uintptr_t)o.p / type_bytes(o.type) % lines.unit);
                lines.step = (uint32_t)(o.ld % lines.unit);
            }
    for (const Operand& o : operands) {
        if (!o.p) continue;
        const uint32_t unit = o.type == CLEAVE_T_F32 ? 4 : 8;
        if (((uintptr_t)o.p / type_bytes(o.type) - lines.at) % unit || (o.ld - lines.step) % unit) return false;
    }
    return true;
}
// the column that thread `tid` of a row has to itself, or none (`cols`)
__device__ __forceinline__ uint32_t edge_column(uint32_t tid, uint32_t head, uint32_t tail, uint32_t cols) {
    if (tid < head) return tid;
    return tid >= 8u && tid - 8u < tail ? cols - tail + (tid - 8u) : cols;
}
template <typename T> __device__ __forceinline__ void store_one(T* p, float v) { *p = from_f32<T>(v); }
__device__ __forceinline__ void store_one(uint8_t* p, float v) { *p = e4m3_nearest(v); }

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

// ---- forward, a row held by its CTA -------------------------------------------------------------------------
template <int T>
__global__ void __launch_bounds__(T) layernorm_own_kernel(const __grid_constant__ cleave_layernorm_t d) {
    __shared__ float2 parts[3][32];
    begin_chained();
    float w[kOwn], b[kOwn];
    uint32_t x[kOwn], r[kOwn];
#pragma unroll
    for (uint32_t k = 0; k < kOwn; ++k) { w[k] = 1.f; b[k] = 0.f; r[k] = 0u; }
    if (d.w) { load_own(d.w, d.w_type, 0, d.cols, x); own_values(x, d.w_type, d.cols, w); }
    if (d.b) { load_own(d.b, d.b_type, 0, d.cols, x); own_values(x, d.b_type, d.cols, b); }
    const Reciprocal inv_cols(d.cols);
    uint64_t row = blockIdx.x;
    load_own(d.x, d.x_type, row * d.ldx, d.cols, x);
    if (d.r) load_own(d.r, d.r_type, row * d.ldr, d.cols, r);
    for (; row < d.rows; row += gridDim.x) {
        float h[kOwn], s = 0.f, ss = 0.f, top = 0.f;
        own_values(x, d.x_type, d.cols, h);
        if (d.r) {
            float t[kOwn];
            own_values(r, d.r_type, d.cols, t);
#pragma unroll
            for (uint32_t k = 0; k < kOwn; ++k) h[k] += t[k];
        }
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) s += h[k];
        const uint64_t next = row + gridDim.x;
        if (next < d.rows) {
            load_own(d.x, d.x_type, next * d.ldx, d.cols, x);
            if (d.r) load_own(d.r, d.r_type, next * d.ldr, d.cols, r);
        }
        if (d.h) store_own(d.h, d.r_type, row * d.ldh, d.cols, h);
        const float mean = inv_cols.mean(cta_join(s, 0.f, parts[0]).x);
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) {
            h[k] = threadIdx.x + k * blockDim.x < d.cols ? h[k] - mean : 0.f;
            ss = fmaf(h[k], h[k], ss);
        }
        const float rstd = rsqrtf(fmaf(cta_join(ss, 0.f, parts[1]).x, inv_cols.first, d.eps));
        if (threadIdx.x == 0) {
            if (d.mean) d.mean[row] = mean;
            if (d.rstd) d.rstd[row] = rstd;
        }
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) { h[k] = fmaf(h[k] * rstd, w[k], b[k]); top = max_nan(top, fabsf(h[k])); }       // (columns that do not exist: 0)
        if (d.y_type == CLEAVE_T_E4M3) {
            const float2 sc = row_scale(cta_join(0.f, top, parts[2]).y);
            if (threadIdx.x == 0) d.scale[row] = sc.x;
#pragma unroll
            for (uint32_t k = 0; k < kOwn; ++k) h[k] *= sc.y;
        }
        store_own(d.y, d.y_type, row * d.ldy, d.cols, h);
    }
}

// ---- forward, wide -----------------------------------------------------------------------------------
// V groups of 8 columns per thread.  WARP: blockDim (32, 8), a warp per row; otherwise a CTA per row.  A row has a ring of `stages` of the
// next ones in shared memory, [stage][operand][group] with a thread's groups blockDim.x apart, and weights and biases stay in registers
// over all rows.  Warps an SM: 24 of two groups, 16 of four (8192 x 8192 with a bf16 residual into E4M3 81 us; with 512 threads of two
// groups 84); 8 warps with a row each, all registers theirs (8192 x 768 15.4 us; with one row ahead 16.8).
// EDGES: rows that do not begin or end with a line (their threads hold more: 8192 x 2048 bf16 33 us in place of 26).
constexpr int row_warps(int V) { return V <= 2 ? 24 : 16; }
template <typename X, typename R, typename Y, int V, bool WARP, int T, bool EDGES>
__global__ void __launch_bounds__(T, WARP ? 1 : row_warps(V) * 32 / T) layernorm_wide_kernel(const __grid_constant__ cleave_layernorm_t d, uint32_t stages, const Lines lines) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float parts[3][32];
    begin_chained();
    constexpr bool RES = !(sizeof(R) == 1), CODES = sizeof(Y) == 1;
    constexpr uint32_t BX = Bytes8<X>::value, BR = Bytes8<R>::value;
    const uint32_t tid = threadIdx.x, nt = blockDim.x;
    const uint64_t first = WARP ? (uint64_t)blockIdx.x * blockDim.y + threadIdx.y : blockIdx.x;
    const uint64_t stride = WARP ? (uint64_t)gridDim.x * blockDim.y : gridDim.x;         // (whole units of rows where rows differ: one head for all)
    const uint32_t head = EDGES ? lines.head(first, d.cols) : 0u, groups = (d.cols - head) / 8, edge = EDGES ? edge_column(tid, head, d.cols - head - groups * 8, d.cols) : d.cols;
    const uint32_t off_r = d.cols / 8 * BX, stage_bytes = off_r + d.cols / 8 * BR;
    const Reciprocal inv_cols(d.cols);
    bool live[V];
#pragma unroll
    for (int v = 0; v < V; ++v) live[v] = tid + v * nt < groups;
    const uint8_t* px = reinterpret_cast<const uint8_t*>(static_cast<const X*>(d.x) + first * d.ldx + head) + tid * BX;
    const uint8_t* pr = reinterpret_cast<const uint8_t*>(d.r) + (RES ? (first * d.ldr + head) * (BR / 8) + tid * BR : 0);
    const uint64_t step_x = stride * d.ldx * (BX / 8), step_r = stride * d.ldr * (BR / 8);
    const uint8_t* mine = ring + (WARP ? threadIdx.y * stages * stage_bytes : 0u);
    const uint32_t slot = (uint32_t)__cvta_generic_to_shared(mine);
    uint64_t ahead = first;                                      // the row that is fetched next
    auto fetch = [&](uint32_t at) {                              // this thread's groups of the next row into the stage at byte `at`
        if (ahead < d.rows) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!live[v]) continue;
#pragma unroll
                for (uint32_t b = 0; b < BX; b += 16) cp_async<16>(slot + at + (tid + v * nt) * BX + b, px + v * nt * BX + b);
                if constexpr (RES) {
#pragma unroll
                    for (uint32_t b = 0; b < BR; b += 16) cp_async<16>(slot + off_r + at + (tid + v * nt) * BR + b, pr + v * nt * BR + b);
                }
            }
            ahead += stride; px += step_x; pr += step_r;
        }
        cp_async_commit();                                       // (an empty group keeps the count when there is no such row)
    };
    for (uint32_t s = 0; s < stages; ++s) fetch(s * stage_bytes);
    F2 w[V][4], b[V][4];
    load_vectors8<V>(d.w, d.w_type, head + tid * 8, nt * 8, live, 1.f, w);
    load_vectors8<V>(d.b, d.b_type, head + tid * 8, nt * 8, live, 0.f, b);
    // the thread's single column: its weight and bias, and the next row's value
    const float edge_w = EDGES && edge < d.cols && d.w ? load_as(d.w, d.w_type, edge) : 1.f, edge_b = EDGES && edge < d.cols && d.b ? load_as(d.b, d.b_type, edge) : 0.f;
    X next_x = from_f32<X>(0.f);                                 // (as it is stored: a conversion would wait for the load)
    typename std::conditional<RES, R, X>::type next_r = from_f32<typename std::conditional<RES, R, X>::type>(0.f);
    auto ask_edge = [&](uint64_t row) {
        if (EDGES && edge < d.cols && row < d.rows) {
            next_x = static_cast<const X*>(d.x)[row * d.ldx + edge];
            if constexpr (RES) next_r = static_cast<const R*>(d.r)[row * d.ldr + edge];
        }
    };
    ask_edge(first);
    auto join = [&](float v, float* p) {                         // sum over the row's threads
        v = warp_sum(v);
        if constexpr (!WARP) {
            if ((tid & 31u) == 0) p[tid >> 5] = v;
            __syncthreads();
            v = warp_sum((tid & 31u) < nt / 32 ? p[tid & 31u] : 0.f);
        }
        return v;
    };
    Y* py = static_cast<Y*>(d.y) + first * d.ldy + head + tid * 8;
    R* ph = RES && d.h ? static_cast<R*>(d.h) + first * d.ldh + head + tid * 8 : nullptr;
    uint32_t at = 0;
    for (uint64_t row = first; row < d.rows; row += stride) {
        F2 h[V][4];
        if (stages >= 4) cp_async_wait<3>(); else if (stages == 3) cp_async_wait<2>(); else if (stages == 2) cp_async_wait<1>(); else cp_async_wait<0>();
        F2 sum = f2(0.f, 0.f), squares = f2(0.f, 0.f);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!live[v]) continue;
            unpack8(*reinterpret_cast<const Raw8<X>*>(mine + at + (tid + v * nt) * BX), h[v]);
            if constexpr (RES) {
                F2 r[4];
                unpack8(*reinterpret_cast<const Raw8<R>*>(mine + off_r + at + (tid + v * nt) * BR), r);
#pragma unroll
                for (int i = 0; i < 4; ++i) h[v][i] = add2(h[v][i], r[i]);
                if (ph) store8(ph + v * nt * 8, h[v]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = add2(sum, h[v][i]);
        }
        float lone = 0.f;
        if (EDGES && edge < d.cols) {
            lone = to_f32(next_x);
            if constexpr (RES) lone += to_f32(next_r);
            if constexpr (RES) if (d.h) store_one(static_cast<R*>(d.h) + row * d.ldh + edge, lone);
            ask_edge(row + stride);
        }
        const float mean = inv_cols.mean(join(sum_of(sum) + lone, parts[0]));
        if (EDGES && edge < d.cols) lone -= mean;
        fetch(at);                                               // (this thread has read its groups of this stage)
        at = at + stage_bytes == stages * stage_bytes ? 0 : at + stage_bytes;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!live[v]) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) { h[v][i] = add2(h[v][i], f2(-mean, -mean)); squares = fma2(h[v][i], h[v][i], squares); }
        }
        const float rstd = rsqrtf(fmaf(join(fmaf(lone, lone, sum_of(squares)), parts[1]), inv_cols.first, d.eps));
        if (tid == 0) {
            if (d.mean) d.mean[row] = mean;
            if (d.rstd) d.rstd[row] = rstd;
        }
        if (EDGES && edge < d.cols) lone = fmaf(lone * rstd, edge_w, edge_b);
        float top = fabsf(lone);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!live[v]) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[v][i] = fma2(mul2(h[v][i], f2(rstd, rstd)), w[v][i], b[v][i]);
                if constexpr (CODES) top = top2(top, h[v][i]);
            }
            if constexpr (!CODES) store8(py + v * nt * 8, h[v]);
        }
        if constexpr (CODES) {
            top = warp_abs_max(top);
            if constexpr (!WARP) {
                if ((tid & 31u) == 0) parts[2][tid >> 5] = top;
                __syncthreads();
                top = warp_abs_max((tid & 31u) < nt / 32 ? parts[2][tid & 31u] : 0.f);
            }
            const float2 sc = row_scale(top);
            if (tid == 0) d.scale[row] = sc.x;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!live[v]) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i) h[v][i] = mul2(h[v][i], f2(sc.y, sc.y));
                store8(py + v * nt * 8, h[v]);
            }
            lone *= sc.y;
        }
        if (EDGES && edge < d.cols) store_one(static_cast<Y*>(d.y) + row * d.ldy + edge, lone);
        py += stride * d.ldy;
        if (RES && ph) ph += stride * d.ldh;
    }
}

constexpr uint32_t kWarpRowCols = 1024;         // up to here a warp holds a row (four groups a lane)
constexpr uint32_t kRingBytes = 64 * 1024;      // per CTA; three CTAs of 256 threads an SM
constexpr uint32_t kRingMost = 208 * 1024;     // of all rings of a CTA
constexpr uint32_t kWarpRing = 26 * 1024;       // of one of a CTA's eight warps

template <typename X, typename R, typename Y, int V, bool WARP, int T, bool EDGES>
cudaError_t launch_wide_edges(const cleave_layernorm_t& d, uint32_t threads, const Lines& lines, int sms, cudaStream_t st) {
    auto kernel = layernorm_wide_kernel<X, R, Y, V, WARP, T, EDGES>;
    const uint32_t stage = d.cols / 8 * (Bytes8<X>::value + Bytes8<R>::value);
    static SmemLimit limit;
    const cudaError_t e = limit.raise(reinterpret_cast<const void*>(kernel), kRingMost);
    if (e != cudaSuccess) return e;
    if (WARP) {                                                  // a ring a warp
        const uint32_t stages = std::max(1u, std::min(4u, kWarpRing / stage));
        return launch_chained(kernel, (unsigned)std::min<uint64_t>((d.rows + 7) / 8, (uint64_t)sms), dim3(32, 8), 8 * stages * stage, st, d, stages, lines);
    }
    const uint32_t stages = std::max(1u, std::min(4u, kRingBytes / stage)), smem = stage * stages;
    // CTAs that fit an SM by shared memory and registers; each walks the rows in steps of the grid
    const uint32_t fit = std::max(1u, std::min(224u * 1024u / (smem + 2048u), (uint32_t)row_warps(V) * 32u / threads));
    uint64_t ctas = (uint64_t)sms * fit;
    if (lines.step) ctas = std::max<uint64_t>(8, ctas / 8 * 8);  // a CTA's rows begin alike
    return launch_chained(kernel, (unsigned)std::min((uint64_t)d.rows, ctas), threads, smem, st, d, stages, lines);
}
template <typename X, typename R, typename Y, int V, bool WARP, int T>
cudaError_t launch_wide(const cleave_layernorm_t& d, uint32_t threads, const Lines& lines, int sms, cudaStream_t st) {
    return lines.at || lines.step || d.cols % 8 ? launch_wide_edges<X, R, Y, V, WARP, T, true>(d, threads, lines, sms, st)
                                                : launch_wide_edges<X, R, Y, V, WARP, T, false>(d, threads, lines, sms, st);
}
template <typename X, typename R, typename Y>
cudaError_t launch_sizes(const cleave_layernorm_t& d, const Lines& lines, int sms, cudaStream_t st) {
    const uint32_t groups = d.cols / 8;
    if (d.cols <= kWarpRowCols) {
        if (groups <= 32) return launch_wide<X, R, Y, 1, true, 256>(d, 32, lines, sms, st);
        if (groups <= 64) return launch_wide<X, R, Y, 2, true, 256>(d, 32, lines, sms, st);
        if (groups <= 96) return launch_wide<X, R, Y, 3, true, 256>(d, 32, lines, sms, st);
        return launch_wide<X, R, Y, 4, true, 256>(d, 32, lines, sms, st);
    }
    if (groups <= 512) return launch_wide<X, R, Y, 2, false, 256>(d, (groups + 63) / 64 * 32, lines, sms, st);
    const uint32_t threads = (groups + 127) / 128 * 32;
    if (groups <= 1024) return launch_wide<X, R, Y, 4, false, 256>(d, threads, lines, sms, st);
    return launch_wide<X, R, Y, 4, false, 512>(d, threads, lines, sms, st);
}
template <typename X, typename R>
cudaError_t launch_out(const cleave_layernorm_t& d, const Lines& lines, int sms, cudaStream_t st) {
    if (d.y_type == CLEAVE_T_E4M3) return launch_sizes<X, R, uint8_t>(d, lines, sms, st);
    return d.y_type == CLEAVE_T_F32 ? launch_sizes<X, R, float>(d, lines, sms, st) : launch_sizes<X, R, __nv_bfloat16>(d, lines, sms, st);
}
template <typename X>
cudaError_t launch_residual(const cleave_layernorm_t& d, const Lines& lines, int sms, cudaStream_t st) {
    if (!d.r) return launch_out<X, NoRes>(d, lines, sms, st);
    return d.r_type == CLEAVE_T_F32 ? launch_out<X, float>(d, lines, sms, st) : launch_out<X, __nv_bfloat16>(d, lines, sms, st);
}
cudaError_t launch_layernorm(const cleave_layernorm_t& d, int sms, cudaStream_t st) {
    Lines lines;
    const bool wide = d.cols >= 64 && d.cols <= 16384 && lines_agree({{d.x, d.ldx, d.x_type}, {d.r, d.ldr, d.r_type}, {d.h, d.ldh, d.r_type}, {d.y, d.ldy, d.y_type}}, lines);
    if (wide) return d.x_type == CLEAVE_T_F32 ? launch_residual<float>(d, lines, sms, st) : launch_residual<__nv_bfloat16>(d, lines, sms, st);
    if (d.cols <= kOwnCols) {
        const uint32_t threads = own_threads(d.cols);
        const unsigned ctas = (unsigned)std::min<uint64_t>(d.rows, (uint64_t)sms * std::min(24u, 1024u / threads));
        return launch_chained(threads <= 512 ? layernorm_own_kernel<512> : layernorm_own_kernel<1024>, ctas, threads, 0, st, d);
    }
    return launch_chained(layernorm_any_kernel, (unsigned)d.rows, kRowThreads, 0, st, d);
}

// ---- backward ----------------------------------------------------------------------------------------
// A CTA takes the rows part, part + parts, ...; its shares of dw and db go to row `part` of the workspace (fp32
// [parts x 2 cols], dw's columns first; each element belongs to one thread), and layernorm_sum_parts_kernel adds the parts in order.
// The wide form's shape: threads a row, groups of 8 columns a thread, rows that a CTA works on at a time.  What counts is work between two
// barriers: many groups a thread and few threads (16384 rows of 4096 columns: 4 groups and 128 threads 95 us, 2 groups and 256
// threads 99); up to 1024 columns a row is one warp's.  A CTA an SM, with as many warps as registers allow
// (16187 x 2968 bf16 with 3 groups and 12 warps 79 us, 4 groups and 6 warps 100; 8000 x 2600 with an fp32 h 77 and 62: its rows spill at 12 warps).
// Not so everywhere: an fp32 h spills at other widths of one to three groups too (up to 768, 1025 to 1536 and 2049 to 2304 columns, 120 to 320 bytes a
// thread), and every type above 8192 columns, with 512 threads (216 to 944 bytes; rows off lines spill more).
struct Shape { uint32_t threads, groups, rows; };
Shape backward_shape(uint32_t cols, bool f32) {                  // f32: h is, and takes more registers
    const uint32_t units = (cols + 7) / 8;
    const uint32_t threads = units <= 128 ? 32u : (units <= 256 ? 64u : (units <= 384 && f32 ? 96u : (units <= 640 ? 128u : (units <= 1024 ? (units + 127) / 128 * 32 : 512u))));
    const uint32_t groups = (units + threads - 1) / threads;
    const uint32_t warps = groups <= 2 ? 16 : (groups == 3 ? 12 : 8);
    return {threads, groups, std::max(1u, warps * 32 / threads)};
}
uint32_t layernorm_backward_parts(uint64_t rows, uint32_t cols) { return (uint32_t)std::min<uint64_t>(rows, kPartSms); }

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

// Two sums over a row's threads with one barrier; the buffers take turns.  The lower half of a warp carries on with the first sum, the upper
// half with the second: half of the shuffles.
__device__ __forceinline__ float half_sum(float v) {
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ float2 row_sums(float a, float b, float (&p)[2][32]) {        // over the threads with this threadIdx.y
    const uint32_t lane = threadIdx.x & 31u, half = lane >> 4, warps = blockDim.x / 32;
    float v = half ? b : a;
    v = half_sum(v + __shfl_xor_sync(0xFFFFFFFFu, half ? a : b, 16));
    if (warps > 1) {
        if ((lane & 15u) == 0) p[half][threadIdx.x >> 5] = v;
        if (blockDim.y == 1) __syncthreads();
        else asm volatile("bar.sync %0, %1;" ::"r"(threadIdx.y + 1), "r"(blockDim.x) : "memory");
        v = (lane & 15u) < warps ? p[half][lane & 15u] : 0.f;
        if (warps > 16 && (lane & 15u) + 16 < warps) v += p[half][(lane & 15u) + 16];
        v = half_sum(v);
    }
    return make_float2(__shfl_sync(0xFFFFFFFFu, v, 0), __shfl_sync(0xFFFFFFFFu, v, 16));
}

template <int T>
__global__ void __launch_bounds__(T) layernorm_backward_own_kernel(const __grid_constant__ cleave_layernorm_backward_t d, float* __restrict__ ws) {
    __shared__ float parts[2][2][32];
    begin_chained();
    float w[kOwn], dw[kOwn], db[kOwn];
    uint32_t ndy[kOwn], nh[kOwn], nres[kOwn];
#pragma unroll
    for (uint32_t k = 0; k < kOwn; ++k) { w[k] = 1.f; dw[k] = db[k] = 0.f; }
    if (d.w) { load_own(d.w, d.w_type, 0, d.cols, nh); own_values(nh, d.w_type, d.cols, w); }
    const Reciprocal inv_cols(d.cols);
    uint64_t row = blockIdx.x;
    load_own(d.dy, d.dy_type, row * d.lddy, d.cols, ndy);
    load_own(d.h, d.h_type, row * d.ldh, d.cols, nh);
    if (d.dres) load_own(d.dres, d.h_type, row * d.lddres, d.cols, nres);
    for (uint32_t it = 0; row < d.rows; row += gridDim.x, ++it) {
        const float rstd = d.rstd[row], mean = d.mean[row];
        float q[kOwn], g[kOwn], res[kOwn], dot = 0.f, sum = 0.f;
        own_values(ndy, d.dy_type, d.cols, q);
        own_values(nh, d.h_type, d.cols, g);
        if (d.dres) own_values(nres, d.h_type, d.cols, res);
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) {                    // (columns that do not exist: dy is 0)
            g[k] = (g[k] - mean) * rstd;
            dw[k] = fmaf(q[k], g[k], dw[k]);
            db[k] += q[k];
            q[k] *= w[k];
            sum += q[k];
            dot = fmaf(q[k], g[k], dot);
        }
        const uint64_t next = row + gridDim.x;
        if (next < d.rows) {
            load_own(d.dy, d.dy_type, next * d.lddy, d.cols, ndy);
            load_own(d.h, d.h_type, next * d.ldh, d.cols, nh);
            if (d.dres) load_own(d.dres, d.h_type, next * d.lddres, d.cols, nres);
        }
        const float2 both = row_sums(sum, dot, parts[it & 1]);
        const float shift = inv_cols.mean(both.x), along = both.y * inv_cols.first;
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) { q[k] = rstd * (q[k] - shift - g[k] * along); if (d.dres) q[k] += res[k]; }
        store_own(d.dx, d.h_type, row * d.lddx, d.cols, q);
    }
    if (d.dw || d.db)
#pragma unroll
        for (uint32_t k = 0; k < kOwn; ++k) {
            const uint32_t j = threadIdx.x + k * blockDim.x;
            if (j < d.cols) { ws[(uint64_t)blockIdx.x * 2 * d.cols + j] = dw[k]; ws[((uint64_t)blockIdx.x * 2 + 1) * d.cols + j] = db[k]; }
        }
}

// V groups of 8 columns a thread, blockDim.y rows at a time, each with a ring of the next rows of (dy, h, dres) in shared memory; the
// weights (where registers hold them) and the shares of dw and db stay in registers over all rows, and the
// CTA's rows add theirs at the end.
// EDGES: rows that do not begin or end with a line (their threads hold more: 16384 x 5120 156 us in place of 123).
template <typename D, typename H, int V, int T, bool EDGES>
__global__ void __launch_bounds__(T, 1) layernorm_backward_wide_kernel(const __grid_constant__ cleave_layernorm_backward_t d, float* __restrict__ ws, uint32_t stages, const Lines lines) {
    extern __shared__ __align__(16) uint8_t rings[];
    __shared__ float buffers[16][2][2][32];
    begin_chained();
    constexpr uint32_t BD = Bytes8<D>::value, BH = Bytes8<H>::value;
    constexpr bool KEEP = T < 512 ? V < 5 || sizeof(H) == 2 : V < 3;
    float (&parts)[2][2][32] = buffers[threadIdx.y];
    const uint32_t tid = threadIdx.x, nt = blockDim.x;
    const bool res = d.dres != nullptr;
    const uint64_t first = blockIdx.x + (uint64_t)gridDim.x * threadIdx.y, stride = (uint64_t)gridDim.x * blockDim.y;        // (whole units of rows where rows differ)
    const uint32_t head = EDGES ? lines.head(first, d.cols) : 0u, groups = (d.cols - head) / 8, edge = EDGES ? edge_column(tid, head, d.cols - head - groups * 8, d.cols) : d.cols;
    const uint32_t off_h = d.cols / 8 * BD, off_res = off_h + d.cols / 8 * BH, stage_bytes = off_res + (res ? d.cols / 8 * BH : 0u);
    uint8_t* ring = rings + threadIdx.y * stages * stage_bytes;
    const uint32_t ring_base = (uint32_t)__cvta_generic_to_shared(ring);
    const Reciprocal inv_cols(d.cols);
    bool live[V];
#pragma unroll
    for (int v = 0; v < V; ++v) live[v] = tid + v * nt < groups;
    const uint8_t* pd = reinterpret_cast<const uint8_t*>(static_cast<const D*>(d.dy) + first * d.lddy + head) + tid * BD;
    const uint8_t* ph = reinterpret_cast<const uint8_t*>(static_cast<const H*>(d.h) + first * d.ldh + head) + tid * BH;
    const uint8_t* pr = res ? reinterpret_cast<const uint8_t*>(static_cast<const H*>(d.dres) + first * d.lddres + head) + tid * BH : nullptr;
    const uint64_t step_d = stride * d.lddy * (BD / 8), step_h = stride * d.ldh * (BH / 8), step_r = stride * d.lddres * (BH / 8);
    uint64_t ahead = first;
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
            ahead += stride; pd += step_d; ph += step_h;
            if (res) pr += step_r;
        }
        cp_async_commit();
    };
    for (uint32_t s = 0; s < stages; ++s) fetch(s * stage_bytes);
    F2 w[KEEP ? V : 1][4], dw[V][4], db[V][4];
    if constexpr (KEEP) load_vectors8<V>(d.w, d.w_type, head + tid * 8, nt * 8, live, 1.f, w);
    // the thread's single column: its weight, its shares, and the next row's values
    const float edge_w = EDGES && edge < d.cols && d.w ? load_as(d.w, d.w_type, edge) : 1.f;
    float edge_dw = 0.f, edge_db = 0.f;
    D next_dy = from_f32<D>(0.f);                                // (as they are stored: a conversion would wait for the load)
    H next_h = from_f32<H>(0.f), next_res = next_h;
    auto ask_edge = [&](uint64_t row) {
        if (EDGES && edge < d.cols && row < d.rows) {
            next_dy = static_cast<const D*>(d.dy)[row * d.lddy + edge];
            next_h = static_cast<const H*>(d.h)[row * d.ldh + edge];
            if (res) next_res = static_cast<const H*>(d.dres)[row * d.lddres + edge];
        }
    };
    ask_edge(first);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[v][i] = db[v][i] = f2(0.f, 0.f);
    H* pdx = static_cast<H*>(d.dx) + first * d.lddx + head + tid * 8;
    uint32_t it = 0, at = 0;
    float next_rstd = first < d.rows ? d.rstd[first] : 0.f, next_mean = first < d.rows ? d.mean[first] : 0.f;
    for (uint64_t row = first; row < d.rows; row += stride, ++it) {
        if (stages >= 4) cp_async_wait<3>(); else if (stages == 3) cp_async_wait<2>(); else if (stages == 2) cp_async_wait<1>(); else cp_async_wait<0>();
        const float rstd = next_rstd, mean = next_mean;
        if (row + stride < d.rows) { next_rstd = d.rstd[row + stride]; next_mean = d.mean[row + stride]; }
        const uint8_t* stage = ring + at;
        F2 q[V][4], dots = f2(0.f, 0.f), sums = f2(0.f, 0.f);    // q = w dy; sums of q (h - mean) and of q
        Raw8<H> rh[V], rr[V];
        const F2 mean2 = f2(-mean, -mean), rstd2 = f2(rstd, rstd);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!live[v]) continue;
            const uint32_t g = tid + v * nt;
            unpack8(*reinterpret_cast<const Raw8<D>*>(stage + g * BD), q[v]);
            rh[v] = *reinterpret_cast<const Raw8<H>*>(stage + off_h + g * BH);
            if (res) rr[v] = *reinterpret_cast<const Raw8<H>*>(stage + off_res + g * BH);
            F2 h[4];
            unpack8(rh[v], h);
            if constexpr (!KEEP) load_vector8(d.w, d.w_type, head + g * 8, 1.f, w[0]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const F2 c = add2(h[i], mean2);
                dw[v][i] = fma2(mul2(q[v][i], rstd2), c, dw[v][i]);
                db[v][i] = add2(db[v][i], q[v][i]);
                q[v][i] = mul2(q[v][i], w[KEEP ? v : 0][i]);
                sums = add2(sums, q[v][i]);
                dots = fma2(q[v][i], c, dots);
            }
        }
        float edge_q = 0.f, edge_c = 0.f, edge_res = 0.f;
        if (EDGES && edge < d.cols) {
            const float dy = to_f32(next_dy);
            edge_c = to_f32(next_h) - mean;
            edge_res = to_f32(next_res);
            edge_dw = fmaf(dy * rstd, edge_c, edge_dw);
            edge_db += dy;
            edge_q = dy * edge_w;
            ask_edge(row + stride);
        }
        const float2 both = row_sums(sum_of(sums) + edge_q, fmaf(edge_q, edge_c, sum_of(dots)), parts[it & 1]);
        fetch(at);
        at = at + stage_bytes == stages * stage_bytes ? 0 : at + stage_bytes;
        // dx = rstd (q - mean(q) - (rstd (rstd mean(q (h - mean)))) (h - mean)) + dres        (rstd^3 by itself is infinite for small rows)
        const float shift = inv_cols.mean(both.x), along = rstd * (rstd * (both.y * inv_cols.first));
        const F2 shift2 = f2(-shift, -shift), along2 = f2(-along, -along);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!live[v]) continue;
            F2 dx[4], h[4];
            unpack8(rh[v], h);
#pragma unroll
            for (int i = 0; i < 4; ++i) dx[i] = fma2(along2, add2(h[i], mean2), add2(q[v][i], shift2));
            if (res) {
                unpack8(rr[v], h);
#pragma unroll
                for (int i = 0; i < 4; ++i) dx[i] = fma2(rstd2, dx[i], h[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) dx[i] = mul2(rstd2, dx[i]);
            }
            store8(pdx + v * nt * 8, dx);
        }
        if (EDGES && edge < d.cols) store_one(static_cast<H*>(d.dx) + row * d.lddx + edge, fmaf(rstd, fmaf(-along, edge_c, edge_q - shift), edge_res));
        pdx += stride * d.lddx;
    }
    if (!d.dw && !d.db) return;
    // (a row's columns may begin elsewhere than another's: the shares meet column by column)
    auto put = [&](float* to) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!live[v]) continue;
            const uint32_t j = head + (tid + v * nt) * 8;
            if (((uintptr_t)(to + j) | ((uint64_t)d.cols * 4)) % 16 == 0) {
                store8(to + j, dw[v]);
                store8(to + d.cols + j, db[v]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 a = halves(dw[v][i]), b = halves(db[v][i]);
                    to[j + 2 * i] = a.x; to[j + 2 * i + 1] = a.y;
                    to[d.cols + j + 2 * i] = b.x; to[d.cols + j + 2 * i + 1] = b.y;
                }
            }
        }
        if (EDGES && edge < d.cols) { to[edge] = edge_dw; to[d.cols + edge] = edge_db; }
    };
    if (blockDim.y > 1) {                                        // the rows' shares, in order
        float* other = reinterpret_cast<float*>(rings);
        cp_async_wait<0>();
        __syncthreads();
        if (threadIdx.y) put(other + (uint64_t)(threadIdx.y - 1) * 2 * d.cols);
        __syncthreads();
        if (threadIdx.y) return;
        for (uint32_t y = 0; y + 1 < blockDim.y; ++y) {
            const float* from = other + (uint64_t)y * 2 * d.cols;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!live[v]) continue;
                const float* a = from + head + (tid + v * nt) * 8;
                const float* b = a + d.cols;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    dw[v][i] = add2(dw[v][i], f2(a[2 * i], a[2 * i + 1]));
                    db[v][i] = add2(db[v][i], f2(b[2 * i], b[2 * i + 1]));
                }
            }
            if (EDGES && edge < d.cols) { edge_dw += from[edge]; edge_db += from[d.cols + edge]; }
        }
    }
    put(ws + (uint64_t)blockIdx.x * 2 * d.cols);
}

// out[j] = sum over the parts of ws[part][j], 0 <= j < cols for dw and behind them for db, each in a fixed order: 32 columns
// per CTA; warp w adds the parts w, w + 32, ... and the 32 sums are added by a shuffle tree.
__global__ void __launch_bounds__(1024) layernorm_sum_parts_kernel(const float* ws, uint32_t parts, uint32_t cols, float* dw, float* db) {
    __shared__ float s[32][33];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, j = blockIdx.x * 32u + lane;
    float* out = blockIdx.y ? db : dw;
    wait_for_primary();                                          // (no early start for what follows: it would land on the SMs unevenly beside the kernel whose sums these are)
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

template <typename D, typename H, int V, int T, bool EDGES>
cudaError_t launch_backward_wide(const cleave_layernorm_backward_t& d, float* ws, uint32_t parts, uint32_t stage, const Shape& sh, const Lines& lines, cudaStream_t st) {
    auto kernel = layernorm_backward_wide_kernel<D, H, V, T, EDGES>;
    static SmemLimit limit;
    const cudaError_t e = limit.raise(reinterpret_cast<const void*>(kernel), kRingMost);
    if (e != cudaSuccess) return e;
    const uint32_t stages = std::max(1u, std::min(4u, kRingMost / sh.rows / stage)), joined = (sh.rows - 1) * 2 * d.cols * 4;
    return launch_chained(kernel, parts, dim3(sh.threads, sh.rows), std::max(stage * stages * sh.rows, joined), st, d, ws, stages, lines);
}
template <typename D, typename H, bool EDGES>
cudaError_t launch_backward_edges(const cleave_layernorm_backward_t& d, float* ws, uint32_t parts, uint32_t stage, const Lines& lines, cudaStream_t st) {
    const Shape sh = backward_shape(d.cols, sizeof(H) == 4);
    if (sh.threads == 512) return sh.groups <= 3 ? launch_backward_wide<D, H, 3, 512, EDGES>(d, ws, parts, stage, sh, lines, st) : launch_backward_wide<D, H, 4, 512, EDGES>(d, ws, parts, stage, sh, lines, st);
    if (sh.groups == 5) return launch_backward_wide<D, H, 5, 256, EDGES>(d, ws, parts, stage, sh, lines, st);
    if (sh.groups == 4) return launch_backward_wide<D, H, 4, 256, EDGES>(d, ws, parts, stage, sh, lines, st);
    if (sh.groups == 3) return launch_backward_wide<D, H, 3, 384, EDGES>(d, ws, parts, stage, sh, lines, st);
    return launch_backward_wide<D, H, 2, 512, EDGES>(d, ws, parts, stage, sh, lines, st);
}
template <typename D, typename H>
cudaError_t launch_backward_types(const cleave_layernorm_backward_t& d, float* ws, uint32_t parts, uint32_t stage, const Lines& lines, cudaStream_t st) {
    return lines.at || lines.step || d.cols % 8 ? launch_backward_edges<D, H, true>(d, ws, parts, stage, lines, st) : launch_backward_edges<D, H, false>(d, ws, parts, stage, lines, st);
}
cudaError_t launch_layernorm_backward(const cleave_layernorm_backward_t& d, float* ws, cudaStream_t st) {
    uint32_t parts = layernorm_backward_parts(d.rows, d.cols);
    const Shape sh = backward_shape(d.cols, d.h_type == CLEAVE_T_F32);
    const uint64_t stage = (uint64_t)(d.cols / 8) * 8 * (type_bytes(d.dy_type) + type_bytes(d.h_type) * (d.dres ? 2u : 1u));
    Lines lines;
    const bool wide = d.cols >= 64 && d.cols <= 16384 && stage * sh.rows <= kRingMost &&
                      lines_agree({{d.dy, d.lddy, d.dy_type}, {d.h, d.ldh, d.h_type}, {d.dx, d.lddx, d.h_type}, {d.dres, d.lddres, d.h_type}}, lines);
    if (wide && lines.step && parts * sh.rows % 8 && d.rows > parts) parts = parts / 8 * 8;          // a row's next one begins like it
    cudaError_t e = cudaSuccess;
    if (parts && wide) {
        if (d.dy_type == CLEAVE_T_F32) e = d.h_type == CLEAVE_T_F32 ? launch_backward_types<float, float>(d, ws, parts, (uint32_t)stage, lines, st) : launch_backward_types<float, __nv_bfloat16>(d, ws, parts, (uint32_t)stage, lines, st);
        else e = d.h_type == CLEAVE_T_F32 ? launch_backward_types<__nv_bfloat16, float>(d, ws, parts, (uint32_t)stage, lines, st) : launch_backward_types<__nv_bfloat16, __nv_bfloat16>(d, ws, parts, (uint32_t)stage, lines, st);
    } else if (parts && d.cols <= kOwnCols) {
        const uint32_t threads = own_threads(d.cols);
        e = launch_chained(threads <= 512 ? layernorm_backward_own_kernel<512> : layernorm_backward_own_kernel<1024>, parts, threads, 0, st, d, ws);
    } else if (parts) {
        e = launch_chained(layernorm_backward_any_kernel, parts, kRowThreads, 0, st, d, ws);
    }
    if (e != cudaSuccess || (!d.dw && !d.db)) return e;
    return launch_chained(layernorm_sum_parts_kernel, dim3((d.cols + 31) / 32, 2), 1024, 0, st, ws, parts, d.cols, d.dw, d.db);
}

}  // namespace cleave
