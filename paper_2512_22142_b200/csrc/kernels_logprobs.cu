// Log probabilities of given tokens with entropy and top alternatives, distillation from a teacher's top scores, and the
// backward passes of both (see cleave.h).
#include <algorithm>

#include "rows.cuh"
#include "tokens.cuh"

namespace cleave {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kMasked = -0x1p126f;             // a row whose largest score is not above this has nothing left
constexpr uint32_t kScoreThreads = 256;

// whole number that orders like a score: NaN above all, +0 and -0 alike
__device__ __forceinline__ uint32_t score_order(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return x != x ? 0xFFFFFFFFu : (b & 0x80000000u ? ~b : b | 0x80000000u);
}
// score, then the lower place: larger is better, no two alike, none 0 or all ones
__device__ __forceinline__ uint64_t candidate(float x, uint32_t j) { return (uint64_t)score_order(x) << 32 | (0x7FFFFFFFu - j); }
__device__ __forceinline__ uint32_t place_of(uint64_t c) { return 0x7FFFFFFFu - (uint32_t)c; }

struct RowSums { float top, sum, mean; };        // largest score; sum of e = exp(s (x - top)); sum of e s (x - top)

template <typename F>
__device__ __forceinline__ float cta_reduce(float v, float* buf, F&& f) {       // buf: one value a warp; ends with a barrier
#pragma unroll
    for (int o = 16; o; o >>= 1) v = f(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    if ((threadIdx.x & 31u) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    v = buf[0];
    for (uint32_t w = 1; w < blockDim.x / 32; ++w) v = f(v, buf[w]);
    __syncthreads();
    return v;
}
__device__ __forceinline__ RowSums row_sums_any(const void* x, uint32_t type, uint64_t at, uint32_t cols, float scale, float* buf) {
    RowSums r = {-INFINITY, 0.f, 0.f};
    for (uint32_t j = threadIdx.x; j < cols; j += blockDim.x) r.top = max_nan(r.top, load_as(x, type, at + j));
    r.top = cta_reduce(r.top, buf, [](float a, float b) { return max_nan(a, b); });
    if (r.top <= kMasked) return r;
    for (uint32_t j = threadIdx.x; j < cols; j += blockDim.x) {
        const float d = scale * (load_as(x, type, at + j) - r.top), e = exp2_fast(d * kLog2e);
        r.sum += e;
        if (e != 0.f) r.mean = fmaf(e, d, r.mean);
    }
    r.sum = cta_sum(r.sum, buf);
    r.mean = cta_sum(r.mean, buf);
    return r;
}
__device__ __forceinline__ float row_lse(const RowSums& r, float scale) { return r.top <= kMasked ? -INFINITY : fmaf(scale, r.top, logf(r.sum)); }

__global__ void __launch_bounds__(kScoreThreads) logprobs_any_kernel(const __grid_constant__ cleave_logprobs_t d) {
    __shared__ float buf[32];
    __shared__ unsigned long long best;
    begin_chained();
    const uint64_t row = blockIdx.x, at = row * d.ldx;
    const RowSums r = row_sums_any(d.x, d.x_type, at, d.cols, d.scale, buf);
    const float lse = row_lse(r, d.scale);
    const bool nothing = r.top <= kMasked;
    if (threadIdx.x == 0) {
        if (d.lse) d.lse[row] = lse;
        if (d.entropy) d.entropy[row] = nothing ? 0.f : logf(r.sum) - r.mean / r.sum;
        if (d.logp) {
            const int32_t t = load_token(d.ids, d.id_type, row, d.cols);
            d.logp[row] = t < 0 ? 0.f : (nothing ? -INFINITY : fmaf(d.scale, load_as(d.x, d.x_type, at + t), -lse));
        }
    }
    uint64_t last = ~0ull;                                       // the best candidate of each round is the best below the last one
    for (uint32_t k = 0; k < d.top; ++k) {
        if (threadIdx.x == 0) best = 0;
        __syncthreads();
        unsigned long long mine = 0;
        for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x) {
            const uint64_t c = candidate(load_as(d.x, d.x_type, at + j), j);
            if (c < last && c > mine) mine = c;
        }
        atomicMax(&best, mine);
        __syncthreads();
        last = best;
        __syncthreads();
        if (threadIdx.x == 0) {
            const uint32_t j = place_of(last);
            if (d.top_index) d.top_index[row * d.ldti + k] = (int32_t)j;
            if (d.top_values) d.top_values[row * d.ldtv + k] = nothing ? -INFINITY : fmaf(d.scale, load_as(d.x, d.x_type, at + j), -lse);
        }
    }
}
cudaError_t launch_logprobs(const cleave_logprobs_t& d, int, cudaStream_t st) {
    return launch_chained(logprobs_any_kernel, (unsigned)d.rows, kScoreThreads, 0, st, d);
}

// ---- gradients -----------------------------------------------------------------------------------------
// dx_j = s (a p_j + b p_j log p_j - [what the row's named places hold]): the whole row from the scores and lse, then the
// named places once more, from scores that were read before the row was written (dx may be x's buffer).  A row of which
// nothing is asked (a = b = 0 and no place) is zeros whatever stands in it: padded rows may hold anything.
struct RowSlope { float a, b; };
__device__ __forceinline__ float slope_at(float x, float scale, float lse, const RowSlope& g) {
    const float t = fmaf(scale, x, -lse), p = exp2_fast(t * kLog2e);
    return p == 0.f ? 0.f : fmaf(g.b, t, g.a) * p;
}
__device__ __forceinline__ void write_row_any(const void* x, uint32_t x_type, uint64_t ox, void* dx, uint32_t dx_type, uint64_t odx, uint32_t cols, float scale, float lse,
                                              const RowSlope& g) {
    const bool zeros = lse == -INFINITY || (g.a == 0.f && g.b == 0.f);
    for (uint32_t j = threadIdx.x; j < cols; j += blockDim.x)
        store_as(dx, dx_type, odx + j, zeros ? 0.f : scale * slope_at(load_as(x, x_type, ox + j), scale, lse, g));
}
__global__ void __launch_bounds__(kScoreThreads) logprobs_backward_any_kernel(const __grid_constant__ cleave_logprobs_backward_t d) {
    begin_chained();
    const uint64_t row = blockIdx.x, ox = row * d.ldx, odx = row * d.lddx;
    const float lse = d.lse[row];
    const int32_t t = d.dlogp ? load_token(d.ids, d.id_type, row, d.cols) : -1;
    const float up = t < 0 ? 0.f : d.dlogp[row], dh = d.dentropy ? d.dentropy[row] : 0.f;
    const RowSlope g = {(d.dlse ? d.dlse[row] : 0.f) - up - (dh != 0.f ? dh * d.entropy[row] : 0.f), -dh};
    const bool named = up != 0.f && lse != -INFINITY;            // (a NaN counts)
    const float own = named ? slope_at(load_as(d.x, d.x_type, ox + t), d.scale, lse, g) : 0.f;
    __syncthreads();                                             // every thread has its token's score
    write_row_any(d.x, d.x_type, ox, d.dx, d.dx_type, odx, d.cols, d.scale, lse, g);
    __syncthreads();
    if (named && threadIdx.x == 0) store_as(d.dx, d.dx_type, odx + t, d.scale * (own + up));
}
cudaError_t launch_logprobs_backward(const cleave_logprobs_backward_t& d, int, cudaStream_t st) {
    return launch_chained(logprobs_backward_any_kernel, (unsigned)d.rows, kScoreThreads, 0, st, d);
}

// ---- distillation ------------------------------------------------------------------------------------------
// The row's teacher: thread k < d.k has place k (or -1) and q_k; `log_q` where q_k > 0.  All threads of the CTA take part.
struct Place { int32_t j; float q, log_q; };
__device__ __forceinline__ Place teacher(const cleave_distill_t& d, uint64_t row, float* buf) {
    Place p = {-1, 0.f, 0.f};
    float v = -INFINITY;
    if (threadIdx.x < d.k) {
        p.j = load_token(d.index, d.index_type, row * d.ldindex + threadIdx.x, d.cols);
        if (p.j >= 0) v = d.scale * load_as(d.values, d.values_type, row * d.ldvalues + threadIdx.x);
    }
    if (d.normalize) {
        const float top = cta_reduce(v, buf, [](float a, float b) { return max_nan(a, b); });
        v = top == -INFINITY ? -INFINITY : v - top;
        p.q = v == -INFINITY ? 0.f : exp2_fast(v * kLog2e);
        const float sum = cta_sum(p.q, buf);
        p.log_q = v - logf(sum);
        p.q = p.q == 0.f ? 0.f : p.q / sum;
    } else {
        p.log_q = v;
        p.q = v == -INFINITY ? 0.f : exp2_fast(v * kLog2e);
    }
    if (p.q == 0.f) p.j = -1;
    return p;
}
__global__ void __launch_bounds__(kScoreThreads) distill_any_kernel(const __grid_constant__ cleave_distill_t d) {
    __shared__ float buf[32];
    begin_chained();
    const uint64_t row = blockIdx.x, at = row * d.ldx;
    const RowSums r = row_sums_any(d.x, d.x_type, at, d.cols, d.scale, buf);
    const float lse = row_lse(r, d.scale);
    const Place p = teacher(d, row, buf);
    float term = 0.f;
    if (p.j >= 0) term = p.q * (p.log_q - (lse == -INFINITY ? -INFINITY : fmaf(d.scale, load_as(d.x, d.x_type, at + p.j), -lse)));
    term = cta_sum(term, buf);
    if (threadIdx.x == 0) {
        d.loss[row] = term;
        if (d.lse) d.lse[row] = lse;
    }
}
cudaError_t launch_distill(const cleave_distill_t& d, int, cudaStream_t st) {
    return launch_chained(distill_any_kernel, (unsigned)d.rows, kScoreThreads, 0, st, d);
}
__global__ void __launch_bounds__(kScoreThreads) distill_backward_any_kernel(const __grid_constant__ cleave_distill_backward_t d) {
    __shared__ float buf[32];
    __shared__ int32_t places[CLEAVE_DISTILL_MOST];
    __shared__ float weights[CLEAVE_DISTILL_MOST];
    begin_chained();
    const uint64_t row = blockIdx.x, ox = row * d.f.ldx, odx = row * d.lddx;
    const float lse = d.f.lse[row], up = d.dloss[row];
    const Place p = teacher(d.f, row, buf);
    if (threadIdx.x < d.f.k) { places[threadIdx.x] = p.j; weights[threadIdx.x] = p.q; }
    const float all = cta_sum(p.q, buf);                         // (its barriers show the places to all)
    const RowSlope g = {up == 0.f || all == 0.f ? 0.f : up * all, 0.f};
    bool named = p.j >= 0 && up != 0.f && lse != -INFINITY;
    float own = 0.f;
    if (named) {
        float q = 0.f;
        for (uint32_t k = 0; k < d.f.k; ++k)
            if (places[k] == p.j) { q += weights[k]; named = named && k >= threadIdx.x; }      // of entries with the same place the first writes
        own = slope_at(load_as(d.f.x, d.f.x_type, ox + p.j), d.f.scale, lse, g) - up * q;
    }
    __syncthreads();
    write_row_any(d.f.x, d.f.x_type, ox, d.dx, d.dx_type, odx, d.f.cols, d.f.scale, lse, g);
    __syncthreads();
    if (named) store_as(d.dx, d.dx_type, odx + p.j, d.f.scale * own);
}
cudaError_t launch_distill_backward(const cleave_distill_backward_t& d, int, cudaStream_t st) {
    return launch_chained(distill_backward_any_kernel, (unsigned)d.f.rows, kScoreThreads, 0, st, d);
}

}  // namespace cleave
