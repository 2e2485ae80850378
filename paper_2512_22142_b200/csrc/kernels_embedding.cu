// Embedding lookup and its gradient by sorted tokens (see cleave.h).
//
// Lookup: out_i = scale table[ids_i].
//
// Gradient.  The rows of dy have to be added by token, in an order that does not change from run to run, and a vocabulary's
// tokens are far from evenly spread (a few make up half of a batch).  So:
//   order    the tokens' places are sorted by (token, place): a counting sort without communication.  CTA c owns a
//            range of the vocabulary and reads all tokens (n of them stand in L2): what is below its range is its offset,
//            what is inside is counted per warp and value; a second reading puts each place where it belongs.
//   sum      the sorted places are cut into chunks of the same length, whatever the tokens; a CTA adds the rows of a
//            chunk run by run.  A run that lies inside one chunk is a finished row; the ends of longer runs go to the workspace.
//            Other CTAs of the launch write zeros into the rows of tokens that do not occur.
//   join     the pieces of each longer run are added in order.
#include <algorithm>

#include "tokens.cuh"

namespace cleave {

// ---- lookup ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) embedding_any_kernel(const __grid_constant__ cleave_embedding_t d) {
    begin_chained();
    const uint64_t row = blockIdx.x;
    const int32_t t = load_token(d.ids, d.id_type, row, d.vocab);
    for (uint32_t j = threadIdx.x; j < d.cols; j += blockDim.x)
        store_as(d.out, d.out_type, row * d.ldo + j, t < 0 ? 0.f : d.scale * load_as(d.table, d.table_type, (uint64_t)t * d.ldt + j));
}
cudaError_t launch_embedding(const cleave_embedding_t& d, int, cudaStream_t st) {
    return launch_chained(embedding_any_kernel, (unsigned)d.n, 256, 0, st, d);
}

// ---- gradient: the tokens' order ------------------------------------------------------------------------
constexpr uint32_t kOrderThreads = 512, kOrderWarps = kOrderThreads / 32, kOrderMost = 2 * kOrderThreads;     // values a CTA owns at most

uint32_t order_values(uint32_t vocab) { return std::min(kOrderMost, std::max(32u, (vocab + kPartSms - 1) / kPartSms)); }

// offsets[v] = number of tokens below v, for v <= vocab; order[offsets[v] ...] = the places of token v, ascending
template <typename ID>
__global__ void __launch_bounds__(kOrderThreads) token_order_kernel(const ID* ids, uint32_t n, uint32_t vocab, uint32_t values, uint32_t* offsets, uint32_t* order) {
    extern __shared__ uint32_t counts[];                         // [warp][value]
    __shared__ uint32_t sums[32], below_all;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, lo = blockIdx.x * values, hi = min(vocab, lo + values);
    uint32_t* mine = counts + warp * values;
    for (uint32_t i = threadIdx.x; i < kOrderWarps * values; i += kOrderThreads) counts[i] = 0;
    if (threadIdx.x == 0) below_all = 0;
    begin_chained();
    __syncthreads();
    const uint32_t part = ((n + kOrderWarps - 1) / kOrderWarps + 31) / 32 * 32;
    const uint64_t from = (uint64_t)warp * part, to = min((uint64_t)n, from + part);
    uint32_t below = 0;
    for (uint64_t i = from + lane; i < to; i += 32) {
        const ID t = ids[i];
        if (t < 0) continue;
        if ((uint64_t)t < lo) ++below;
        else if ((uint64_t)t < hi) atomicAdd(mine + (uint32_t)(t - lo), 1u);
    }
    below = __reduce_add_sync(0xFFFFFFFFu, below);
    if (lane == 0 && below) atomicAdd(&below_all, below);        // (whole numbers: any order)
    __syncthreads();
    // a thread owns the values 2 tid and 2 tid + 1: counts become offsets among the warps, then in the whole
    uint32_t total[2] = {0, 0};
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
        const uint32_t v = 2 * threadIdx.x + k;
        if (v < values)
            for (uint32_t w = 0; w < kOrderWarps; ++w) { const uint32_t c = counts[w * values + v]; counts[w * values + v] = total[k]; total[k] += c; }
    }
    uint32_t sum = total[0] + total[1], up = sum;
    for (uint32_t o = 1; o < 32; o <<= 1) { const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, up, o); if (lane >= o) up += x; }
    if (lane == 31) sums[warp] = up;
    __syncthreads();
    uint32_t before = below_all + up - sum;
    for (uint32_t w = 0; w < warp; ++w) before += sums[w];
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
        const uint32_t v = 2 * threadIdx.x + k;
        if (v < values && lo + v < hi) {
            offsets[lo + v] = before;
            for (uint32_t w = 0; w < kOrderWarps; ++w) counts[w * values + v] += before;
        }
        before += total[k];
        if (v < values && lo + v + 1 == vocab) offsets[vocab] = before;
    }
    __syncthreads();
    for (uint64_t i = from; i < to; i += 32) {                   // in order: 32 places at a time
        const uint64_t at = i + lane;
        const int64_t t = at < to ? (int64_t)ids[at] : -1;
        const bool in = t >= (int64_t)lo && t < (int64_t)hi;
        const uint32_t some = __ballot_sync(0xFFFFFFFFu, in);
        if (in) {
            const uint32_t same = __match_any_sync(some, (uint32_t)(t - lo)), rank = __popc(same & ((1u << lane) - 1u));
            const uint32_t base = mine[(uint32_t)(t - lo)];
            order[base + rank] = (uint32_t)at;
            __syncwarp(some);
            if (rank == 0) mine[(uint32_t)(t - lo)] = base + __popc(same);
        }
        __syncwarp();
    }
}

// ---- gradient: sums --------------------------------------------------------------------------------------
constexpr uint32_t kChunkLeast = 16, kChunksMost = 16 * kPartSms;
uint32_t sum_chunk(uint64_t n) { return (uint32_t)std::max<uint64_t>(kChunkLeast, (n + kChunksMost - 1) / kChunksMost); }      // places a chunk

struct Ordered {                    // what the order kernel left
    const uint32_t* offsets;
    const uint32_t* order;
    float* parts;                   // [2 chunk + 0: the run that began before the chunk, 1: the run that goes on after it][cols]
    uint32_t chunk, chunks;
};
constexpr uint32_t kSumThreads = 256;

__device__ __forceinline__ void finish_row(const cleave_embedding_backward_t& d, uint32_t v, uint32_t j, float sum) {
    const uint64_t at = (uint64_t)v * d.lddt + j;
    sum *= d.scale;
    if (d.accumulate) sum += load_as(d.dtable, d.dtable_type, at);
    store_as(d.dtable, d.dtable_type, at, sum);
}
__global__ void __launch_bounds__(kSumThreads) embedding_sum_any_kernel(const __grid_constant__ cleave_embedding_backward_t d, const __grid_constant__ Ordered o, uint32_t zero_rows) {
    begin_chained();
    const uint32_t column = blockIdx.y * kSumThreads + threadIdx.x, columns = gridDim.y * kSumThreads;
    if (blockIdx.x >= o.chunks) {                                // rows of tokens that do not occur
        const uint64_t v0 = (uint64_t)(blockIdx.x - o.chunks) * zero_rows;
        for (uint64_t v = v0; v < min((uint64_t)d.vocab, v0 + zero_rows); ++v)
            if (o.offsets[v] == o.offsets[v + 1])
                for (uint32_t j = column; j < d.cols; j += columns) store_as(d.dtable, d.dtable_type, v * d.lddt + j, 0.f);
        return;
    }
    const uint32_t total = o.offsets[d.vocab], first = blockIdx.x * o.chunk, last = min(total, first + o.chunk);
    for (uint32_t p = first; p < last;) {
        const uint32_t v = (uint32_t)load_token(d.ids, d.id_type, o.order[p], d.vocab), begin = o.offsets[v], end = o.offsets[v + 1], stop = min(end, last);
        for (uint32_t j = column; j < d.cols; j += columns) {
            float sum = 0.f;
            for (uint32_t i = p; i < stop; ++i) sum += load_as(d.dy, d.dy_type, (uint64_t)o.order[i] * d.lddy + j);
            if (begin >= first && end <= last) finish_row(d, v, j, sum);
            else o.parts[((uint64_t)blockIdx.x * 2 + (begin < first ? 0 : 1)) * d.cols + j] = sum;
        }
        p = stop;
    }
}
__global__ void __launch_bounds__(kSumThreads) embedding_join_kernel(const __grid_constant__ cleave_embedding_backward_t d, const __grid_constant__ Ordered o) {
    begin_chained();
    const uint32_t total = o.offsets[d.vocab], first = blockIdx.x * o.chunk, after = first + o.chunk;
    if (after >= total) return;                                  // nothing goes on behind the chunk
    const uint32_t v = (uint32_t)load_token(d.ids, d.id_type, o.order[after - 1], d.vocab), begin = o.offsets[v], end = o.offsets[v + 1];
    if (begin < first || end <= after) return;                   // the run began before the chunk, or ends with it
    for (uint32_t j = blockIdx.y * kSumThreads + threadIdx.x; j < d.cols; j += gridDim.y * kSumThreads) {
        float sum = o.parts[((uint64_t)blockIdx.x * 2 + 1) * d.cols + j];
        for (uint32_t c = blockIdx.x + 1; c <= (end - 1) / o.chunk; ++c) sum += o.parts[(uint64_t)c * 2 * d.cols + j];
        finish_row(d, v, j, sum);
    }
}

static uint64_t order_bytes(uint64_t n, uint32_t vocab) { return ((uint64_t)vocab + 1 + n + 3) / 4 * 16; }
uint64_t embedding_backward_workspace(uint64_t n, uint32_t vocab, uint32_t cols) {
    const uint64_t chunks = n ? (n + sum_chunk(n) - 1) / sum_chunk(n) : 0;
    return order_bytes(n, vocab) + chunks * 2 * cols * sizeof(float);
}
cudaError_t launch_embedding_backward(const cleave_embedding_backward_t& d, void* ws, cudaStream_t st) {
    const uint32_t values = order_values(d.vocab), n = (uint32_t)d.n;
    uint32_t* offsets = static_cast<uint32_t*>(ws);
    uint32_t* order = offsets + d.vocab + 1;
    Ordered o = {offsets, order, reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + order_bytes(n, d.vocab)), sum_chunk(n), 0};
    o.chunks = (n + o.chunk - 1) / o.chunk;
    const uint32_t smem = kOrderWarps * values * 4;
    const unsigned ctas = (d.vocab + values - 1) / values;
    static SmemLimit limits[2];
    cudaError_t e;
    if (d.id_type == CLEAVE_T_I64) {
        e = limits[1].raise(reinterpret_cast<const void*>(token_order_kernel<int64_t>), kOrderWarps * kOrderMost * 4);
        if (e == cudaSuccess) e = launch_chained(token_order_kernel<int64_t>, ctas, kOrderThreads, smem, st, static_cast<const int64_t*>(d.ids), n, d.vocab, values, offsets, order);
    } else {
        e = limits[0].raise(reinterpret_cast<const void*>(token_order_kernel<int32_t>), kOrderWarps * kOrderMost * 4);
        if (e == cudaSuccess) e = launch_chained(token_order_kernel<int32_t>, ctas, kOrderThreads, smem, st, static_cast<const int32_t*>(d.ids), n, d.vocab, values, offsets, order);
    }
    if (e != cudaSuccess) return e;
    const uint32_t zero_rows = 64, tiles = std::min(65535u, (d.cols + kSumThreads - 1) / kSumThreads);
    const unsigned zeros = d.accumulate ? 0 : (d.vocab + zero_rows - 1) / zero_rows;
    if (o.chunks + zeros) e = launch_chained(embedding_sum_any_kernel, dim3(o.chunks + zeros, tiles), kSumThreads, 0, st, d, o, zero_rows);
    if (e != cudaSuccess || o.chunks < 2) return e;
    return launch_chained(embedding_join_kernel, dim3(o.chunks - 1, tiles), kSumThreads, 0, st, d, o);
}

}  // namespace cleave
