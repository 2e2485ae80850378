// Embedding lookup and its gradient by sorted tokens (see cleave.h).
//
// Lookup: out_i = scale table[ids_i].  A warp takes 1024 columns of a row, four 16-byte groups a lane, all of them asked for at
// once; bound by the HBM (few rows: by one token's and one row's latency).
//
// Gradient.  The rows of dy have to be added by token, in an order that does not change from run to run, and a vocabulary's
// tokens are far from evenly spread (a few make up half of a batch).  So:
//   order    the tokens' places are sorted by (token modulo a power of two, token, place): a counting sort without communication.
//            CTA c owns the tokens v with v mod CTAs = c (neighbours, which are alike in frequency, go to different ones) and reads
//            all tokens (n of them stand in L2): those of lower remainder are its offset, its own are counted per warp and
//            token; a second reading puts each place where it belongs.  Where the table is not added to, other CTAs of the launch fill it with
//            zeros meanwhile (the rows of tokens that occur are written again: a twentieth of the bytes, for a launch's latency).
//   sum      the sorted places are cut into chunks of the same length, whatever the tokens; a CTA adds the rows of a
//            chunk run by run.  A run that lies inside one chunk is a finished row; the ends of longer runs go to the workspace.
//   join     the pieces of each longer run are added in order.
// Bound by the HBM where the whole table is written, by the three launches' latencies where few rows are.  Measured, with tokens whose
// frequency falls with their rank: 8192 tokens into the whole of a 50257 x 768 fp32 table 41.7 us (28 of them the zeros and, beside them,
// the sorting; its bytes take 26), 16384 added to a 32000 x 4096 table 69 us (order 8, sum 50, join 9; its bytes take 44.5).  Lookup of
// 16384 x 5120 bf16 37 us (6.0 TB/s), of 64 x 4096 4.3; rows off 16 bytes go by single elements (5119 columns, evenly spread tokens, 82 us
// where 5120 take 51).
//
// Tried and not kept: zeros beside the sums instead of beside the sorting (82 us for the first of these); a run that ends soon behind its
// chunk finished there instead of in pieces (77 us for the second: chunks of unlike length); ranges of the vocabulary as owners
// (one of them has half of the tokens: 77 us).
#include <algorithm>
#include <type_traits>

#include "tokens.cuh"

namespace cleave {

// ---- lookup ------------------------------------------------------------------------------------------
// WIDE: an item is 1024 columns of a row, in groups of 8; else 256 columns, neighbouring lanes next to each other.
template <typename X, typename D, bool WIDE>
__global__ void __launch_bounds__(256) embedding_kernel(const __grid_constant__ cleave_embedding_t d, uint32_t row_items) {
    begin_chained();
    const uint64_t item = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5), row = item / row_items;
    if (row >= d.n) return;
    const uint32_t lane = threadIdx.x & 31u, j0 = (uint32_t)(item % row_items) * (WIDE ? 1024u : 256u);
    const int32_t t = load_token(d.ids, d.id_type, row, d.vocab);
    const X* from = static_cast<const X*>(d.table) + (uint64_t)max(t, 0) * d.ldt;
    D* to = static_cast<D*>(d.out) + row * d.ldo;
    if constexpr (WIDE) {
        Raw8<X> raw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t j = j0 + (lane + 32 * i) * 8;
            if (j < d.cols && t >= 0) {
#pragma unroll
                for (int k = 0; k < (int)(sizeof(raw[i].w) / 16); ++k) raw[i].w[k] = reinterpret_cast<const uint4*>(from + j)[k];
            }
        }
        const F2 scale = f2(d.scale, d.scale);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t j = j0 + (lane + 32 * i) * 8;
            if (j >= d.cols) continue;
            F2 v[4] = {f2(0.f, 0.f), f2(0.f, 0.f), f2(0.f, 0.f), f2(0.f, 0.f)};
            if (t >= 0) {
                unpack8(raw[i], v);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = mul2(v[k], scale);
            }
            store8(to + j, v);
        }
    } else {
        X raw[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) if (j0 + lane + 32 * i < d.cols && t >= 0) raw[i] = from[j0 + lane + 32 * i];
#pragma unroll
        for (int i = 0; i < 8; ++i) if (j0 + lane + 32 * i < d.cols) to[j0 + lane + 32 * i] = from_f32<D>(t < 0 ? 0.f : d.scale * to_f32(raw[i]));
    }
}
template <typename X, typename D>
cudaError_t launch_embedding_types(const cleave_embedding_t& d, bool wide, cudaStream_t st) {
    const uint32_t items = wide ? (d.cols + 1023) / 1024 : (d.cols + 255) / 256;
    const uint64_t ctas = (d.n * items + 7) / 8;
    return launch_chained(wide ? embedding_kernel<X, D, true> : embedding_kernel<X, D, false>, (unsigned)ctas, 256, 0, st, d, items);
}
cudaError_t launch_embedding(const cleave_embedding_t& d, cudaStream_t st) {
    const bool wide = d.cols % 8 == 0 && rows_wide(d.table, d.ldt, d.table_type) && rows_wide(d.out, d.ldo, d.out_type);
    if (d.table_type == CLEAVE_T_F32) return d.out_type == CLEAVE_T_F32 ? launch_embedding_types<float, float>(d, wide, st) : launch_embedding_types<float, __nv_bfloat16>(d, wide, st);
    return d.out_type == CLEAVE_T_F32 ? launch_embedding_types<__nv_bfloat16, float>(d, wide, st) : launch_embedding_types<__nv_bfloat16, __nv_bfloat16>(d, wide, st);
}

// ---- gradient: the tokens' order ------------------------------------------------------------------------
constexpr uint32_t kOrderThreads = 1024, kOrderWarps = kOrderThreads / 32, kOrderMost = kOrderThreads;        // tokens of the vocabulary a CTA owns at most

// log2 of the number of owners: a power of two near the number of SMs, more for a vocabulary beyond 131072
uint32_t order_owners(uint32_t vocab) {
    uint32_t bits = 7;
    while ((uint64_t)kOrderMost << bits < vocab) ++bits;
    return bits;
}

struct Zeros {                      // rows to be filled with zeros, each cut into pieces of kZeroPiece bytes; a row after another is one row
    uint8_t* p;
    uint64_t pitch, row_bytes, pieces, tasks;
    uint32_t element;
};
constexpr uint32_t kZeroPiece = 4096;
// a warp fills [p, p + bytes): elements up to 16 bytes, 16 bytes, elements
__device__ __forceinline__ void fill_zeros(uint8_t* p, uint32_t bytes, uint32_t element) {
    const uint32_t lane = threadIdx.x & 31u, head = min(bytes, (0u - (uint32_t)(uintptr_t)p) % 16u), body = (bytes - head) / 16, tail = bytes - head - body * 16;
    auto one = [&](uint8_t* q) {
        if (element == 4) *reinterpret_cast<uint32_t*>(q) = 0;
        else *reinterpret_cast<uint16_t*>(q) = 0;
    };
    if (lane * element < head) one(p + lane * element);
    if (lane * element < tail) one(p + bytes - tail + lane * element);
#pragma unroll 4
    for (uint32_t i = lane; i < body; i += 32) reinterpret_cast<uint4*>(p + head)[i] = make_uint4(0u, 0u, 0u, 0u);
}

// sorted = (place, v) by v mod owners, v, place; ends[v] = where the places of token v end in it; *count = how many there are
// AHEAD: loads of 32 tokens that a warp has under way; those of the first are kept for the second reading.
template <typename ID, int AHEAD>
__global__ void __launch_bounds__(kOrderThreads) token_order_kernel(const ID* ids, uint32_t n, uint32_t vocab, uint32_t bits, uint32_t values, uint32_t* ends, uint32_t* count, uint2* sorted,
                                                                    const __grid_constant__ Zeros z) {
    const uint32_t owners = 1u << bits, low = owners - 1;
    if (blockIdx.x >= owners) {
        begin_chained();
        const uint64_t step = (uint64_t)(gridDim.x - owners) * kOrderWarps;
        for (uint64_t t = (uint64_t)(blockIdx.x - owners) * kOrderWarps + (threadIdx.x >> 5); t < z.tasks; t += step) {
            const uint64_t row = z.pieces == z.tasks ? 0 : t / z.pieces, at = (t - row * z.pieces) * kZeroPiece;
            fill_zeros(z.p + row * z.pitch + at, (uint32_t)min((uint64_t)kZeroPiece, z.row_bytes - at), z.element);
        }
        return;
    }
    extern __shared__ uint32_t counts[];                         // [warp][value]
    __shared__ uint32_t sums[32], below_all;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    uint32_t* mine = counts + warp * values;
    for (uint32_t i = threadIdx.x; i < kOrderWarps * values; i += kOrderThreads) counts[i] = 0;
    if (threadIdx.x == 0) below_all = 0;
    begin_chained();
    __syncthreads();
    const uint32_t part = ((n + kOrderWarps - 1) / kOrderWarps + 31) / 32 * 32;
    const uint64_t from = (uint64_t)warp * part, to = min((uint64_t)n, from + part);
    auto load = [&](uint64_t i, int32_t (&t)[AHEAD]) {           // 32 tokens each, in order; -1 for padding and behind the warp's part
        ID raw[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) raw[k] = i + 32 * k + lane < to ? ids[i + 32 * k + lane] : (ID)-1;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) t[k] = raw[k] >= 0 && raw[k] < (ID)vocab ? (int32_t)raw[k] : -1;
    };
    int32_t kept[AHEAD];
    load(from, kept);
    uint32_t below = 0;
    for (uint64_t i = from; i < to; i += 32 * AHEAD) {
        int32_t t[AHEAD];
        if (i == from) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) t[k] = kept[k];
        } else load(i, t);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const uint32_t v = (uint32_t)t[k], owner = v & low;
            if (t[k] < 0) continue;
            if (owner < blockIdx.x) ++below;
            else if (owner == blockIdx.x) atomicAdd(mine + (v >> bits), 1u);
        }
    }
    below = __reduce_add_sync(0xFFFFFFFFu, below);
    if (lane == 0 && below) atomicAdd(&below_all, below);        // (whole numbers: any order)
    __syncthreads();
    // a thread owns a value: counts become offsets among the warps, then in the whole
    const uint32_t own = threadIdx.x;
    uint32_t total = 0;
    if (own < values)
#pragma unroll 8
        for (uint32_t w = 0; w < kOrderWarps; ++w) total += counts[w * values + own];
    uint32_t up = total;
#pragma unroll
    for (uint32_t o = 1; o < 32; o <<= 1) { const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, up, o); if (lane >= o) up += x; }
    if (lane == 31) sums[warp] = up;
    __syncthreads();
    uint32_t before = below_all + up - total + __reduce_add_sync(0xFFFFFFFFu, lane < warp ? sums[lane] : 0u);
    if (own < values) {
#pragma unroll 8
        for (uint32_t w = 0; w < kOrderWarps; ++w) { const uint32_t c = counts[w * values + own]; counts[w * values + own] = before; before += c; }
        const uint64_t v = ((uint64_t)own << bits) + blockIdx.x;
        if (v < vocab) ends[v] = before;
        if (own == values - 1 && blockIdx.x == low) *count = before;
    }
    __syncthreads();
    for (uint64_t i = from; i < to; i += 32 * AHEAD) {
        int32_t t[AHEAD];
        if (i == from) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) t[k] = kept[k];
        } else load(i, t);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const bool in = t[k] >= 0 && ((uint32_t)t[k] & low) == blockIdx.x;
            const uint32_t some = __ballot_sync(0xFFFFFFFFu, in);
            if (!some) continue;
            if (in) {
                const uint32_t v = (uint32_t)t[k] >> bits, same = __match_any_sync(some, v), rank = __popc(same & ((1u << lane) - 1u)), base = mine[v];
                sorted[base + rank] = make_uint2((uint32_t)(i + 32 * k + lane), (uint32_t)t[k]);
                __syncwarp(some);
                if (rank == 0) mine[v] = base + __popc(same);
            }
            __syncwarp();
        }
    }
}

// ---- gradient: sums --------------------------------------------------------------------------------------
// Places a chunk: the most of 8, 16, 32 or 64 that leave eight CTAs an SM (8192 places of 768 columns 41.9 us with 8, 44.4 with 16; 16384 of 4096
// columns 76 with 8, 69 with 16; 2048 of 4096 20.5 and 22.7), because each chunk leaves up to two pieces; more where there would be more than kChunksMost, which
// bounds the workspace.
constexpr uint32_t kChunksMost = 16 * kPartSms;
uint32_t sum_chunk(uint64_t n, uint32_t cols) {
    uint64_t chunk = 8;
    while (chunk < 64 && n / (2 * chunk) * ((cols + 2047u) / 2048u) >= 8 * kPartSms) chunk *= 2;
    return (uint32_t)std::max<uint64_t>(chunk, (n + kChunksMost - 1) / kChunksMost);
}

struct Ordered {                    // what the order kernel left
    const uint32_t* ends;           // [token]
    const uint32_t* count;
    const uint2* sorted;
    uint2* runs;                    // [chunk]: token and number of pieces of the run that begins in the chunk and goes on (0 pieces: none)
    float* parts;                   // [2 chunk + 0: the run that began before the chunk, 1: the run that begins in it and goes on][cols]
    uint32_t chunk, chunks;
};
// rows of dy under way: 128 bytes a thread, and as much of the table's rows where they are added to
template <typename X, bool ADD> constexpr int kRowsAhead = sizeof(X) == 2 && !ADD ? 8 : 4;

// What a thread holds of a row: 8 columns in a group (wide), or four of `step` columns apart, of which there are `left` more.
struct Span { uint32_t step, left; };
template <typename T, bool WIDE> struct Cols;
template <typename T> struct Cols<T, true> {
    Raw8<T> r;
    __device__ __forceinline__ void load(const T* p, Span) {
#pragma unroll
        for (int k = 0; k < (int)(sizeof(r.w) / 16); ++k) r.w[k] = reinterpret_cast<const uint4*>(p)[k];
    }
};
template <typename T> struct Cols<T, false> {
    T r[4];
    __device__ __forceinline__ void load(const T* p, Span s) {
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) if (k * s.step < s.left) r[k] = p[k * s.step];
    }
};
template <bool WIDE> struct Acc;
template <> struct Acc<true> {
    F2 v[4];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = f2(0.f, 0.f);
    }
    template <typename T> __device__ __forceinline__ void add(const Cols<T, true>& c) {
        F2 x[4];
        unpack8(c.r, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = add2(v[i], x[i]);
    }
    __device__ __forceinline__ void scale(float s) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], f2(s, s));
    }
    template <typename T> __device__ __forceinline__ void store(T* p, Span) const { store8(p, v); }
};
template <> struct Acc<false> {
    float v[4];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = 0.f;
    }
    template <typename T> __device__ __forceinline__ void add(const Cols<T, false>& c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += to_f32(c.r[i]);      // (columns that do not exist: anything, and never stored)
    }
    __device__ __forceinline__ void scale(float s) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= s;
    }
    template <typename T> __device__ __forceinline__ void store(T* p, Span s) const {
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) if (k * s.step < s.left) p[k * s.step] = from_f32<T>(v[k]);
    }
};

template <typename X, typename D, bool WIDE, bool ADD>
__global__ void __launch_bounds__(256) embedding_sum_kernel(const __grid_constant__ cleave_embedding_backward_t d, const __grid_constant__ Ordered o) {
    constexpr uint32_t W = WIDE ? 8 : 1, C = WIDE ? 8 : 4;       // a thread's first column after its neighbour's; columns a thread
    constexpr int N = kRowsAhead<X, ADD>;
    begin_chained();
    const uint32_t lane = threadIdx.x & 31u, columns = gridDim.y * blockDim.x * C, n = (uint32_t)d.n, first = blockIdx.x * o.chunk, most = min(n, first + o.chunk);
    // a lane looks at a place: its row, its token, the next place's token (behind the last token's place stands nothing in particular)
    auto look = [&](uint32_t p, uint2& here, uint32_t& next) {
        here = p < most ? o.sorted[p] : make_uint2(0u, 0u);
        next = p + 1 < n ? o.sorted[p + 1].y : 0u;
    };
    uint2 here;
    uint32_t next;
    look(first + lane, here, next);
    const uint32_t ahead = first ? o.sorted[first - 1].y : 0u, total = *o.count, last = min(total, most);
    if (first >= last) {
        if (blockIdx.y == 0 && threadIdx.x == 0) o.runs[blockIdx.x] = make_uint2(0u, 0u);
        return;
    }
    const bool began = first > 0 && ahead == __shfl_sync(0xFFFFFFFFu, here.y, 0);            // the first run began before the chunk
    for (uint32_t j = blockIdx.y * blockDim.x * C + threadIdx.x * W; j - lane * W < d.cols; j += columns) {       // (a warp stays together)
        const bool live = j < d.cols;
        const Span span = {blockDim.x, live ? d.cols - j : 0u};
        const X* dy = static_cast<const X*>(d.dy) + j;
        D* dt = static_cast<D*>(d.dtable) + j;
        Acc<WIDE> acc;
        acc.clear();
        bool before = began, open = false;                       // open: the run goes on at the end of the chunk
        uint32_t token = 0;
        for (uint32_t base = first; base < last; base += 32) {
            if (o.chunk > 32) look(base + lane, here, next);
            const uint32_t p = base + lane, count = min(32u, last - base), stops = __ballot_sync(0xFFFFFFFFu, p < last && (p + 1 >= total || next != here.y));
            for (uint32_t i = 0; i < count; i += N) {
                Cols<X, WIDE> x[N];
                Cols<D, WIDE> old[ADD ? N : 1];
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const uint32_t row = __shfl_sync(0xFFFFFFFFu, here.x, (i + k) & 31u), v = __shfl_sync(0xFFFFFFFFu, here.y, (i + k) & 31u);
                    if (!live || i + k >= count) continue;
                    x[k].load(dy + (uint64_t)row * d.lddy, span);
                    if (ADD && (stops >> (i + k) & 1u)) old[ADD ? k : 0].load(dt + (uint64_t)v * d.lddt, span);      // (not used where the run's other piece is missing)
                }
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const uint32_t v = __shfl_sync(0xFFFFFFFFu, here.y, (i + k) & 31u);
                    if (i + k >= count) continue;
                    token = v;
                    open = !(stops >> (i + k) & 1u);
                    if (live) {
                        acc.add(x[k]);
                        if (!open) {
                            if (before) acc.store(o.parts + (uint64_t)blockIdx.x * 2 * d.cols + j, span);
                            else {
                                acc.scale(d.scale);
                                if (ADD) acc.add(old[ADD ? k : 0]);
                                acc.store(dt + (uint64_t)v * d.lddt, span);
                            }
                            acc.clear();
                        }
                    }
                    if (!open) before = false;
                }
            }
        }
        if (open && live) acc.store(o.parts + ((uint64_t)blockIdx.x * 2 + (before ? 0 : 1)) * d.cols + j, span);
        if (j == 0) o.runs[blockIdx.x] = make_uint2(token, open && !before ? (o.ends[token] - 1) / o.chunk - blockIdx.x + 1 : 0u);
    }
}

// A CTA looks at 8 chunks for runs that begin in a chunk and go on.  A warp adds the pieces of its chunk's run in order; a run of
// more than kLongRun pieces is left to all warps (each adds every eighth piece, and the warps' sums are added in order).
constexpr uint32_t kLongRun = 6;
template <typename D, bool WIDE>
__global__ void __launch_bounds__(256, 6) embedding_join_kernel(const __grid_constant__ cleave_embedding_backward_t d, const __grid_constant__ Ordered o) {
    constexpr uint32_t W = WIDE ? 8 : 1, C = WIDE ? 8 : 4;
    __shared__ __align__(16) float s[8][32 * C];
    begin_chained();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    uint32_t v = 0, pieces = 0;                                  // of lane k < 8: the run that begins in chunk k
    if (lane < 8 && blockIdx.x * 8 + lane < o.chunks) {
        const uint2 run = o.runs[blockIdx.x * 8 + lane];
        v = run.x;
        pieces = run.y;
    }
    auto span_at = [&](uint32_t j) { return Span{32, d.cols - j}; };
    auto add = [&](Acc<WIDE>& acc, uint32_t k, uint32_t begin, uint32_t step, uint32_t end, uint32_t j) {      // pieces of the run of chunk k
        const float* from = o.parts + (uint64_t)(blockIdx.x * 8 + k) * 2 * d.cols + j;
#pragma unroll 4
        for (uint32_t c = begin; c < end; c += step) {
            Cols<float, WIDE> x;
            x.load(from + ((uint64_t)c * 2 + (c == 0 ? 1 : 0)) * d.cols, span_at(j));
            acc.add(x);
        }
    };
    auto at = [&](uint32_t token, uint32_t j) { return static_cast<D*>(d.dtable) + (uint64_t)token * d.lddt + j; };
    auto finish = [&](Acc<WIDE>& acc, const Cols<D, WIDE>& old, uint32_t token, uint32_t j) {
        acc.scale(d.scale);
        if (d.accumulate) acc.add(old);
        acc.store(at(token, j), span_at(j));
    };
    const uint32_t mine = __shfl_sync(0xFFFFFFFFu, pieces, warp), token = __shfl_sync(0xFFFFFFFFu, v, warp);
    if (mine && mine <= kLongRun)
        for (uint32_t j = blockIdx.y * 32 * C + lane * W; j < d.cols; j += gridDim.y * 32 * C) {
            Acc<WIDE> acc;
            Cols<D, WIDE> old;
            acc.clear();
            if (d.accumulate) old.load(at(token, j), span_at(j));
            add(acc, warp, 0, 1, mine, j);
            finish(acc, old, token, j);
        }
    for (uint32_t some = __ballot_sync(0xFFFFFFFFu, pieces > kLongRun); some; some &= some - 1) {
        const uint32_t k = (uint32_t)__ffs((int)some) - 1, many = __shfl_sync(0xFFFFFFFFu, pieces, k), token = __shfl_sync(0xFFFFFFFFu, v, k);
        for (uint32_t j0 = blockIdx.y * 32 * C; j0 < d.cols; j0 += gridDim.y * 32 * C) {
            const uint32_t j = j0 + lane * W;
            Acc<WIDE> acc;
            Cols<D, WIDE> old;
            acc.clear();
            if (d.accumulate && warp == 0 && j < d.cols) old.load(at(token, j), span_at(j));
            if (j < d.cols) add(acc, k, warp, 8, many, j);
            acc.store(&s[warp][lane * W], Span{32, 32 * C});
            __syncthreads();
            if (warp == 0 && j < d.cols) {
                acc.clear();
#pragma unroll
                for (uint32_t w = 0; w < 8; ++w) { Cols<float, WIDE> x; x.load(&s[w][lane * W], Span{32, 32 * C}); acc.add(x); }
                finish(acc, old, token, j);
            }
            __syncthreads();
        }
    }
}

// the workspace: the count and the ends, sorted places, runs, pieces; each begins on 16 bytes
struct Space { uint64_t sorted, runs, parts, bytes; };
static Space space_of(uint64_t n, uint32_t vocab, uint32_t cols) {
    const uint64_t chunk = sum_chunk(n, cols), chunks = (n + chunk - 1) / chunk;
    Space s;
    s.sorted = ((uint64_t)vocab + 1 + 3) / 4 * 16;
    s.runs = s.sorted + (n + 1) / 2 * 16;
    s.parts = s.runs + (chunks + 1) / 2 * 16;
    s.bytes = s.parts + chunks * 2 * cols * sizeof(float);
    return s;
}
uint64_t embedding_backward_workspace(uint64_t n, uint32_t vocab, uint32_t cols) { return space_of(n, vocab, cols).bytes; }
template <typename ID, int AHEAD>
cudaError_t launch_order(const cleave_embedding_backward_t& d, const Ordered& o, cudaStream_t st) {
    const uint32_t bits = order_owners(d.vocab), owners = 1u << bits, values = (uint32_t)(((uint64_t)d.vocab + owners - 1) >> bits);
    auto kernel = token_order_kernel<ID, AHEAD>;
    static SmemLimit limit;
    const cudaError_t e = limit.raise(reinterpret_cast<const void*>(kernel), kOrderWarps * kOrderMost * 4);
    if (e != cudaSuccess) return e;
    Zeros z = {};
    if (!d.accumulate) {
        const uint64_t b = type_bytes(d.dtable_type), rows = d.lddt == d.cols ? 1 : d.vocab;
        z = {static_cast<uint8_t*>(d.dtable), d.lddt * b, rows == 1 ? (uint64_t)d.vocab * d.cols * b : d.cols * b, 0, 0, (uint32_t)b};
        z.pieces = (z.row_bytes + kZeroPiece - 1) / kZeroPiece;
        z.tasks = z.pieces * rows;
    }
    const uint32_t zeros = (uint32_t)std::min<uint64_t>(2 * kPartSms, (z.tasks + kOrderWarps - 1) / kOrderWarps);
    return launch_chained(kernel, owners + zeros, kOrderThreads, kOrderWarps * values * 4, st, static_cast<const ID*>(d.ids), (uint32_t)d.n, d.vocab, bits, values,
                          const_cast<uint32_t*>(o.ends), const_cast<uint32_t*>(o.count), const_cast<uint2*>(o.sorted), z);
}
// as many loads under way as a warp's part of the tokens has, up to 16 (16384 tokens 8.5 us with 16, 11.7 with 8; 8192 tokens 7.7 and 6.1)
template <typename ID>
cudaError_t launch_order_ids(const cleave_embedding_backward_t& d, const Ordered& o, cudaStream_t st) {
    return d.n <= 32 * 8 * kOrderWarps ? launch_order<ID, 8>(d, o, st) : launch_order<ID, 16>(d, o, st);
}
template <typename X, typename D, bool WIDE>
cudaError_t launch_sums(const cleave_embedding_backward_t& d, const Ordered& o, cudaStream_t st) {
    if (!o.chunks) return cudaSuccess;
    const uint32_t units = WIDE ? d.cols / 8 : (d.cols + 3) / 4, tiles = std::min(65535u, (units + 255) / 256), threads = std::min(256u, ((units + tiles - 1) / tiles + 31) / 32 * 32);
    const cudaError_t e = launch_chained(d.accumulate ? embedding_sum_kernel<X, D, WIDE, true> : embedding_sum_kernel<X, D, WIDE, false>, dim3(o.chunks, tiles), threads, 0, st, d, o);
    if (e != cudaSuccess || o.chunks < 2) return e;
    return launch_chained(embedding_join_kernel<D, WIDE>, dim3((o.chunks + 7) / 8, std::min(65535u, (units + 31) / 32)), 256, 0, st, d, o);
}
template <typename X, typename D>
cudaError_t launch_sums_types(const cleave_embedding_backward_t& d, const Ordered& o, cudaStream_t st) {
    // (the pieces in the workspace stand on 16 bytes with whole groups of 8 columns)
    const bool wide = d.cols % 8 == 0 && rows_wide(d.dy, d.lddy, d.dy_type) && rows_wide(d.dtable, d.lddt, d.dtable_type);
    return wide ? launch_sums<X, D, true>(d, o, st) : launch_sums<X, D, false>(d, o, st);
}
cudaError_t launch_embedding_backward(const cleave_embedding_backward_t& d, void* ws, cudaStream_t st) {
    const Space sp = space_of(d.n, d.vocab, d.cols);
    uint8_t* w = static_cast<uint8_t*>(ws);
    uint32_t* head = reinterpret_cast<uint32_t*>(w);
    Ordered o = {head + 1, head, reinterpret_cast<const uint2*>(w + sp.sorted), reinterpret_cast<uint2*>(w + sp.runs), reinterpret_cast<float*>(w + sp.parts), sum_chunk(d.n, d.cols), 0};
    o.chunks = (uint32_t)((d.n + o.chunk - 1) / o.chunk);
    const cudaError_t e = d.id_type == CLEAVE_T_I64 ? launch_order_ids<int64_t>(d, o, st) : launch_order_ids<int32_t>(d, o, st);
    if (e != cudaSuccess) return e;
    if (d.dy_type == CLEAVE_T_F32) return d.dtable_type == CLEAVE_T_F32 ? launch_sums_types<float, float>(d, o, st) : launch_sums_types<float, __nv_bfloat16>(d, o, st);
    return d.dtable_type == CLEAVE_T_F32 ? launch_sums_types<__nv_bfloat16, float>(d, o, st) : launch_sums_types<__nv_bfloat16, __nv_bfloat16>(d, o, st);
}

}  // namespace cleave
