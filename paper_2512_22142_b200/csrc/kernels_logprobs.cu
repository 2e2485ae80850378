// Log probabilities of given tokens with entropy and top alternatives, distillation from a teacher's top scores, and the
// backward passes of both (see cleave.h).
//
// Forward: one reading of the scores.  A thread keeps a base and, relative to it, s = sum 2^a and t = sum 2^a a with
// a = c (x - base), c = scale log2(e).  The base is a score that only a score far above it replaces: then both sums are
// rescaled.  lse = scale m + ln 2 log2(s) and entropy = ln 2 (log2(s) - t / s), relative to the largest score m.
// The top places go through a bar that only rises: a score below it is dropped after one comparison (shared by 32 bytes of
// scores), the places of the others are collected by warp and, where a warp's room is full, cut to those that the bar
// has not passed, or to the best.
// A row goes to one CTA, or with few rows to a cluster of them, joined through distributed shared memory.
// Backward: each element from its score and the row's lse; one reading, one writing.
//
// Bound: the forward pass by the HBM and, beside it, instruction issue (64 % of the cycles) and exponentials (one an element, half of what
// the SM has at that rate); few rows by latency; the backward passes by the HBM.  Measured: 8192 x 50257 bf16 with entropy 141 to 158 us from
// GPU to GPU (5.2 to 5.8 TB/s; without entropy 130 to 136), the 20 best of 16 x 128000 fp32 16 us (6.3 without them), of 2048 rows 220 us;
// gradient of 8192 x 128000 bf16 628 to 645 us (6.6 TB/s; a plain copy of as many bytes takes 635); distillation, loss and gradient, 8192 x 32000 with 64
// places 267 to 281 us (5.7 TB/s).
#include <algorithm>
#include <type_traits>

#include "ptx.cuh"
#include "rows.cuh"
#include "tokens.cuh"

namespace cleave {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kMasked = -0x1p126f;             // a row whose largest score is not above this has nothing left
constexpr uint32_t kScoreThreads = 256;          // of a CTA that writes gradients
constexpr uint32_t kPartsMost = 8;               // CTAs a row in the forward passes

// ---- order of scores -----------------------------------------------------------------------------------
// whole number that orders like a score: NaN above all, +0 and -0 alike
__device__ __forceinline__ uint32_t score_order(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return x != x ? 0xFFFFFFFFu : (b & 0x80000000u ? ~b : b | 0x80000000u);
}
__device__ __forceinline__ float order_score(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }       // (NaN: some NaN)
// score, then the lower place: larger is better, no two alike, none 0 or all ones
__device__ __forceinline__ uint64_t candidate(float x, uint32_t j) { return (uint64_t)score_order(x) << 32 | (0x7FFFFFFFu - j); }
__device__ __forceinline__ uint32_t place_of(uint64_t c) { return 0x7FFFFFFFu - (uint32_t)c; }
__device__ __forceinline__ float score_of(uint64_t c) { return (uint32_t)(c >> 32) == 0xFFFFFFFFu ? __uint_as_float(0x7FFFFFFFu) : order_score((uint32_t)(c >> 32)); }

// ---- sums of a row ---------------------------------------------------------------------------------------
struct Sums {                       // m: largest score (a NaN stays); base: what the exponents are relative to, not above m, or 0 while nothing is above kMasked
    float m, base, s, t;
};
// the same sums relative to a largest score that is not below the old one
__device__ __forceinline__ void raise(Sums& a, float m, float c) {
    const float base = m <= kMasked ? 0.f : m, d = c * (a.base - base), f = a.s == 0.f ? 0.f : exp2_fast(d);
    a.t = f == 0.f ? 0.f : f * fmaf(d, a.s, a.t);
    a.s *= f;
    a.m = m;
    a.base = base;
}
__device__ __forceinline__ float warp_max_nan(float v) {
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
template <bool ENT>
__device__ __forceinline__ Sums warp_join(Sums a, float c) {
    raise(a, warp_max_nan(a.m), c);
    a.s = warp_sum(a.s);
    if (ENT) a.t = warp_sum(a.t);
    return a;
}
__device__ __forceinline__ Sums nothing() { return {-INFINITY, 0.f, 0.f, 0.f}; }
// lse, entropy, and what log p is formed from: log p = scale (x - top) - rest.  (From lse, which is rounded at its own size, it would be
// off by 7e-4 at scores of 30000, and above 0 for a sure token.)
struct Stats { float lse, entropy, top, rest; };
__device__ __forceinline__ Stats stats_of(const Sums& a, float scale, float c) {
    const float nan = __uint_as_float(0x7FFFFFFFu);
    if (a.m <= kMasked) return {-INFINITY, 0.f, 0.f, 0.f};
    if (!(a.m < INFINITY)) return {nan, nan, nan, nan};
    const float bits = log2f(a.s);
    // (the largest score's own term is 1: a sum below that is rounding)
    return {fmaf(scale, a.m, kLn2 * bits), fmaxf(kLn2 * (bits - a.t / a.s), 0.f), a.m, fmaxf(kLn2 * bits, 0.f)};
}
__device__ __forceinline__ float log_p(float x, float scale, const Stats& r) {
    if (r.lse == -INFINITY) return -INFINITY;
    return fmaf(2.f * scale, 0.5f * x - 0.5f * r.top, -r.rest);      // (halves: the difference of scores of both signs may pass fp32's range)
}

// ---- 16 bytes of scores ------------------------------------------------------------------------------------
template <typename T> constexpr int kUnit = 16 / sizeof(T);
__device__ __forceinline__ float2 pair_of(const uint4& w, int i, float) { return i == 0 ? make_float2(__uint_as_float(w.x), __uint_as_float(w.y)) : make_float2(__uint_as_float(w.z), __uint_as_float(w.w)); }
__device__ __forceinline__ float2 pair_of(const uint4& w, int i, __nv_bfloat16) {
    const uint32_t v = i == 0 ? w.x : (i == 1 ? w.y : (i == 2 ? w.z : w.w));
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}
__device__ __forceinline__ float unit_max(const uint4& w, float) {
    return max_nan(max_nan(__uint_as_float(w.x), __uint_as_float(w.y)), max_nan(__uint_as_float(w.z), __uint_as_float(w.w)));
}
__device__ __forceinline__ uint32_t max_nan_pair(uint32_t a, uint32_t b) { uint32_t r; asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }
__device__ __forceinline__ float unit_max(const uint4& w, __nv_bfloat16) {
    const uint32_t m = max_nan_pair(max_nan_pair(w.x, w.y), max_nan_pair(w.z, w.w));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
}
template <typename T, int N> __device__ __forceinline__ float units_max(const uint4 (&w)[N]) {
    if constexpr (sizeof(T) == 4) {
        float m = unit_max(w[0], T());
#pragma unroll
        for (int q = 1; q < N; ++q) m = max_nan(m, unit_max(w[q], T()));
        return m;
    } else {
        uint4 m = w[0];
#pragma unroll
        for (int q = 1; q < N; ++q) m = make_uint4(max_nan_pair(m.x, w[q].x), max_nan_pair(m.y, w[q].y), max_nan_pair(m.z, w[q].z), max_nan_pair(m.w, w[q].w));
        return unit_max(m, T());
    }
}
template <typename T> __device__ __forceinline__ uint4 masked_unit() {
    const uint32_t v = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
    return make_uint4(v, v, v, v);
}
__device__ __forceinline__ uint4 load_unit(const void* p) {      // (not kept in L1; L2 may serve the backward pass)
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
    return r;
}

// A score lifted to where 2^a is 0 but a is finite: a masked place then adds 0 a = 0 to t.  The floor lies `far` = 250 / c below the
// base, rounded down.  A NaN need not stay: the largest score has it.
template <typename T> struct Floor;
template <> struct Floor<float> {
    float at;
    __device__ __forceinline__ void set(float base, float far) { at = __fsub_rd(base, far); }
    __device__ __forceinline__ uint4 lift(const uint4& w) const {
        auto one = [&](uint32_t v) { return __float_as_uint(fmaxf(__uint_as_float(v), at)); };
        return make_uint4(one(w.x), one(w.y), one(w.z), one(w.w));
    }
};
template <> struct Floor<__nv_bfloat16> {
    uint32_t at;
    __device__ __forceinline__ void set(float base, float far) {
        const uint32_t v = __bfloat16_as_ushort(__float2bfloat16_rd(__fsub_rd(base, far)));
        at = v << 16 | v;
    }
    __device__ __forceinline__ uint4 lift(const uint4& w) const {
        auto two = [&](uint32_t v) { uint32_t r; asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(at)); return r; };
        return make_uint4(two(w.x), two(w.y), two(w.z), two(w.w));
    }
};

// which of a unit's scores reach a bar (bit i: score i): not below it, or with `tie` false above it; a NaN reaches every bar
__device__ __forceinline__ uint32_t unit_hits(const uint4& w, float bar, bool tie, float) {
    auto one = [&](uint32_t v, uint32_t bit) { const float x = __uint_as_float(v); return (tie ? x < bar : x <= bar) ? 0u : bit; };
    return one(w.x, 1u) | one(w.y, 2u) | one(w.z, 4u) | one(w.w, 8u);
}
__device__ __forceinline__ uint32_t unit_hits(const uint4& w, float bar, bool tie, __nv_bfloat16) {
    // (a bar is a bf16 value, or a little below one on the negative side: rounded towards it, it is reached by the same scores)
    const __nv_bfloat162 b = __bfloat162bfloat162(__float2bfloat16_rz(bar));
    auto two = [&](uint32_t v, uint32_t bits) {
        const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&v);
        return ~(tie ? __hlt2_mask(x, b) : __hle2_mask(x, b)) & bits;
    };
    const uint32_t m = two(w.x, 0x00020001u) | two(w.y, 0x00080004u) | two(w.z, 0x00200010u) | two(w.w, 0x00800040u);
    return (m | m >> 16) & 0xFFu;
}

// ---- the best places -----------------------------------------------------------------------------------------
constexpr uint32_t kRoom = 128;                  // candidates a warp collects before it cuts them to the best
template <int T>
struct TopRoom {
    uint32_t room[T / 32][kRoom];                // places
    uint64_t pool[(T / 32 > kPartsMost ? T / 32 : kPartsMost) * CLEAVE_TOP_MOST];      // (each warp's best, or each part's)
    uint64_t best[CLEAVE_TOP_MOST], joined[CLEAVE_TOP_MOST];
    uint32_t pooled, held;
};
// Makes room: the warp's n places without those that the bar has passed by now or, where that leaves more than `enough`, those of the best
// k candidates alone.  Returns how many there are; `last` becomes the k-th candidate where the best were taken, else 0.
template <typename T>
__device__ __noinline__ uint32_t cut(const T* x, uint32_t* room, uint32_t n, uint32_t enough, uint32_t k, uint64_t bar, uint64_t& last) {
    const uint32_t lane = threadIdx.x & 31u;
    uint64_t c[kRoom / 32];
    uint32_t rank[kRoom / 32], kept = 0;
    __syncwarp();
#pragma unroll
    for (uint32_t i = 0; i < kRoom / 32; ++i) {
        const bool live = lane + 32 * i < n;
        const uint32_t j = live ? room[lane + 32 * i] : 0u;
        c[i] = live ? candidate(to_f32(x[j]), j) : 0;
        if (c[i] <= bar) c[i] = 0;
    }
    __syncwarp();
#pragma unroll
    for (uint32_t i = 0; i < kRoom / 32; ++i) {
        const uint32_t some = __ballot_sync(0xFFFFFFFFu, c[i] != 0);
        rank[i] = kept + __popc(some & ((1u << lane) - 1u));
        kept += __popc(some);
    }
    last = 0;
    if (kept > enough) {
#pragma unroll
        for (uint32_t i = 0; i < kRoom / 32; ++i) rank[i] = 0;
#pragma unroll
        for (uint32_t i = 0; i < kRoom / 32; ++i)
            for (uint32_t l = 0; l < 32; ++l) {
                const uint64_t o = __shfl_sync(0xFFFFFFFFu, c[i], l);
#pragma unroll
                for (uint32_t e = 0; e < kRoom / 32; ++e) rank[e] += o > c[e];
            }
#pragma unroll
        for (uint32_t i = 0; i < kRoom / 32; ++i)
            if (c[i] && rank[i] == k - 1) last = c[i];
#pragma unroll
        for (int o = 16; o; o >>= 1) last = max(last, (uint64_t)__shfl_xor_sync(0xFFFFFFFFu, last, o));
        kept = min(kept, k);
    }
#pragma unroll
    for (uint32_t i = 0; i < kRoom / 32; ++i)
        if (c[i] && rank[i] < kept) room[rank[i]] = place_of(c[i]);
    __syncwarp();
    return kept;
}
// the best k of a pool of n (zeros do not count) into best[0 .. k), zeros behind them; all threads of the CTA
template <int T>
__device__ __forceinline__ void pick(const uint64_t* pool, uint32_t n, uint64_t* best, uint32_t k) {
    if (threadIdx.x < k) best[threadIdx.x] = 0;
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < n; e += T) {
        const uint64_t c = pool[e];
        if (!c) continue;
        uint32_t rank = 0;
#pragma unroll 8
        for (uint32_t j = 0; j < n; ++j) rank += pool[j] > c;
        if (rank < k) best[rank] = c;
    }
    __syncthreads();
}

// the best k of `lists` lists of k candidates each, best first with zeros at their ends, into best[0 .. k): a candidate's rank is its place in
// its own list and, by bisection, the number of better ones in each other
template <int T>
__device__ __forceinline__ void merge(const uint64_t* pool, uint32_t lists, uint64_t* best, uint32_t k) {
    if (threadIdx.x < k) best[threadIdx.x] = 0;
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < lists * k; e += T) {
        const uint64_t c = pool[e];
        const uint32_t own = e / k;
        uint32_t rank = e - own * k;
        if (!c) continue;
        for (uint32_t l = 0; l < lists && rank < k; ++l) {
            if (l == own) continue;
            uint32_t lo = 0, hi = k;                             // how many of list l are better than c
            while (lo < hi) { const uint32_t mid = (lo + hi) / 2; if (pool[l * k + mid] > c) lo = mid + 1; else hi = mid; }
            rank += lo;
        }
        if (rank < k) best[rank] = c;
    }
    __syncthreads();
}

// ---- forward ---------------------------------------------------------------------------------------------------
// Threads an SM: 48 registers each, 64 with top places; units a thread takes at once, with as many again under way: 3, 2 with top places.
// (8192 x 50257 with entropy 143 us; two units and 1536 threads 146, four and 1024 148.  4096 rows in fp32 126, 135 and 126; 600 rows of bf16 17, 20
// and 23.  The 20 best of 2048 x 128000 fp32 220 with two units, 280 with three.)
constexpr int kSumThreads = 1280, kTopThreads = 1024;
constexpr float kSlack = 8.f;

// The CTA's part (rank `part` of `parts`) of a row: its sums, joined over the CTA (every thread receives them), and with TOP its
// best `top` candidates in room->best.
template <typename T, bool ENT, bool TOP, int THREADS>
__device__ __forceinline__ Sums row_part(const T* x, uint32_t cols, float c, uint32_t part, uint32_t parts, Sums* warps, TopRoom<THREADS>* top_room, uint32_t top) {
    constexpr int V = kUnit<T>, kSteps = TOP ? 2 : 3;
    constexpr uint32_t kScoreThreads = THREADS;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5;
    // the row's units stand on 16 bytes; what is before them and behind them (less than a unit each) goes to threads of
    // the first and the last part
    const uint32_t head = min(cols, (uint32_t)((0u - (uint32_t)(uintptr_t)x) % 16u) / (uint32_t)sizeof(T)), units = (cols - head) / V, tail = cols - head - units * V;
    const uint32_t each = (units + parts - 1) / parts, begin = min(units, part * each), end = min(units, begin + each);
    const T* body = x + head;
    uint32_t edge = cols;                                        // the place of this thread's single score
    if (part == 0 && tid < head) edge = tid;
    if (part == parts - 1 && tid >= 32u && tid - 32u < tail) edge = cols - tail + (tid - 32u);
    float lone = -INFINITY;
    constexpr uint32_t kStride = kScoreThreads * kSteps;         // units a step of the CTA
    const uint32_t steps = (end - begin + kStride - 1) / kStride;                // (the same for every thread)
    const uint32_t whole = (end - begin) / kStride;              // steps in which every thread has all of its units
    const T* from = body + (uint64_t)(begin + tid) * V;
    struct Step { uint4 w[kSteps]; };
    auto fetch = [&](Step& b, uint32_t step) {
        if (step < whole) {
#pragma unroll
            for (int q = 0; q < kSteps; ++q) b.w[q] = load_unit(from + q * kScoreThreads * V);
        } else {
#pragma unroll
            for (int q = 0; q < kSteps; ++q) b.w[q] = begin + step * kStride + tid + q * kScoreThreads < end ? load_unit(from + q * kScoreThreads * V) : masked_unit<T>();
        }
        from += (uint64_t)kStride * V;
    };
    Step even, odd;
    fetch(even, 0);
    if (edge < cols) lone = to_f32(x[edge]);

    Sums a = nothing();
    F2 s2 = f2(0.f, 0.f), t2 = f2(0.f, 0.f);
    const F2 c2 = f2(c, c);
    // The base follows the largest score only when 2^kSlack is passed: after its first units a thread hardly ever rescales, and
    // what t and log2(s) cancel of each other stays below log2 of a vocabulary's size.
    const float far = ENT ? __fdiv_ru(250.f, c) : 0.f, slack = kSlack / c;
    float limit = -INFINITY;                                     // what m may reach without a new base
    Floor<T> floor;
    floor.set(0.f, far);
    // TOP.  When `top` threads have seen a score of at least v, nothing below v is among the best: the largest such v, to 16 bits, is
    // the bar, found bit by bit from the threads' largest scores and raised each time there are four times as many steps.  What reaches it goes to the
    // warp's room; a room that would run over is cut to its best, the last of which is a bar of the warp's own.
    uint32_t held = 0;
    uint64_t bar = 0;                                            // (candidates above it may be among the best)
    float bar_score = -INFINITY;
    uint32_t* room = TOP ? top_room->room[warp] : nullptr;
    auto raise_bar = [&](uint64_t b) {
        if (b > bar) { bar = b; bar_score = score_of(b); }
    };
    auto common_bar = [&](float most) {                          // all threads of the CTA
        const uint32_t mine = score_order(most);                 // (a thread that has seen nothing has -infinity, below which nothing is)
        uint32_t least = 0;
#pragma unroll 1
        for (uint32_t bit = 1u << 31; bit >= 1u << 16; bit >>= 1)
            if ((uint32_t)__syncthreads_count(mine >= (least | bit)) >= top) least |= bit;
        raise_bar((uint64_t)least << 32);                        // (below every candidate of that score)
    };
    auto offer = [&](bool good, uint32_t j) {                    // one place a lane; all lanes of the warp
        const uint32_t some = __ballot_sync(0xFFFFFFFFu, good), n = __popc(some);
        if (held + n > kRoom) {
            uint64_t last;
            held = cut(x, room, held, kRoom - 32, top, bar, last);
            if (last) raise_bar(last - 1);
        }
        if (good) room[held + __popc(some & ((1u << lane) - 1u))] = j;
        held += n;
    };
    // (an equal score counts only where it can stand before the bar's place: a row of few different scores, masked ones most of
    // all, is not offered again and again)
    auto ties = [&](uint32_t step) { return place_of(bar) >= head + (begin + step * kStride) * V; };
    auto reaches = [&](float v, bool tie) { return !(v < bar_score) && (tie || v != bar_score); };           // (a NaN reaches every bar)
    auto offer_step = [&](const Step& b, uint32_t step) {
        const uint32_t at = begin + step * kStride + tid;
        uint32_t hits;
        auto count = [&] {
            const bool tie = ties(step);
            hits = 0;
#pragma unroll
            for (int q = 0; q < kSteps; ++q)
                if (at + q * kScoreThreads < end) hits |= unit_hits(b.w[q], bar_score, tie, T()) << (q * V);
            return __reduce_add_sync(0xFFFFFFFFu, (uint32_t)__popc(hits));
        };
        if (count() > kRoom - held) {                            // more than the room takes: a bar from the step's own units first
            uint32_t least = 0, most[kSteps];
#pragma unroll
            for (int q = 0; q < kSteps; ++q) most[q] = score_order(unit_max(b.w[q], T()));
#pragma unroll 1
            for (uint32_t bit = 1u << 31; bit >= 1u << 16; bit >>= 1) {
                uint32_t many = 0;
#pragma unroll
                for (int q = 0; q < kSteps; ++q) many += __popc(__ballot_sync(0xFFFFFFFFu, most[q] >= (least | bit)));
                if (many >= top) least |= bit;
            }
            raise_bar((uint64_t)least << 32);
            count();
        }
        while (__any_sync(0xFFFFFFFFu, hits != 0)) {             // (once or twice)
            const uint32_t e = (uint32_t)__ffs((int)hits) - 1, q = e / V;
            offer(hits != 0, head + (at + q * kScoreThreads) * V + e - q * V);
            hits &= hits - 1;
        }
    };
    if (TOP) {
        if (tid == 0) top_room->pooled = top_room->held = 0;
        common_bar(max_nan(lone, units_max<T>(even.w)));
        offer(edge < cols && reaches(lone, true), edge);
    }
    if (edge < cols) {
        raise(a, lone, c);
        a.s = lone <= kMasked ? 0.f : 1.f;                       // 2^0 at its own base
        floor.set(a.base, far);
        limit = lone <= kMasked ? kMasked : a.base + slack;
    }
    auto take = [&](const Step& b, uint32_t step) {
        const float most = units_max<T>(b.w), m = max_nan(a.m, most);
        if (TOP && __any_sync(0xFFFFFFFFu, reaches(most, ties(step)))) offer_step(b, step);
        if (!(m <= limit)) {
            const float2 s0 = halves(s2), t0 = halves(t2);
            a.s += s0.x + s0.y;
            a.t += t0.x + t0.y;
            raise(a, m, c);
            s2 = t2 = f2(0.f, 0.f);
            floor.set(a.base, far);
            limit = m <= kMasked ? kMasked : a.base + slack;
        }
        a.m = m;
        const F2 b2 = f2(-a.base, -a.base);
#pragma unroll
        for (int q = 0; q < kSteps; ++q) {
            if (step >= whole && begin + step * kStride + q * kScoreThreads + warp * 32 >= end) break;           // (the whole warp)
            const uint4 w = ENT ? floor.lift(b.w[q]) : b.w[q];
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float2 p = pair_of(w, i, T());
                const F2 e2 = mul2(add2(f2(p.x, p.y), b2), c2);
                const float2 e = halves(e2);
                const F2 p2 = f2(exp2_fast(e.x), exp2_fast(e.y));
                s2 = add2(s2, p2);
                if (ENT) t2 = fma2(p2, e2, t2);
            }
        }
        if (TOP && step && (step & (step + 1)) == 0 && ((step + 1) & 0x55555555u) && step + 1 < steps) common_bar(a.m);        // behind the steps 3, 15, 63, ...
    };
    for (uint32_t step = 0; step < steps; step += 2) {
        if (step + 1 < steps) fetch(odd, step + 1);
        take(even, step);
        if (step + 1 >= steps) break;
        if (step + 2 < steps) fetch(even, step + 2);
        take(odd, step + 1);
    }
    const float2 s0 = halves(s2), t0 = halves(t2);
    a.s += s0.x + s0.y;
    a.t += t0.x + t0.y;
    const float seen = a.m;
    a = warp_join<ENT>(a, c);
    if (lane == 0) warps[warp] = a;
    if (TOP && lane == 0) atomicAdd(&top_room->held, held);
    __syncthreads();
    a = lane < THREADS / 32 ? warps[lane] : nothing();
    a = warp_join<ENT>(a, c);
    if (TOP) {
        const uint32_t all = top_room->held;
        if (all > kRoom) common_bar(seen);                       // (worth its barriers where it leaves less to sort)
        if (all > THREADS / 32 * CLEAVE_TOP_MOST) { uint64_t last; held = cut(x, room, held, CLEAVE_TOP_MOST, top, bar, last); }       // more than the pool has room for
        __syncwarp();
        for (uint32_t i = lane; i < held; i += 32) {
            const uint64_t c = candidate(to_f32(x[room[i]]), room[i]);
            if (c > bar) top_room->pool[atomicAdd(&top_room->pooled, 1u)] = c;       // (in any order: none are alike)
        }
        __syncthreads();
        pick<THREADS>(top_room->pool, top_room->pooled, top_room->best, top);
    }
    return a;
}

// joins the parts of a row over its cluster; every thread of the CTA with rank 0 receives the sums
template <bool ENT>
__device__ __forceinline__ Sums cluster_join(Sums a, float c, uint32_t rank, uint32_t parts, Sums* shared) {
    if (threadIdx.x == 0) *shared = a;
    cluster_arrive_wait();
    if (rank == 0) {
        const uint32_t lane = threadIdx.x & 31u;
        a = nothing();
        if (lane < parts) {
            const uint32_t at = mapa_shared((uint32_t)__cvta_generic_to_shared(shared), lane);
            a = {ld_dsmem(at), ld_dsmem(at + 4), ld_dsmem(at + 8), ld_dsmem(at + 12)};
        }
        a = warp_join<ENT>(a, c);
    }
    return a;
}
__device__ __forceinline__ uint64_t ld_dsmem_u64(uint32_t at) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
    return v;
}

template <typename T, bool ENT, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS, TOP ? kTopThreads / THREADS : kSumThreads / THREADS) logprobs_kernel(const __grid_constant__ cleave_logprobs_t d) {
    __shared__ Sums warps[THREADS / 32], whole;
    __shared__ typename std::conditional<TOP, TopRoom<THREADS>, int>::type top_room;
    begin_chained();
    const uint32_t part = blockIdx.x, parts = gridDim.x;
    const uint64_t row = blockIdx.y + (uint64_t)gridDim.y * blockIdx.z;
    if (row >= d.rows) return;                                   // (the whole cluster)
    const float c = d.scale * kLog2e;
    const T* x = static_cast<const T*>(d.x) + row * d.ldx;
    int32_t token = -1;                                          // (asked for ahead of the scores)
    if (d.logp && part == 0 && threadIdx.x == 0) token = load_token(d.ids, d.id_type, row, d.cols);
    TopRoom<THREADS>* top = nullptr;
    if constexpr (TOP) top = &top_room;
    Sums a = row_part<T, ENT, TOP, THREADS>(x, d.cols, c, part, parts, warps, top, d.top);
    if (parts > 1) a = cluster_join<ENT>(a, c, part, parts, &whole);
    if (part == 0) {
        if constexpr (TOP) {
            if (parts > 1) {
                const uint32_t at = (uint32_t)__cvta_generic_to_shared(top_room.best);
                for (uint32_t e = threadIdx.x; e < parts * d.top; e += THREADS) top_room.pool[e] = ld_dsmem_u64(mapa_shared(at, e / d.top) + (e % d.top) * 8);
                __syncthreads();
                merge<THREADS>(top_room.pool, parts, top_room.joined, d.top);
            }
        }
        const Stats r = stats_of(a, d.scale, c);
        if (threadIdx.x == 0) {
            if (d.lse) d.lse[row] = r.lse;
            if (ENT && d.entropy) d.entropy[row] = r.entropy;
            if (d.logp) d.logp[row] = token < 0 ? 0.f : log_p(to_f32(x[token]), d.scale, r);
        }
        if constexpr (TOP) {
            const uint64_t* best = parts > 1 ? top_room.joined : top_room.best;
            if (threadIdx.x < d.top) {
                if (d.top_index) d.top_index[row * d.ldti + threadIdx.x] = (int32_t)place_of(best[threadIdx.x]);
                if (d.top_values) d.top_values[row * d.ldtv + threadIdx.x] = log_p(score_of(best[threadIdx.x]), d.scale, r);
            }
        }
    }
    if (parts > 1) cluster_arrive_wait();                        // no CTA leaves while another reads its shared memory
}

// CTAs a row: as many as it takes, at 512 threads each, to fill the SMs once, each with 16 KB of scores at least.  (More would each
// look for places of their own: the 20 best of 292 x 128864 fp32 take 45 us, with 8 CTAs a row 85.)
uint32_t row_parts(uint64_t rows, uint64_t row_bytes, int sms, uint32_t sm_threads) {
    uint32_t parts = 1;
    while (parts < kPartsMost && rows * parts * 512 < (uint64_t)sms * sm_threads && row_bytes / (parts * 2) >= 16 * 1024) parts *= 2;
    return parts;
}
// Threads: as many as fill the SMs (16 x 128000 fp32 6.3 us with 512, 8.8 with 256); many rows go to CTAs of 128, whose joins cost
// less (8192 x 50257 with entropy 143 us against 154 with 256).  An SM holds sm_threads in CTAs of 128 or 256; of 512 without top places
// it holds 1024, which the rule does not know: 42 rows of 128000 bf16 come in two rounds of CTAs (9.4 us; with 256 threads 6.7).
struct RowGrid { dim3 cluster, grid; uint32_t threads; };
RowGrid row_grid(uint64_t rows, uint64_t row_bytes, int sms, uint32_t sm_threads) {
    const uint32_t parts = row_parts(rows, row_bytes, sms, sm_threads), y = (uint32_t)std::min<uint64_t>(rows, 65535);
    const uint64_t held = (uint64_t)sms * sm_threads / (rows * parts);       // threads a CTA if all are to run at once
    const uint32_t least = (uint32_t)std::min<uint64_t>(row_bytes / parts / 32, 512);        // two units each at least
    const uint64_t most = std::min<uint64_t>(held, least);
    return {dim3(parts), dim3(parts, y, (unsigned)((rows + y - 1) / y)), most >= 512 ? 512u : (most >= 256 ? 256u : 128u)};
}
template <typename T, bool ENT, bool TOP>
cudaError_t launch_logprobs_kernel(const cleave_logprobs_t& d, const RowGrid& g, cudaStream_t st) {
    auto kernel = g.threads == 512 ? logprobs_kernel<T, ENT, TOP, 512> : (g.threads == 256 ? logprobs_kernel<T, ENT, TOP, 256> : logprobs_kernel<T, ENT, TOP, 128>);
    return launch_chained_clusters(kernel, g.cluster, g.grid, g.threads, 0, st, d);
}
template <typename T, bool ENT>
cudaError_t launch_logprobs_types(const cleave_logprobs_t& d, const RowGrid& g, cudaStream_t st) {
    return d.top ? launch_logprobs_kernel<T, ENT, true>(d, g, st) : launch_logprobs_kernel<T, ENT, false>(d, g, st);
}
cudaError_t launch_logprobs(const cleave_logprobs_t& d, int sms, cudaStream_t st) {
    const RowGrid g = row_grid(d.rows, (uint64_t)d.cols * type_bytes(d.x_type), sms, d.top ? kTopThreads : kSumThreads);
    if (d.x_type == CLEAVE_T_F32) return d.entropy ? launch_logprobs_types<float, true>(d, g, st) : launch_logprobs_types<float, false>(d, g, st);
    return d.entropy ? launch_logprobs_types<__nv_bfloat16, true>(d, g, st) : launch_logprobs_types<__nv_bfloat16, false>(d, g, st);
}

// ---- gradients -----------------------------------------------------------------------------------------
// dx_j = s (a p_j + b p_j log p_j - [what the row's named places hold]).  A row of which nothing is asked (a = b = 0 and no
// place) is zeros whatever stands in it: padded rows may hold anything.  Rows are taken from the last to the first: the last
// ones are what L2 still holds of the forward pass.
struct RowSlope { float lse, a, b; };            // a and b with the scale
template <bool ENT>
__device__ __forceinline__ float slope_at(float x, float scale, const RowSlope& g) {
    float t = fmaf(scale, x, -g.lse);
    if (ENT) { t = max_nan(t, -200.f); return fmaf(g.b, t, g.a) * exp2_fast(t * kLog2e); }      // (p is 0 there, and so is p log p)
    return g.a * exp2_fast(t * kLog2e);
}
template <bool ENT>
__device__ __forceinline__ F2 slope_at(F2 x, F2 scale, const RowSlope& g) {
    F2 t = fma2(scale, x, f2(-g.lse, -g.lse));
    if (ENT) { const float2 h = halves(t); t = f2(max_nan(h.x, -200.f), max_nan(h.y, -200.f)); }
    const float2 e = halves(mul2(t, f2(kLog2e, kLog2e)));
    const F2 p = f2(exp2_fast(e.x), exp2_fast(e.y));
    return ENT ? mul2(fma2(f2(g.b, g.b), t, f2(g.a, g.a)), p) : mul2(f2(g.a, g.a), p);
}
// The columns of a row that a CTA writes.  Wide: groups of 8 that stand on 16 bytes in x and in dx; what is before and behind
// them (less than a group each) goes to the first and the last part.
struct Part { uint32_t head, tail, begin, end; };        // wide: groups; else columns
template <typename X, typename D, bool WIDE>
__device__ __forceinline__ Part row_columns(const X* x, const D* dx, uint32_t cols, uint32_t part, uint32_t parts) {
    if (!WIDE) {
        const uint32_t each = (cols + parts - 1) / parts, begin = min(cols, part * each);
        return {0u, 0u, begin, min(cols, begin + each)};
    }
    // (the operand of 2 bytes says where a group begins; the other one agrees, or the form would not have been chosen)
    const uint32_t at = sizeof(X) == 2 ? (uint32_t)((uintptr_t)x / 2 % 8) : (sizeof(D) == 2 ? (uint32_t)((uintptr_t)dx / 2 % 8) : (uint32_t)((uintptr_t)x / 4 % 4));
    const uint32_t head = min(cols, (0u - at) % (sizeof(X) == 2 || sizeof(D) == 2 ? 8u : 4u)), groups = (cols - head) / 8;
    const uint32_t each = (groups + parts - 1) / parts, begin = min(groups, part * each);
    return {part == 0 ? head : 0u, part == parts - 1 ? cols - head - groups * 8 : 0u, begin, min(groups, begin + each)};
}
// Writes a part.  `slope` is asked for once the first scores are on their way; it may hold barriers.  `fix(j, y)` may change what
// is stored in column j.
template <typename X, typename D, bool ENT, bool WIDE, typename SLOPE, typename FIX>
__device__ __forceinline__ void write_part(const X* x, D* dx, uint32_t cols, float scale, uint32_t part, uint32_t parts, SLOPE&& slope, FIX&& fix) {
    constexpr int N = WIDE ? (sizeof(X) == 2 ? 4 : 2) : 8;       // groups, or columns, that a thread has in flight
    const uint32_t tid = threadIdx.x;
    const Part p = row_columns<X, D, WIDE>(x, dx, cols, part, parts);
    using Raw = typename std::conditional<WIDE, Raw8<X>, X>::type;
    Raw next[N];
    uint32_t edge = cols;
    float lone = 0.f;
    const uint32_t first = WIDE && p.head == 0 ? row_columns<X, D, WIDE>(x, dx, cols, 0, 1).head : p.head;       // where group 0 begins
    auto fetch = [&](uint32_t at) {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const uint32_t k = at + q * kScoreThreads;
            if (k >= p.end) continue;
            if constexpr (WIDE) {
                const uint4* from = reinterpret_cast<const uint4*>(x + first + (uint64_t)k * 8);
#pragma unroll
                for (int i = 0; i < (int)(sizeof(Raw) / 16); ++i) next[q].w[i] = load_unit(from + i);
            } else next[q] = x[k];
        }
    };
    fetch(p.begin + tid);
    if (WIDE) {
        if (tid < p.head) edge = tid;
        if (tid >= 32u && tid - 32u < p.tail) edge = cols - p.tail + (tid - 32u);
        if (edge < cols) lone = to_f32(x[edge]);
    }
    const RowSlope g = slope();
    const bool zeros = g.lse == -INFINITY || (g.a == 0.f && g.b == 0.f);
    const F2 scale2 = f2(scale, scale);
    if (edge < cols) dx[edge] = from_f32<D>(fix(edge, zeros ? 0.f : slope_at<ENT>(lone, scale, g)));
    for (uint32_t u = p.begin + tid; u < p.end; u += N * kScoreThreads) {
        Raw now[N];
#pragma unroll
        for (int q = 0; q < N; ++q) now[q] = next[q];
        if (!zeros) fetch(u + N * kScoreThreads);
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const uint32_t k = u + q * kScoreThreads;
            if (k >= p.end) continue;
            if constexpr (WIDE) {
                F2 v[4];
                unpack8(now[q], v);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = zeros ? f2(0.f, 0.f) : slope_at<ENT>(v[i], scale2, g);
                const uint32_t j = first + k * 8;
                fix(j, v);
                store8(dx + j, v);
            } else dx[k] = from_f32<D>(fix(k, zeros ? 0.f : slope_at<ENT>(to_f32(now[q]), scale, g)));
        }
    }
}
__device__ __forceinline__ uint64_t row_from_end(uint64_t rows) { return rows - 1 - (blockIdx.y + (uint64_t)gridDim.y * blockIdx.z); }      // (below 0: beyond rows)

template <typename X, typename D, bool ENT, bool WIDE>
__global__ void __launch_bounds__(kScoreThreads) logprobs_backward_kernel(const __grid_constant__ cleave_logprobs_backward_t d) {
    begin_chained();
    const uint64_t row = row_from_end(d.rows);
    if (row >= d.rows) return;
    uint32_t named = 0xFFFFFFFFu;                                // the row's token
    float up = 0.f;
    auto slope = [&] {
        const float lse = d.lse[row];
        const int32_t t = d.dlogp ? load_token(d.ids, d.id_type, row, d.cols) : -1;
        up = t < 0 ? 0.f : d.dlogp[row];
        const float dh = ENT ? d.dentropy[row] : 0.f;
        const float a = (d.dlse ? d.dlse[row] : 0.f) - up - (dh != 0.f ? dh * d.entropy[row] : 0.f);
        if (up != 0.f && lse != -INFINITY) named = (uint32_t)t;  // (a NaN counts)
        up *= d.scale;
        return RowSlope{lse, a * d.scale, -dh * d.scale};
    };
    struct Fix {
        const uint32_t& named;
        const float& up;
        __device__ float operator()(uint32_t j, float y) const { return j == named ? y + up : y; }
        __device__ void operator()(uint32_t j, F2 (&v)[4]) const {
            const uint32_t e = named - j;
            if (e < 8u) {
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) { const float2 h = halves(v[i]); v[i] = f2(e == 2 * i ? h.x + up : h.x, e == 2 * i + 1 ? h.y + up : h.y); }
            }
        }
    };
    write_part<X, D, ENT, WIDE>(static_cast<const X*>(d.x) + row * d.ldx, static_cast<D*>(d.dx) + row * d.lddx, d.cols, d.scale, blockIdx.x, gridDim.x, slope, Fix{named, up});
}

// whether rows of x and dx allow groups of 8 that stand on 16 bytes in both
bool groups_agree(const void* x, uint64_t ldx, uint32_t x_type, const void* dx, uint64_t lddx, uint32_t dx_type) {
    const uint32_t sx = type_bytes(x_type), sd = type_bytes(dx_type), unit = sx == 2 && sd == 2 ? 8 : 4;
    return ((uintptr_t)x / sx - (uintptr_t)dx / sd) % unit == 0 && (ldx - lddx) % unit == 0;
}
// Parts of a row: 32768 columns each, less where there are too few rows to fill the GPU.
dim3 backward_grid(uint64_t rows, uint32_t cols, int sms) {
    const uint64_t most = (cols + 2047u) / 2048u, wanted = (8ull * sms + rows - 1) / rows;
    const uint32_t parts = (uint32_t)std::max<uint64_t>((cols + 32767u) / 32768u, std::min(most, wanted)), y = (uint32_t)std::min<uint64_t>(rows, 65535);
    return dim3(parts, y, (unsigned)((rows + y - 1) / y));
}
template <typename X, typename D>
cudaError_t launch_logprobs_backward_types(const cleave_logprobs_backward_t& d, dim3 grid, cudaStream_t st) {
    if (groups_agree(d.x, d.ldx, d.x_type, d.dx, d.lddx, d.dx_type))
        return launch_chained(d.dentropy ? logprobs_backward_kernel<X, D, true, true> : logprobs_backward_kernel<X, D, false, true>, grid, kScoreThreads, 0, st, d);
    return launch_chained(d.dentropy ? logprobs_backward_kernel<X, D, true, false> : logprobs_backward_kernel<X, D, false, false>, grid, kScoreThreads, 0, st, d);
}
cudaError_t launch_logprobs_backward(const cleave_logprobs_backward_t& d, int sms, cudaStream_t st) {
    const dim3 grid = backward_grid(d.rows, d.cols, sms);
    if (d.x_type == CLEAVE_T_F32) return d.dx_type == CLEAVE_T_F32 ? launch_logprobs_backward_types<float, float>(d, grid, st) : launch_logprobs_backward_types<float, __nv_bfloat16>(d, grid, st);
    return d.dx_type == CLEAVE_T_F32 ? launch_logprobs_backward_types<__nv_bfloat16, float>(d, grid, st) : launch_logprobs_backward_types<__nv_bfloat16, __nv_bfloat16>(d, grid, st);
}

// ---- distillation ------------------------------------------------------------------------------------------
// The row's teacher: `take(k, j, q, log_q)` for the entries of this thread's share whose q is not 0, and the sum of q to every thread.
// Every warp reads the whole row (at most 8 entries a lane), so nothing waits for another warp; the entries are shared out 32 by 32.
// (Where a value is NaN or +infinity every q is NaN, those of empty entries too: an entry is empty by its place, which is no address.)
constexpr int kEntries = CLEAVE_DISTILL_MOST / 32;
template <int THREADS, typename TAKE>
__device__ __forceinline__ float teacher(const cleave_distill_t& d, uint64_t row, TAKE&& take) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    float v[kEntries], top = -INFINITY;
    int32_t j[kEntries];
#pragma unroll
    for (int i = 0; i < kEntries; ++i) {
        const uint32_t k = lane + 32 * i;
        j[i] = -1;
        v[i] = -INFINITY;
        if (k < d.k) {
            j[i] = load_token(d.index, d.index_type, row * d.ldindex + k, d.cols);
            v[i] = load_as(d.values, d.values_type, row * d.ldvalues + k);
        }
    }
#pragma unroll
    for (int i = 0; i < kEntries; ++i) {
        v[i] = j[i] < 0 ? -INFINITY : d.scale * v[i];
        top = max_nan(top, v[i]);
    }
    top = d.normalize ? warp_max_nan(top) : 0.f;
    if (top == -INFINITY) return 0.f;                            // an empty row
    float e[kEntries], sum = 0.f;
#pragma unroll
    for (int i = 0; i < kEntries; ++i) { v[i] -= top; e[i] = exp2_fast(v[i] * kLog2e); sum += e[i]; }
    sum = warp_sum(sum);
    const float inv = d.normalize ? 1.f / sum : 1.f, log_sum = d.normalize ? logf(sum) : 0.f;
#pragma unroll
    for (int i = 0; i < kEntries; ++i)
        if (i % (THREADS / 32) == warp && j[i] >= 0 && e[i] * inv != 0.f) take(lane + 32 * i, (uint32_t)j[i], e[i] * inv, v[i] - log_sum);
    return sum * inv;
}
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, kSumThreads / THREADS) distill_kernel(const __grid_constant__ cleave_distill_t d) {
    __shared__ Sums warps[THREADS / 32], whole;
    __shared__ float buf[32];
    begin_chained();
    const uint32_t part = blockIdx.x, parts = gridDim.x;
    const uint64_t row = blockIdx.y + (uint64_t)gridDim.y * blockIdx.z;
    if (row >= d.rows) return;
    const float c = d.scale * kLog2e;
    const T* x = static_cast<const T*>(d.x) + row * d.ldx;
    Sums a = row_part<T, false, false, THREADS>(x, d.cols, c, part, parts, warps, nullptr, 0);
    if (parts > 1) a = cluster_join<false>(a, c, part, parts, &whole);
    if (part == 0) {
        const Stats r = stats_of(a, d.scale, c);
        float term = 0.f;
        teacher<THREADS>(d, row, [&](uint32_t, uint32_t j, float q, float log_q) {
            term = fmaf(q, log_q - log_p(to_f32(x[j]), d.scale, r), term);
        });
        term = cta_sum(term, buf);
        if (threadIdx.x == 0) {
            d.loss[row] = term;
            if (d.lse) d.lse[row] = r.lse;
        }
    }
    if (parts > 1) cluster_arrive_wait();
}
template <typename T>
cudaError_t launch_distill_types(const cleave_distill_t& d, const RowGrid& g, cudaStream_t st) {
    auto kernel = g.threads == 512 ? distill_kernel<T, 512> : (g.threads == 256 ? distill_kernel<T, 256> : distill_kernel<T, 128>);
    return launch_chained_clusters(kernel, g.cluster, g.grid, g.threads, 0, st, d);
}
cudaError_t launch_distill(const cleave_distill_t& d, int sms, cudaStream_t st) {
    const RowGrid g = row_grid(d.rows, (uint64_t)d.cols * type_bytes(d.x_type), sms, kSumThreads);
    return d.x_type == CLEAVE_T_F32 ? launch_distill_types<float>(d, g, st) : launch_distill_types<__nv_bfloat16>(d, g, st);
}
template <typename X, typename D, bool WIDE>
__global__ void __launch_bounds__(kScoreThreads) distill_backward_kernel(const __grid_constant__ cleave_distill_backward_t d) {
    __shared__ uint32_t places[CLEAVE_DISTILL_MOST];
    __shared__ float weights[CLEAVE_DISTILL_MOST];
    begin_chained();
    const uint64_t row = row_from_end(d.f.rows);
    if (row >= d.f.rows) return;
    const X* x = static_cast<const X*>(d.f.x) + row * d.f.ldx;
    D* dx = static_cast<D*>(d.dx) + row * d.lddx;
    // the columns of this CTA: it alone writes them, the named places among them once the rest is written, from scores that are read
    // before (dx may be x's buffer)
    const Part p = row_columns<X, D, WIDE>(x, dx, d.f.cols, blockIdx.x, gridDim.x);
    const uint32_t first = WIDE ? row_columns<X, D, WIDE>(x, dx, d.f.cols, 0, 1).head : 0u, unit = WIDE ? 8u : 1u;
    const uint32_t from = first + p.begin * unit - p.head, to = first + p.end * unit + p.tail;
    bool named = false;
    uint32_t place = 0;
    float own = 0.f;
    auto slope = [&] {
        const float lse = d.f.lse[row], up = d.dloss[row];
        if (threadIdx.x < d.f.k) places[threadIdx.x] = 0xFFFFFFFFu;
        const float all = teacher<kScoreThreads>(d.f, row, [&](uint32_t k, uint32_t j, float q, float) {        // (k is threadIdx.x)
            places[k] = place = j;
            weights[k] = q;
            named = j >= from && j < to;
        });
        const RowSlope g = {lse, up == 0.f || all == 0.f ? 0.f : up * all * d.f.scale, 0.f};
        named = named && up != 0.f && lse != -INFINITY;
        float score = 0.f;
        if (named) score = to_f32(x[place]);
        __syncthreads();
        if (named) {
            float q = 0.f;
            for (uint32_t k = 0; k < d.f.k; ++k)
                if (places[k] == place) { q += weights[k]; named = named && k >= threadIdx.x; }        // of entries with the same place the first writes
            own = slope_at<false>(score, d.f.scale, g) - up * d.f.scale * q;
        }
        return g;
    };
    struct Fix {
        __device__ float operator()(uint32_t, float y) const { return y; }
        __device__ void operator()(uint32_t, F2 (&)[4]) const {}
    };
    write_part<X, D, false, WIDE>(x, dx, d.f.cols, d.f.scale, blockIdx.x, gridDim.x, slope, Fix{});
    __syncthreads();
    if (named) dx[place] = from_f32<D>(own);
}
template <typename X, typename D>
cudaError_t launch_distill_backward_types(const cleave_distill_backward_t& d, dim3 grid, cudaStream_t st) {
    return launch_chained(groups_agree(d.f.x, d.f.ldx, d.f.x_type, d.dx, d.lddx, d.dx_type) ? distill_backward_kernel<X, D, true> : distill_backward_kernel<X, D, false>, grid,
                          kScoreThreads, 0, st, d);
}
cudaError_t launch_distill_backward(const cleave_distill_backward_t& d, int sms, cudaStream_t st) {
    const dim3 grid = backward_grid(d.f.rows, d.f.cols, sms);
    if (d.f.x_type == CLEAVE_T_F32) return d.dx_type == CLEAVE_T_F32 ? launch_distill_backward_types<float, float>(d, grid, st) : launch_distill_backward_types<float, __nv_bfloat16>(d, grid, st);
    return d.dx_type == CLEAVE_T_F32 ? launch_distill_backward_types<__nv_bfloat16, float>(d, grid, st) : launch_distill_backward_types<__nv_bfloat16, __nv_bfloat16>(d, grid, st);
}

}  // namespace cleave
