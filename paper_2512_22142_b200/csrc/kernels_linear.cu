// Matrix product with an epilogue (see cleave.h): z = scale_a scale_b (op(A) op(B)) + bias, C = act(z) mul + res.
//
// linear_split_kernel: one 128 x 128 tile of C per cluster of S = 1, 2, 4 or 8 CTAs; each CTA runs a K-range of the
// tile (TMA loads into a ring of 128-byte-swizzled stages, one thread issuing tcgen05.mma, the accumulator in tensor
// memory), then the S accumulators are laid into the CTAs' own shared memory and CTA r adds columns r * 128 / S ... of
// all of them, in the order of the K-ranges, through distributed shared memory.  So a product of few rows is spread
// over the whole GPU -- its time is the weights' bytes, which need every SM's loads in flight -- without a
// workspace, a second launch or an order that changes.  Two CTAs share an SM: the write-out of one runs beside the
// products of the other.
//
// linear_pair_kernel: tiles of 256 x 256 on pairs of CTAs, persistent, for large products (its comment below).
//
// Bound by: the weights' bytes and the latency of one pass (few rows: 16 x 4096 x 4096 takes 12.3 us after another, 13.0 with
// bias and residual, its 34 MB 5.2 us at the measured copy rate); the write-out beside the products (8192 x 768 x 3072 with
// bias, GELU and z: 52 us with inputs in turn, 43 with them in L2; products alone 27, the write-out alone 28); operands from
// L2 beside the tensor cores, and the clock that the power cap leaves (8192 x 4096 x 11008 in E4M3 with SwiGLU 305 us in short
// runs, 375 to 400 in long ones, 11008 x 8192 x 4096 into fp32 560 and 650; the tensor pipe works in 60 to 66 % of the cycles).
//
// Operands: K-contiguous or M/N-contiguous bf16 through the descriptors' major bits (no transposed copies), or
// K-contiguous E4M3 (kind::f8f6f4), 128 bytes of K a stage either way; TMA fills what lies outside a matrix with
// zeros, and nothing outside C is written.
//
// Every wait is bounded (2 s by default): a wait that runs out records it in a status word of the library, the
// CTA's roles leave, copies and MMAs in flight are given time to end, and the kernel returns.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "kernels.cuh"
#include "ops.cuh"
#include "ptx.cuh"

namespace cleave {

__device__ unsigned int g_linear_status;
static std::atomic<uint64_t> g_linear_wait_limit{2000000000ull};

constexpr uint32_t kLinTile = 128, kLinMaxStages = 5, kLinOperand = 16384, kLinStage = 2 * kLinOperand;
// K-blocks an accumulator takes before its sum moves on, in fp32 results: 32 steps of the tensor core, 512 products of bf16
// or 1024 of E4M3.  It cuts off when it adds, so one accumulator over K = 8192 (bf16) is 9.1e-6 off (operands of one
// sign: 2.5e-5), handed over 4.8e-7 at every K (5e-7).
constexpr uint32_t kLongBlocks = 8;
// Blocks of B that a CTA of linear_split_kernel asks L2 for while the kernel before still runs (16 x 4096 x 4096 right after
// another: none 13.0, three 12.5, eight 13.0 us).
constexpr uint32_t kLinAhead = 3;
constexpr uint32_t kLinThreads = 192, kLinSmem = 112 * 1024;        // two CTAs an SM

// What the write-out needs, the same for every kernel of this file.
struct Epilogue {
    uint32_t M, N;
    uint32_t c_type, bias_type, z_type, mul_type, res_type;
    uint32_t form;                  // 1, 2: C (bf16, fp32) and z (bf16) leave as bulk stores, mul and res allow 16-byte accesses; 0: any
    const float* scale_a;
    const float* scale_b;
    const void* bias;
    void* z;
    const void* mul;
    const void* res;
    void* C;
    uint64_t ldz, ldmul, ldres, ldc;
};

struct LinearParams {
    Epilogue e;
    uint32_t K_blocks, splits, tiles_n;
    uint32_t a_mn, b_mn, a_rows;    // a_rows: rows of a K-contiguous A that a stage brings
    // A stage holds B's 16 KB, then A's rows, so few rows leave room for five stages, 128 for three (16 x 4096 x 4096: three
    // stages 12.5, five 12.3 us; 1 x 11008 x 4096: 23.5, 22.3).  The product reads 128 rows of A; what stands behind those
    // that were brought only reaches accumulator rows that nobody reads.
    uint32_t stages, stage_bytes;
    unsigned long long wait_limit_ns;
};

// A warp's staging tile: 32 rows of 32 fp32, written by a lane a row (what tensor memory gives); the 16-byte groups of row r
// stand at group ^ (r & 7), so that neither a row nor a column of lanes meets bank conflicts.
__device__ __forceinline__ void stage_write(float* tile, uint32_t row, const float* v) {
    float4* base = reinterpret_cast<float4*>(tile) + row * 8u;
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) base[j ^ (row & 7u)] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
}

// The staged chunk (rows row0 ... + 31, columns col ... + 31 of the product) through the epilogue to C and z, any types,
// alignments and edges: a lane a column, so that a row's accesses are neighbours.
template <uint32_t ACT>
__device__ __forceinline__ void write_chunk_any(const Epilogue& e, const float* tile, uint32_t row0, uint32_t col, uint32_t lane) {
    const uint64_t j = col + lane;
    if (j >= e.N) return;
    const float sb = e.scale_b ? e.scale_b[j] : 1.f, bias = e.bias ? load_as(e.bias, e.bias_type, j) : 0.f;
    const uint32_t rows = min(32u, e.M - row0);
    constexpr uint32_t U = 8;                                            // rows asked for before the ones in hand are used
    uint32_t mul[U], res[U];                                             // raw words: nothing waits for a load before all are on their way
    auto column = [&](const void* p, uint32_t type, uint64_t ld, uint32_t r0, uint32_t (&x)[U]) {
        if (type == CLEAVE_T_F32) {
            const uint32_t* s = static_cast<const uint32_t*>(p) + j;
#pragma unroll
            for (uint32_t k = 0; k < U; ++k) x[k] = s[(row0 + min(r0 + k, rows - 1)) * ld];        // (rows beyond the last repeat it)
        } else {
            const uint16_t* s = static_cast<const uint16_t*>(p) + j;
#pragma unroll
            for (uint32_t k = 0; k < U; ++k) x[k] = (uint32_t)s[(row0 + min(r0 + k, rows - 1)) * ld];
        }
    };
    const uint32_t mul_shift = e.mul_type == CLEAVE_T_F32 ? 0u : 16u, res_shift = e.res_type == CLEAVE_T_F32 ? 0u : 16u;
    if (e.mul) column(e.mul, e.mul_type, e.ldmul, 0, mul);
    if (e.res) column(e.res, e.res_type, e.ldres, 0, res);
#pragma unroll 1
    for (uint32_t r0 = 0; r0 < rows; r0 += U) {
        float m[U], a[U];
#pragma unroll
        for (uint32_t k = 0; k < U; ++k) {
            m[k] = e.mul ? __uint_as_float(mul[k] << mul_shift) : 1.f;
            a[k] = e.res ? __uint_as_float(res[k] << res_shift) : 0.f;
        }
        if (e.mul) column(e.mul, e.mul_type, e.ldmul, r0 + U, mul);
        if (e.res) column(e.res, e.res_type, e.ldres, r0 + U, res);
#pragma unroll
        for (uint32_t k = 0; k < U; ++k) {
            const uint32_t r = r0 + k;
            if (r >= rows) break;
            const uint64_t row = row0 + r;
            const float x = tile[r * 32u + ((((lane >> 2) ^ (r & 7u)) << 2) | (lane & 3u))];
            const float z = x * (e.scale_a ? e.scale_a[row] : 1.f) * sb + bias;
            if (e.z) store_as(e.z, e.z_type, row * e.ldz + j, z);
            store_as(e.C, e.c_type, row * e.ldc + j, fmaf(act_value(z, ACT), m[k], a[k]));
        }
    }
}

// 32 consecutive elements of a row added to / multiplied into x; the row allows 16-byte accesses and holds them all.
template <bool MUL>
__device__ __forceinline__ void join_row32(const void* p, uint32_t type, uint64_t at, float (&x)[32]) {
    auto join = [](float& a, float b) { if constexpr (MUL) a *= b; else a += b; };
    if (type == CLEAVE_T_F32) {
        const float4* s = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
        float4 v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = s[q];
#pragma unroll
        for (int q = 0; q < 8; ++q) { join(x[4 * q], v[q].x); join(x[4 * q + 1], v[q].y); join(x[4 * q + 2], v[q].z); join(x[4 * q + 3], v[q].w); }
    } else {
        const uint4* s = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + at);
        uint4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = s[q];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t w[4] = {v[q].x, v[q].y, v[q].z, v[q].w};
#pragma unroll
            for (int h = 0; h < 4; ++h) { join(x[8 * q + 2 * h], __uint_as_float(w[h] << 16)); join(x[8 * q + 2 * h + 1], __uint_as_float(w[h] & 0xFFFF0000u)); }
        }
    }
}
// A row of a 32 x 32 chunk as a bulk tensor store wants it: fp32 rows of 128 bytes with the 128-byte swizzle, or bf16
// rows of 64 bytes with the 64-byte swizzle.
template <bool F32>
__device__ __forceinline__ void stage_out(uint8_t* buf, uint32_t row, const float (&x)[32]) {
    if constexpr (F32) stage_write(reinterpret_cast<float*>(buf), row, x);
    else {
        uint4* base = reinterpret_cast<uint4*>(buf) + row * 4u;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            base[j ^ ((row >> 1) & 3u)] = make_uint4(pack_bf16(x[8 * j], x[8 * j + 1]), pack_bf16(x[8 * j + 2], x[8 * j + 3]),
                                                     pack_bf16(x[8 * j + 4], x[8 * j + 5]), pack_bf16(x[8 * j + 6], x[8 * j + 7]));
    }
}

// A warp's output buffers: `count` of `bytes` each, taken in turn; a buffer is free again when the bulk store that read it
// (the count-th last one) has finished reading.
struct OutRing {
    uint8_t* base;
    uint32_t bytes, count, next;
    __device__ __forceinline__ uint8_t* take(uint32_t lane) {
        if (lane == 0) { if (count >= 3) asm volatile("cp.async.bulk.wait_group.read 2;" ::: "memory"); else if (count == 2) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); else bulk_wait_read_all(); }
        __syncwarp();
        uint8_t* b = base + next * bytes;
        next = next + 1 == count ? 0 : next + 1;
        return b;
    }
    __device__ __forceinline__ void store(const CUtensorMap* map, const uint8_t* buf, uint32_t col, uint32_t row, uint32_t lane) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) { tma_store_2d(map, smem_u32(buf), (int32_t)col, (int32_t)row); bulk_commit(); }
    }
    __device__ __forceinline__ void finish(uint32_t lane) { if (lane == 0) bulk_wait_all(); __syncwarp(); }
};

// A column's scale and bias, a lane a column: asked for one chunk ahead.
struct ColumnPair { float scale, bias; };
__device__ __forceinline__ ColumnPair load_columns(const Epilogue& e, uint32_t col) {
    ColumnPair p = {0.f, 0.f};
    if (col < e.N) {
        if (e.scale_b) p.scale = e.scale_b[col];
        if (e.bias) p.bias = load_as(e.bias, e.bias_type, col);
    }
    return p;
}
// One chunk, 32 columns from `col` on, a lane a row (row0 + lane), from its fp32 sums x to C (and z) through bulk stores,
// which leave out what lies beyond C's edges.
template <uint32_t ACT, bool F32>
__device__ __forceinline__ void write_rows(const Epilogue& e, const CUtensorMap* map_c, const CUtensorMap* map_z, OutRing& out, float (&x)[32], float sa,
                                           ColumnPair columns, uint32_t row0, uint32_t col, uint32_t lane) {
    uint8_t* buf = out.take(lane);
    if (e.scale_a) {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] *= sa;
    }
    if (e.scale_b || e.bias) {
        // through the (still empty) buffer to every lane
        float* vec = reinterpret_cast<float*>(buf);
        vec[lane] = columns.scale;
        vec[32 + lane] = columns.bias;
        __syncwarp();
        if (e.scale_b) {
#pragma unroll
            for (int q = 0; q < 8; ++q) { const float4 v = reinterpret_cast<const float4*>(vec)[q]; x[4 * q] *= v.x; x[4 * q + 1] *= v.y; x[4 * q + 2] *= v.z; x[4 * q + 3] *= v.w; }
        }
        if (e.bias) {
#pragma unroll
            for (int q = 0; q < 8; ++q) { const float4 v = reinterpret_cast<const float4*>(vec + 32)[q]; x[4 * q] += v.x; x[4 * q + 1] += v.y; x[4 * q + 2] += v.z; x[4 * q + 3] += v.w; }
        }
        __syncwarp();
    }
    if (e.z) {
        stage_out<false>(buf, lane, x);
        out.store(map_z, buf, col, row0, lane);
        buf = out.take(lane);
    }
    if constexpr (ACT != CLEAVE_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = act_value(x[i], ACT);
    }
    const uint64_t row = row0 + lane;
    if (row < e.M) {
        if (col + 32 <= e.N) {
            if (e.mul) join_row32<true>(e.mul, e.mul_type, row * e.ldmul + col, x);
            if (e.res) join_row32<false>(e.res, e.res_type, row * e.ldres + col, x);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 32; ++i)
                if (col + i < e.N) {
                    if (e.mul) x[i] *= load_as(e.mul, e.mul_type, row * e.ldmul + col + i);
                    if (e.res) x[i] += load_as(e.res, e.res_type, row * e.ldres + col + i);
                }
        }
    }
    stage_out<F32>(buf, lane, x);
    out.store(map_c, buf, col, row0, lane);
}
template <uint32_t ACT>
__device__ __forceinline__ void write_piece(const Epilogue& e, const CUtensorMap* map_c, const CUtensorMap* map_z, OutRing& out, float (&x)[32], float sa,
                                            ColumnPair columns, uint32_t row0, uint32_t col, uint32_t lane) {
    if (row0 >= e.M || col >= e.N) return;
    if (e.form == 1) write_rows<ACT, false>(e, map_c, map_z, out, x, sa, columns, row0, col, lane);
    else if (e.form == 2) write_rows<ACT, true>(e, map_c, map_z, out, x, sa, columns, row0, col, lane);
    else {
        float* tile = reinterpret_cast<float*>(out.base);
        stage_write(tile, lane, x);
        __syncwarp();
        write_chunk_any<ACT>(e, tile, row0, col, lane);
        __syncwarp();
    }
}
// A warp's part of the accumulator, 32 rows from row0 on, to its place in C: the chunks of 32 columns at c, c + step, ... of
// the `cols` columns that begin at tensor-memory address taddr and column col.  `ready` waits for the accumulator;
// `read` is called when the warp has read it for the last time.
template <uint32_t ACT, typename Ready, typename Read>
__device__ __forceinline__ bool write_strip(const Epilogue& e, const CUtensorMap* map_c, const CUtensorMap* map_z, OutRing& out, uint32_t taddr, uint32_t row0,
                                            uint32_t col, uint32_t c, uint32_t step, uint32_t cols, uint32_t lane, Ready ready, Read read) {
    const float sa = e.scale_a && row0 + lane < e.M ? e.scale_a[row0 + lane] : 1.f;
    ColumnPair next = load_columns(e, col + c + lane);
    if (!ready()) return false;
    if (c >= cols) read();
#pragma unroll 1
    for (; c < cols; c += step) {
        const ColumnPair columns = next;
        float x[32];
        {
            uint32_t u[32];
            tmem_ld_32x32(taddr + c, u);
            if (c + step < cols) next = load_columns(e, col + c + step + lane);
            tmem_ld_wait();
            if (c + step >= cols) read();
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(u[i]);
        }
        write_piece<ACT>(e, map_c, map_z, out, x, sa, columns, row0, col + c, lane);
    }
    return true;
}
// The rows of mul and res that a strip of 32 rows x `cols` columns will need, brought into L2 ahead of time.
__device__ __forceinline__ void prefetch_strip(const void* p, uint32_t type, uint64_t ld, const Epilogue& e, uint32_t row, uint32_t col, uint32_t cols) {
    if (!p || row >= e.M || col >= e.N) return;
    const uint32_t es = type == CLEAVE_T_F32 ? 4u : 2u;
    const uint8_t* at = static_cast<const uint8_t*>(p) + (row * ld + col) * es;
    const uint32_t bytes = min(cols, e.N - col) * es;
    for (uint32_t b = 0; b < bytes; b += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(at + b));
}

// ---- PTX of one-CTA products ---------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void* tmap, uint32_t bar, int32_t c0, int32_t c1) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(tmap), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void tma_prefetch_2d(const void* tmap, int32_t c0, int32_t c1) {
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(tmap), "r"(c0), "r"(c1) : "memory");
}
template <bool E4M3>
__device__ __forceinline__ void umma_one(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    if constexpr (E4M3)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_commit_one(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_st_32x32(uint32_t taddr, const float* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]),
          "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]),
          "f"(v[21]), "f"(v[22]), "f"(v[23]), "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]),
          "f"(v[31]), "r"(taddr) : "memory");
}
// Instruction descriptor of kind::f8f6f4: fp32 accumulator (bits 4-5 = 1), E4M3 A and B (format 0), both K-contiguous.
__device__ __forceinline__ uint32_t instr_desc_e4m3(uint32_t m, uint32_t n) { return (1u << 4) | ((n >> 3) << 17) | ((m >> 4) << 24); }

__device__ __forceinline__ void tmem_ld_32x16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr) : "memory");
}

// mbarrier.try_wait may hold the thread for microseconds, longer than many a wait here: with a limit of 0 the MMA issuer's
// first wait is asked for without holding.
__device__ __forceinline__ bool mbar_is_done(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
struct LinWait { volatile uint32_t* abort_flag; uint64_t limit_ns; };
static __device__ __noinline__ bool lin_wait_slow(uint32_t bar, uint32_t parity, const LinWait& w) {
    const uint64_t t0 = global_timer_ns();
    uint32_t spins = 0;
    while (!mbar_try_wait(bar, parity)) {
        if ((spins++ & 255u) == 0) {                     // at the first unsuccessful poll, then every 256
            if (*w.abort_flag) return false;
            if (global_timer_ns() - t0 >= w.limit_ns) { *w.abort_flag = 1u; atomicOr(&g_linear_status, STATUS_TIMEOUT); return false; }
        }
    }
    return true;
}
__device__ __forceinline__ bool lin_wait(uint32_t bar, uint32_t parity, const LinWait& w) {
    return mbar_try_wait(bar, parity) || lin_wait_slow(bar, parity, w);
}

// the same without a call (a call would have to save the caller's sums)
__device__ __forceinline__ bool lin_wait_inline(uint32_t bar, uint32_t parity, const LinWait& w) {
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = global_timer_ns();
    for (uint32_t spins = 0; !mbar_try_wait(bar, parity); ++spins)
        if ((spins & 255u) == 0) {
            if (*w.abort_flag) return false;
            if (global_timer_ns() - t0 >= w.limit_ns) { *w.abort_flag = 1u; atomicOr(&g_linear_status, STATUS_TIMEOUT); return false; }
        }
    return true;
}

struct __align__(16) LinShared {
    uint64_t full[kLinMaxStages], empty[kLinMaxStages], acc_full[2], acc_empty[2], drain;
    uint32_t tmem_base, abort_flag;
};

// LONG: the accumulator is handed over every kLongBlocks K-blocks.  Two of them take turns, 256 columns of tensor
// memory a CTA (two CTAs share an SM's 512); each of the four write-out warps keeps the sums of its 32 rows in registers,
// adds a chunk while the next one's products run, and lays the sums into the last accumulator's place at the end.
// Measured against one accumulator: 16 x 4096 x 11008 21.4 to 20.6 us, 1 x 50304 x 2048 43.7 to 41.1, 768 x 3072 x 8192
// 41.2 to 39.7.  (Sums 16 columns a load: 24 bytes spilled at the 168 registers that two CTAs an SM leave.)
template <bool E4M3, bool LONG, uint32_t ACT>
__global__ void __launch_bounds__(kLinThreads, 2)
linear_split_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_c,
                    const __grid_constant__ CUtensorMap map_z, const __grid_constant__ LinearParams P) {
    extern __shared__ uint8_t dyn_smem[];
    __shared__ LinShared sh;
    constexpr uint32_t kBlk = E4M3 ? 128u : 64u;         // K per stage: 128 bytes
    constexpr uint32_t kTmem = LONG ? 2 * kLinTile : kLinTile;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t base = (smem_u32(dyn_smem) + 1023u) & ~1023u;
    const uint32_t rank = blockIdx.x % P.splits, tile = blockIdx.x / P.splits;
    const uint32_t m0 = (tile / P.tiles_n) * kLinTile, n0 = (tile % P.tiles_n) * kLinTile;
    const uint32_t kb0 = (uint32_t)((uint64_t)P.K_blocks * rank / P.splits), kb1 = (uint32_t)((uint64_t)P.K_blocks * (rank + 1) / P.splits);
    const LinWait W = {&sh.abort_flag, P.wait_limit_ns};
    let_dependents_start();

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < P.stages; ++s) { mbar_init(smem_u32(&sh.full[s]), 1); mbar_init(smem_u32(&sh.empty[s]), 1); }
        mbar_init(smem_u32(&sh.acc_full[0]), 1);
        if constexpr (LONG) { mbar_init(smem_u32(&sh.acc_full[1]), 1); mbar_init(smem_u32(&sh.acc_empty[0]), 4); mbar_init(smem_u32(&sh.acc_empty[1]), 4); }
        mbar_init(smem_u32(&sh.drain), 1);
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (threadIdx.x == 64) {                              // (a thread of the write-out)
        prefetch_map(&map_a); prefetch_map(&map_b);
        if (P.e.form) { prefetch_map(&map_c); if (P.e.z) prefetch_map(&map_z); }
        // B's first blocks are on their way to L2 (where a later write by the kernel before reaches them) while that
        // kernel still runs
        for (uint32_t kb = kb0; kb < min(kb1, kb0 + kLinAhead); ++kb) {
            const int32_t k = (int32_t)(kb * kBlk);
            if (P.b_mn) { tma_prefetch_2d(&map_b, (int32_t)n0, k); tma_prefetch_2d(&map_b, (int32_t)n0 + 64, k); }
            else tma_prefetch_2d(&map_b, k, (int32_t)n0);
        }
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;
    wait_for_primary();

    if (warp == 0 && lane == 0) {
        // ---- producer ----
        for (uint32_t kb = kb0, s = 0, ph = 0; kb < kb1; ++kb) {
            if (!lin_wait(smem_u32(&sh.empty[s]), ph ^ 1u, W)) break;
            const uint32_t bar = smem_u32(&sh.full[s]), sb = base + s * P.stage_bytes, sa = sb + kLinOperand;
            mbar_arrive_expect_tx(bar, kLinOperand + P.a_rows * 128u);
            const int32_t k = (int32_t)(kb * kBlk);
            if (P.a_mn) { tma_load_2d(sa, &map_a, bar, (int32_t)m0, k); tma_load_2d(sa + kSubBytes, &map_a, bar, (int32_t)m0 + 64, k); }
            else tma_load_2d(sa, &map_a, bar, k, (int32_t)m0);
            if (P.b_mn) { tma_load_2d(sb, &map_b, bar, (int32_t)n0, k); tma_load_2d(sb + kSubBytes, &map_b, bar, (int32_t)n0 + 64, k); }
            else tma_load_2d(sb, &map_b, bar, k, (int32_t)n0);
            if (++s == P.stages) { s = 0; ph ^= 1u; }
        }
    } else if (warp == 1 && lane == 0) {
        // ---- MMA issuer ----
        const uint32_t idesc = E4M3 ? instr_desc_e4m3(kLinTile, kLinTile) : instr_desc_bf16(kLinTile, kLinTile, P.a_mn, P.b_mn);
        const uint32_t a_lbo = P.a_mn ? kSubBytes : 16u, a_step = P.a_mn ? 2048u : 32u;
        const uint32_t b_lbo = P.b_mn ? kSubBytes : 16u, b_step = P.b_mn ? 2048u : 32u;
        bool ok = W.limit_ns != 0 || mbar_is_done(smem_u32(&sh.full[0]), 0u);
        if (!ok) { sh.abort_flag = 1u; atomicOr(&g_linear_status, STATUS_TIMEOUT); }
        uint32_t s = 0, ph = 0;                           // stage, its phase
        auto block = [&](uint32_t d, uint32_t accumulate) {
            if (!lin_wait(smem_u32(&sh.full[s]), ph, W)) { ok = false; return; }
            tc_fence_after();
            const uint32_t sb = base + s * P.stage_bytes, sa = sb + kLinOperand;
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q)              // 32 bytes of K each
                umma_one<E4M3>(d, smem_desc_sw128(sa + q * a_step, a_lbo, 1024u), smem_desc_sw128(sb + q * b_step, b_lbo, 1024u), idesc, accumulate | (q != 0u));
            umma_commit_one(smem_u32(&sh.empty[s]));
            if (++s == P.stages) { s = 0; ph ^= 1u; }
        };
        if constexpr (LONG) {
            uint32_t use = 0;                             // accumulators used so far
            for (uint32_t k0 = kb0; ok && k0 < kb1; k0 += kLongBlocks, ++use) {
                const uint32_t acc = use & 1u;
                if (!lin_wait(smem_u32(&sh.acc_empty[acc]), ((use >> 1) & 1u) ^ 1u, W)) { ok = false; break; }
                tc_fence_after();
                for (uint32_t kb = k0; ok && kb < min(kb1, k0 + kLongBlocks); ++kb) block(tmem + acc * kLinTile, kb != k0);
                if (ok) umma_commit_one(smem_u32(&sh.acc_full[acc]));
            }
        } else {
            for (uint32_t kb = kb0; ok && kb < kb1; ++kb) block(tmem, kb != kb0);
            if (ok) umma_commit_one(smem_u32(&sh.acc_full[0]));
        }
        // everything issued above has completed before tensor memory is released
        umma_commit_one(smem_u32(&sh.drain));
        const uint64_t t0 = global_timer_ns();
        while (!mbar_try_wait(smem_u32(&sh.drain), 0u))
            if (global_timer_ns() - t0 > 2000000000ull) { atomicOr(&g_linear_status, STATUS_TIMEOUT); break; }
    }
    __syncwarp();
    // ---- write-out: warps 2..5, warp w owns the accumulator rows 32 (w % 4) ... ----
    const uint32_t quad = warp & 3u;
    bool ok = true;
    if (warp >= 2) {
        if (P.splits == 1) {                              // what the write-out reads is brought into L2 beside the products
            prefetch_strip(P.e.mul, P.e.mul_type, P.e.ldmul, P.e, m0 + quad * 32u + lane, n0, kLinTile);
            prefetch_strip(P.e.res, P.e.res_type, P.e.ldres, P.e, m0 + quad * 32u + lane, n0, kLinTile);
        } else {
            const uint32_t cols = P.splits == 2 ? 64u : 32u;
            if (rank * cols < kLinTile) {
                prefetch_strip(P.e.mul, P.e.mul_type, P.e.ldmul, P.e, m0 + quad * 32u + lane, n0 + rank * cols, cols);
                prefetch_strip(P.e.res, P.e.res_type, P.e.ldres, P.e, m0 + quad * 32u + lane, n0 + rank * cols, cols);
            }
        }
        uint32_t taddr = tmem + ((quad * 32u) << 16);
        if constexpr (LONG) {
            const bool rows = m0 + quad * 32u < P.e.M;
            float sum[kLinTile];
#pragma unroll
            for (uint32_t i = 0; i < kLinTile; ++i) sum[i] = 0.f;
            uint32_t use = 0;
            for (uint32_t k0 = kb0; k0 < kb1; k0 += kLongBlocks, ++use) {
                const uint32_t acc = use & 1u, at = taddr + acc * kLinTile;
                ok = __all_sync(0xFFFFFFFFu, lin_wait_inline(smem_u32(&sh.acc_full[acc]), (use >> 1) & 1u, W));
                if (!ok) break;
                tc_fence_after();
                if (rows) {
#pragma unroll
                    for (uint32_t c = 0; c < kLinTile; c += 16) {
                        uint32_t u[16];
                        tmem_ld_32x16(at + c, u);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[c + i] += __uint_as_float(u[i]);
                    }
                    if (k0 + kLongBlocks >= kb1) {        // nothing is accumulated here any more
#pragma unroll
                        for (uint32_t c = 0; c < kLinTile; c += 32) tmem_st_32x32(at + c, sum + c);
                        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.acc_empty[acc]));
            }
            taddr += ((use - 1u) & 1u) * kLinTile;
        } else {
            ok = __all_sync(0xFFFFFFFFu, lin_wait(smem_u32(&sh.acc_full[0]), 0u, W));
            tc_fence_after();
        }
        if (m0 + quad * 32u >= P.e.M) {
            // (no rows for this warp)
        } else if (ok && P.splits == 1) {
            OutRing out = {dyn_smem + (base - smem_u32(dyn_smem)) + (warp - 2) * 12288, 4096u, 3u, 0u};        // the stages are read
            write_strip<ACT>(P.e, &map_c, &map_z, out, taddr, m0 + quad * 32u, n0, 0u, 32u, kLinTile, lane, [] { return true; }, [] {});
            if (P.e.form) out.finish(lane);
        } else if (ok) {
            float* part = reinterpret_cast<float*>(dyn_smem + (base - smem_u32(dyn_smem)));      // the stages are read: column-major [128][128]
#pragma unroll 1
            for (uint32_t c = 0; c < kLinTile; c += 32) {
                uint32_t u[32];
                tmem_ld_32x32(taddr + c, u);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) part[(c + i) * kLinTile + quad * 32u + lane] = __uint_as_float(u[i]);
            }
        }
        tc_fence_before();
    }
    if (P.splits > 1) {
        cluster_arrive_wait();
        if (warp >= 2 && ok) {
            // (of eight CTAs the first four add: a chunk of 32 columns is the least that is written at once)
            const uint32_t cols = P.splits == 2 ? 64u : 32u, c0 = rank * cols, row0 = m0 + quad * 32u;
            OutRing out = {dyn_smem + (base - smem_u32(dyn_smem)) + 65536 + (warp - 2) * 8192, 4096u, 2u, 0u};   // behind the accumulators
            if (row0 < P.e.M) {
                const float sa = P.e.scale_a && row0 + lane < P.e.M ? P.e.scale_a[row0 + lane] : 1.f;
#pragma unroll 1
                for (uint32_t c = c0; c < min(c0 + cols, kLinTile) && n0 + c < P.e.N; c += 32) {
                    float x[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = 0.f;
#pragma unroll 1
                    for (uint32_t r = 0; r < P.splits; r += 2) {           // K-ranges in order, two asked for at a time
                        const uint32_t off = ((c * kLinTile) + quad * 32u + lane) * 4u, s0 = mapa_shared(base, r) + off, s1 = mapa_shared(base, r + 1) + off;
                        float y[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) y[i] = ld_dsmem(s0 + i * kLinTile * 4u);
                        float w[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) w[i] = ld_dsmem(s1 + i * kLinTile * 4u);
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = (x[i] + y[i]) + w[i];
                    }
                    write_piece<ACT>(P.e, &map_c, &map_z, out, x, sa, load_columns(P.e, n0 + c + lane), row0, n0 + c, lane);
                }
                if (P.e.form) out.finish(lane);
            }
        }
        cluster_arrive_wait();                            // no CTA leaves while another reads its shared memory
    }
    __syncthreads();
    if (sh.abort_flag) {                                  // a role gave up: copies may still be in flight towards this CTA
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 200000ull) { }
        __syncthreads();
    }
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmem) : "memory");
}

// ---- large products: pairs of CTAs ---------------------------------------------------------------------
// linear_pair_kernel: one persistent cluster of two CTAs per pair of SMs.  A tile is 256 rows x BN <= 256 columns; CTA
// r loads rows 128 r ... of A and columns r BN / 2 ... of B, the leader's MMA thread issues M = 256 products over both
// CTAs' shared memory (four to six stages of 32 KB each, what the output buffers leave), and each CTA finds its 128 rows in its own tensor memory, in two
// slots, so the write-out of a tile runs beside the products of the next.  Tiles go to clusters round robin, in bands
// of eight row tiles so that tiles in flight share operands in L2.
//
// LONG (fp32 results of a long K, see kLongBlocks): the accumulator is handed over every `chunk` K-blocks and the write-out
// warps keep the sum in registers with ordinary rounded additions; the two slots take turns by chunk instead of by tile.
constexpr uint32_t kLpMaxStages = 6, kLpEpiWarp0 = 4, kLpBand = 8;
// Write-out warps: 16 keep pace with the products of a short K (bias, activation and a second output: 55 -> 50 us at 8192 x 768
// x 3072 against 8); LONG takes 8, whose threads hold 128 sums each (with 16 warps 96 registers a thread are left:
// 419 -> 544 us at 8192 x 8192 x 4096; with 8 the instances still spill, 204 bytes a thread, 252 with ReLU).
__host__ __device__ constexpr uint32_t pair_warps(bool lng) { return lng ? 8u : 16u; }
__host__ __device__ constexpr uint32_t pair_threads(bool lng) { return 32u * (kLpEpiWarp0 + pair_warps(lng)); }
constexpr uint32_t kLpSmemMost = 227 * 1024 - 256;       // (what is declared statically comes on top)

struct PairParams {
    Epilogue e;
    uint32_t K_blocks, chunk, bn, b_boxes, b_bytes;      // b_bytes: what one CTA loads of B per stage
    uint32_t tiles_m, tiles_n;
    uint32_t a_mn, b_mn;                                 // 0: K-contiguous, 1: M/N-contiguous in boxes of 64, 2: in double boxes
    uint32_t stages, out_bytes, out_count;               // operand ring; output buffers of a write-out warp
    unsigned long long wait_limit_ns;
};
// mbar_wait_cl without a call (a call would have to save the caller's sums)
__device__ __forceinline__ bool pair_wait_inline(uint32_t bar, uint32_t parity, const WaitCtx& w) {
    if (mbar_try_wait_cl(bar, parity)) return true;
    const uint64_t t0 = global_timer_ns();
    for (uint32_t spins = 0; !mbar_try_wait_cl(bar, parity); ++spins)
        if ((spins & 255u) == 0) {
            if (*w.abort_flag) return false;
            if (global_timer_ns() - t0 >= w.limit_ns) { raise_abort(w); return false; }
        }
    return true;
}
struct __align__(16) LpShared {
    uint64_t full[kLpMaxStages], empty[kLpMaxStages], acc_full[2], acc_empty[2], drain;
    uint32_t tmem_base, abort_flag;
};
// tile number -> row and column tile: bands of kLpBand row tiles, column by column inside a band
__device__ __forceinline__ uint2 pair_tile(const PairParams& P, uint32_t t) {
    const uint32_t per_band = kLpBand * P.tiles_n, band = t / per_band, in = t - band * per_band;
    const uint32_t rows = min(kLpBand, P.tiles_m - band * kLpBand);
    return make_uint2(band * kLpBand + in % rows, in / rows);
}
template <bool E4M3>
__device__ __forceinline__ void umma_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    if constexpr (E4M3)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
    else umma_bf16_pair(d_tmem, a_desc, b_desc, idesc, accumulate);
}

template <bool E4M3, bool LONG, uint32_t ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(pair_threads(LONG), 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_c,
                   const __grid_constant__ CUtensorMap map_z, const __grid_constant__ PairParams P) {
    extern __shared__ uint8_t dyn_smem[];
    __shared__ LpShared sh;
    constexpr uint32_t kBlk = E4M3 ? 128u : 64u;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, rank = cluster_ctarank();
    const uint32_t base = (smem_u32(dyn_smem) + 1023u) & ~1023u;
    const uint32_t tiles = P.tiles_m * P.tiles_n, cluster = blockIdx.x >> 1, clusters = gridDim.x >> 1;
    const WaitCtx W = {&sh.abort_flag, &g_linear_status, P.wait_limit_ns};
    let_dependents_start();

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < P.stages; ++s) { mbar_init(smem_u32(&sh.full[s]), 1); mbar_init(smem_u32(&sh.empty[s]), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(smem_u32(&sh.acc_full[a]), 1); mbar_init(smem_u32(&sh.acc_empty[a]), 16); }
        mbar_init(smem_u32(&sh.drain), 1);
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(&sh.tmem_base), 512);
    tc_fence_before();
    cluster_arrive_wait();                            // barriers of both CTAs are ready before any remote arrive
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;
    wait_for_primary();

    if (warp < kLpEpiWarp0) {
        if constexpr (LONG) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");       // 128 x 40 + 256 x 216 <= 384 x 168 registers
        if (warp == 0 && lane == 0) {
            // ---- producer (both CTAs) ----
            const uint32_t full0 = mapa_shared(smem_u32(&sh.full[0]), 0u), tx = 2u * (kLinOperand + P.b_bytes);
            uint32_t s = 0, ph = 0;
            bool ok = true;
            for (uint32_t t = cluster; ok && t < tiles; t += clusters) {
                const uint2 at = pair_tile(P, t);
                const int32_t m = (int32_t)(at.x * 256u + rank * 128u), n = (int32_t)(at.y * P.bn + rank * (P.bn / 2));
                for (uint32_t kb = 0; kb < P.K_blocks; ++kb) {
                    if (!mbar_wait_cl(smem_u32(&sh.empty[s]), ph ^ 1u, W)) { ok = false; break; }
                    if (rank == 0) mbar_arrive_expect_tx(smem_u32(&sh.full[s]), tx);
                    const uint32_t bar = full0 + s * 8u, sa = base + s * kLinStage, sb = sa + kLinOperand;
                    const int32_t k = (int32_t)(kb * kBlk);
                    if (P.a_mn == 2) tma_load_3d_pair(sa, &map_a, bar, 0, k, m / 64);
                    else if (P.a_mn) { tma_load_2d_pair(sa, &map_a, bar, m, k); tma_load_2d_pair(sa + kSubBytes, &map_a, bar, m + 64, k); }
                    else tma_load_2d_pair(sa, &map_a, bar, k, m);
                    if (P.b_mn == 2) tma_load_3d_pair(sb, &map_b, bar, 0, k, n / 64);
                    else if (P.b_mn) for (uint32_t j = 0; j < P.b_boxes; ++j) tma_load_2d_pair(sb + j * kSubBytes, &map_b, bar, n + 64 * (int32_t)j, k);
                    else tma_load_2d_pair(sb, &map_b, bar, k, n);
                    if (++s == P.stages) { s = 0; ph ^= 1u; }
                }
            }
        } else if (warp == 1 && lane == 0 && rank == 0) {
            // ---- MMA issuer (leader) ----
            const uint32_t idesc = E4M3 ? instr_desc_e4m3(256, P.bn) : instr_desc_bf16(256, P.bn, P.a_mn ? 1u : 0u, P.b_mn ? 1u : 0u);
            const uint32_t a_lbo = P.a_mn ? kSubBytes : 16u, a_step = P.a_mn ? 2048u : 32u;
            const uint32_t b_lbo = P.b_mn ? kSubBytes : 16u, b_step = P.b_mn ? 2048u : 32u;
            uint32_t s = 0, ph = 0, use = 0;          // stage, its phase, accumulator slots used so far
            bool ok = W.limit_ns != 0 || mbar_is_done(smem_u32(&sh.full[0]), 0u);
            if (!ok) raise_abort(W);
            for (uint32_t t = cluster; ok && t < tiles; t += clusters) {
                for (uint32_t k0 = 0; ok && k0 < P.K_blocks; k0 += P.chunk, ++use) {
                    const uint32_t k1 = min(P.K_blocks, k0 + P.chunk), acc = use & 1u, d = tmem + acc * 256u;
                    if (!mbar_wait_cl(smem_u32(&sh.acc_empty[acc]), ((use >> 1) & 1u) ^ 1u, W)) { ok = false; break; }
                    tc_fence_after();
                    for (uint32_t kb = k0; kb < k1; ++kb) {
                        if (!mbar_wait_cl(smem_u32(&sh.full[s]), ph, W)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t sa = base + s * kLinStage, sb = sa + kLinOperand;
#pragma unroll
                        for (uint32_t q = 0; q < 4; ++q)
                            umma_pair<E4M3>(d, smem_desc_sw128(sa + q * a_step, a_lbo, 1024u), smem_desc_sw128(sb + q * b_step, b_lbo, 1024u), idesc, (kb != k0) | (q != 0u));
                        umma_commit_both(smem_u32(&sh.empty[s]));
                        if (++s == P.stages) { s = 0; ph ^= 1u; }
                    }
                    if (ok) umma_commit_both(smem_u32(&sh.acc_full[acc]));
                }
            }
            // every MMA issued above has completed before either CTA releases tensor memory
            umma_commit_local_pair(smem_u32(&sh.drain));
            const uint64_t t0 = global_timer_ns();
            while (!mbar_try_wait_cl(smem_u32(&sh.drain), 0u))
                if (global_timer_ns() - t0 > 2000000000ull) { atomicOr(&g_linear_status, STATUS_TIMEOUT); break; }
        }
    } else {
        // ---- write-out (both CTAs) ----
        if constexpr (LONG) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const uint32_t quad = warp & 3u, part = (warp - kLpEpiWarp0) >> 2;      // four warps, one a quadrant of lanes, per part
        const uint32_t lane_base = (quad * 32u) << 16;
        OutRing out = {dyn_smem + (base - smem_u32(dyn_smem)) + P.stages * kLinStage + (warp - kLpEpiWarp0) * (P.out_bytes * P.out_count), P.out_bytes, P.out_count, 0u};
        if constexpr (!LONG) {
            // parts 0, 1 drain slot 0, parts 2, 3 slot 1 (every second tile of the cluster); the two parts of a slot
            // take its chunks of 32 columns in turn, and all four those of the last tile
            const uint32_t count = (tiles - cluster + clusters - 1) / clusters;
            for (uint32_t k = 0; k < count; ++k) {
                const bool last = k + 1 == count;
                const uint32_t slot = k & 1u, sharers = last ? 4u : 2u;
                if (!last && part >> 1 != slot) continue;
                const uint2 at = pair_tile(P, cluster + k * clusters);
                const uint32_t empty = mapa_shared(smem_u32(&sh.acc_empty[slot]), 0u), taddr = tmem + slot * 256u + lane_base;
                const uint32_t row0 = at.x * 256u + rank * 128u + quad * 32u, col = at.y * P.bn, mine = part & (sharers - 1);
                if (mine & 1u) prefetch_strip(P.e.mul, P.e.mul_type, P.e.ldmul, P.e, row0 + lane, col, P.bn);
                else prefetch_strip(P.e.res, P.e.res_type, P.e.ldres, P.e, row0 + lane, col, P.bn);
                const bool ok = write_strip<ACT>(P.e, &map_c, &map_z, out, taddr, row0, col, mine * 32u, sharers * 32u, P.bn, lane,
                    [&] {
                        const bool r = __all_sync(0xFFFFFFFFu, mbar_wait_cl(smem_u32(&sh.acc_full[slot]), (k >> 1) & 1u, W));
                        tc_fence_after();
                        return r;
                    },
                    [&] {                             // the warp has read the slot: hand it back
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster_read_done(empty);
                    });
                if (!ok) break;
            }
        } else {
            // all eight warps on one tile: part p keeps columns 128 p ... of its rows; the finished sums go back into the last
            // slot, from where they are written out piece by piece (registers hold nothing else meanwhile)
            uint32_t use = 0;
            bool ok = true;
            for (uint32_t t = cluster; ok && t < tiles; t += clusters) {
                const uint2 at = pair_tile(P, t);
                const uint32_t row0 = at.x * 256u + rank * 128u + quad * 32u, col = at.y * P.bn + part * 128u;
                const uint32_t cols = P.bn > part * 128u ? min(128u, P.bn - part * 128u) : 0u;
                float sum[128];
#pragma unroll
                for (int i = 0; i < 128; ++i) sum[i] = 0.f;
                for (uint32_t k0 = 0; k0 < P.K_blocks; k0 += P.chunk, ++use) {
                    const uint32_t acc = use & 1u, taddr = tmem + acc * 256u + part * 128u + lane_base;
                    ok = __all_sync(0xFFFFFFFFu, pair_wait_inline(smem_u32(&sh.acc_full[acc]), (use >> 1) & 1u, W));
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (uint32_t c = 0; c < 128; c += 32) {
                        uint32_t u[32];
                        tmem_ld_32x32(taddr + c, u);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) sum[c + i] += __uint_as_float(u[i]);
                    }
                    if (k0 + P.chunk >= P.K_blocks) {
#pragma unroll
                        for (uint32_t c = 0; c < 128; c += 32) tmem_st_32x32(taddr + c, sum + c);
                        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                        if (cols) write_strip<ACT>(P.e, &map_c, &map_z, out, taddr, row0, col, 0u, 32u, cols, lane, [] { return true; }, [] {});
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster_read_done(mapa_shared(smem_u32(&sh.acc_empty[acc]), 0u));
                }
            }
        }
        if (P.e.form) out.finish(lane);               // the last stores are complete, their buffers read
        tc_fence_before();
    }
    __syncwarp();
    cluster_arrive_wait();                            // both CTAs are done with both tensor memories and all barriers
    if (sh.abort_flag) {                              // a role gave up: copies may still be in flight towards this CTA
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 200000ull) { }
        cluster_arrive_wait();
    }
    tc_fence_after();
    if (warp == 1) tmem_dealloc_pair(tmem, 512);
}

// ---- host --------------------------------------------------------------------------------------------
namespace {

// Boxes of 128 bytes along the contiguous dimension x `box_rows` rows of a row-major [rows x cols] matrix.
int encode_operand(CUtensorMap* out, const void* base, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t box_rows, bool e4m3) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return CLEAVE_E_CUDA;
    const uint32_t es = e4m3 ? 1u : 2u;
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {ld * es};
    cuuint32_t box[2] = {128u / es, box_rows};
    cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(out, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims,
                          strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? 0 : CLEAVE_E_CUDA;
}

// Boxes of 32 x 32 of a row-major [rows x cols] output, bf16 or fp32, for bulk stores.
int encode_output(CUtensorMap* out, void* base, uint64_t rows, uint64_t cols, uint64_t ld, bool f32) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return CLEAVE_E_CUDA;
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {ld * (f32 ? 4u : 2u)};
    cuuint32_t box[2] = {32, 32};
    cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(out, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, f32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                          CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? 0 : CLEAVE_E_CUDA;
}

// A row-major [rows x cols] bf16 matrix, cols a multiple of 64, as [cols / 64][rows][64]: a box of 64 x 64 x 2 brings two
// neighbouring groups of 64 columns (8 KB each, one after the other) with one operation.
int encode_groups(CUtensorMap* out, const void* base, uint64_t rows, uint64_t cols, uint64_t ld) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return CLEAVE_E_CUDA;
    cuuint64_t dims[3] = {64, rows, cols / 64};
    cuuint64_t strides[2] = {ld * 2, 128};
    cuuint32_t box[3] = {64, 64, 2};
    cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? 0 : CLEAVE_E_CUDA;
}

bool rows16(const void* p, uint64_t ld, uint32_t type) { return (uintptr_t)p % 16 == 0 && (ld * type_bytes(type)) % 16 == 0; }

constexpr uint32_t kActs = CLEAVE_ACT_SILU + 1;
using PairKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const PairParams);
using SplitKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const LinearParams);
struct PickPair {
    using Kernel = PairKernel;
    template <uint32_t ACT> static Kernel get(bool e4m3, bool lng) {
        if (e4m3) return lng ? linear_pair_kernel<true, true, ACT> : linear_pair_kernel<true, false, ACT>;
        return lng ? linear_pair_kernel<false, true, ACT> : linear_pair_kernel<false, false, ACT>;
    }
};
struct PickSplit {
    using Kernel = SplitKernel;
    template <uint32_t ACT> static Kernel get(bool e4m3, bool lng) {
        if (e4m3) return lng ? linear_split_kernel<true, true, ACT> : linear_split_kernel<true, false, ACT>;
        return lng ? linear_split_kernel<false, true, ACT> : linear_split_kernel<false, false, ACT>;
    }
};
template <typename Pick>
typename Pick::Kernel pick_act(uint32_t act, bool e4m3, bool lng) {
    switch (act) {
        case CLEAVE_ACT_RELU: return Pick::template get<CLEAVE_ACT_RELU>(e4m3, lng);
        case CLEAVE_ACT_GELU: return Pick::template get<CLEAVE_ACT_GELU>(e4m3, lng);
        case CLEAVE_ACT_GELU_TANH: return Pick::template get<CLEAVE_ACT_GELU_TANH>(e4m3, lng);
        case CLEAVE_ACT_SILU: return Pick::template get<CLEAVE_ACT_SILU>(e4m3, lng);
        default: return Pick::template get<CLEAVE_ACT_NONE>(e4m3, lng);
    }
}

}  // namespace

int launch_linear(const cleave_linear_t& d, int sms, cudaStream_t st) {
    const bool e4m3 = d.in_type == CLEAVE_T_E4M3;
    const cleave_gemm_t& g = d.g;
    LinearParams P = {};
    Epilogue& e = P.e;
    e.M = g.M; e.N = g.N;
    e.c_type = d.c_type; e.bias_type = d.bias_type; e.z_type = d.z_type; e.mul_type = d.mul_type; e.res_type = d.res_type;
    e.scale_a = d.scale_a; e.scale_b = d.scale_b; e.bias = d.bias; e.z = d.z; e.mul = d.mul; e.res = d.res; e.C = d.C;
    e.ldz = d.ldz; e.ldmul = d.ldmul; e.ldres = d.ldres; e.ldc = d.ldc;
    // bulk stores want 16-byte rows, and so do the row loads of mul and res
    const bool bulk = rows16(d.C, d.ldc, d.c_type) && d.ldc * type_bytes(d.c_type) < (1ull << 40) && (!d.z || (d.z_type == CLEAVE_T_BF16 && rows16(d.z, d.ldz, d.z_type) && d.ldz < (1ull << 39))) &&
                      (!d.mul || rows16(d.mul, d.ldmul, d.mul_type)) && (!d.res || rows16(d.res, d.ldres, d.res_type));
    e.form = !bulk ? 0u : (d.c_type == CLEAVE_T_BF16 ? 1u : 2u);
    CUtensorMap mc = {}, mz = {};
    int rc = 0;
    if (e.form && (rc = encode_output(&mc, d.C, g.M, g.N, d.ldc, e.form == 2))) return rc;
    if (e.form && d.z && (rc = encode_output(&mz, d.z, g.M, g.N, d.ldz, false))) return rc;
    P.wait_limit_ns = g_linear_wait_limit.load(std::memory_order_relaxed);
    P.a_mn = g.transA ? 1u : 0u;
    P.b_mn = g.transB ? 0u : 1u;
    const uint32_t kblk = e4m3 ? 128u : 64u;
    P.K_blocks = (g.K + kblk - 1) / kblk;
    CUtensorMap ma, mb;
    auto encode_b = [&](uint32_t rows) { return g.transB ? encode_operand(&mb, d.B, g.N, g.K, g.ldb, rows, e4m3) : encode_operand(&mb, d.B, g.K, g.N, g.ldb, 64, e4m3); };
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cfg.stream = st;
    cudaError_t err;
    const uint64_t tiles_m = (g.M + kLinTile - 1) / kLinTile, tiles_n = (g.N + kLinTile - 1) / kLinTile, tiles = tiles_m * tiles_n;
    const uint32_t pairs = (uint32_t)sms / 2;
    // Results of an fp32 output of a long K move on every kLongBlocks K-blocks (both kernels)
    const bool lng = (d.c_type == CLEAVE_T_F32 || d.z_type == CLEAVE_T_F32) && P.K_blocks > kLongBlocks;
    // Pairs of CTAs bring half the operand bytes for a product, one CTA a tile starts and ends sooner and spreads few tiles
    // wider.  With one row of tiles half of a pair's rows would be empty (16 x 50304 x 2048: 56 us by pairs, 42 by tiles);
    // from two tiles a place on, pairs win at every K (4096 x 2048: K = 256 10.1 against 12.6 us, K = 4096 51 against 66);
    // between one tile an SM and two, when the pairs take them in one go, from a K of 32 blocks on (1536 x 2048: K = 1024 10.8
    // against 11.1 us, 2048 16.1 against 17.7, 4096 26.4 against 30.2; fp32 weight gradients 2048 20.8 against 22.0,
    // 4096 33 against 37); with fewer tiles, K is split (1152 x 2048 x 4096: 26.3 against 21.4).
    const uint64_t pair_tiles = (uint64_t)((g.M + 255) / 256) * ((g.N + 255) / 256);
    const bool by_pairs = g.M > kLinTile && (tiles >= 2u * (uint32_t)sms || (tiles > (uint32_t)sms && pair_tiles <= pairs && P.K_blocks >= 32));
    if (by_pairs) {
        PairParams Q = {};
        Q.e = P.e; Q.K_blocks = P.K_blocks; Q.a_mn = P.a_mn; Q.b_mn = P.b_mn; Q.wait_limit_ns = P.wait_limit_ns;
        Q.tiles_m = (g.M + 255) / 256;
        // 256 columns (the whole of a narrower C): narrower tiles fill the last wave better, but bring fewer products per
        // byte from L2, about 62 bytes a cycle and SM, and lost at every size tried (8192 x 768 x 3072: 39 us with 256
        // columns, 43 with 224 and 192, 56 with 128; 4096^3: 106, 127, 130, 160).
        Q.bn = g.N >= 256 ? 256u : (g.N + 31) / 32 * 32;
        Q.tiles_n = (g.N + Q.bn - 1) / Q.bn;
        Q.b_boxes = (Q.bn / 2 + 63) / 64;
        Q.b_bytes = Q.b_mn ? Q.b_boxes * kSubBytes : Q.bn / 2 * 128u;
        Q.chunk = lng ? kLongBlocks : Q.K_blocks;
        // (an M- or N-contiguous operand by one copy a stage instead of two, where its columns are whole groups of 64: 4096^3
        // 98.8 us against 105.9, 11008 x 4096 x 4096 285 against 308)
        if (Q.a_mn && g.M % 64 == 0) { Q.a_mn = 2; rc = encode_groups(&ma, d.A, g.K, g.M, g.lda); }
        else rc = g.transA ? encode_operand(&ma, d.A, g.K, g.M, g.lda, 64, e4m3) : encode_operand(&ma, d.A, g.M, g.K, g.lda, 128, e4m3);
        if (rc) return rc;
        if (Q.b_mn && Q.bn == 256 && g.N % 64 == 0) { Q.b_mn = 2; rc = encode_groups(&mb, d.B, g.K, g.N, g.ldb); }
        else rc = encode_b(Q.bn / 2);
        if (rc) return rc;
        // output buffers a warp takes in turn (one of 4 KB for the general form); the rest of the shared memory holds stages
        const uint32_t out_warps = pair_warps(lng);
        Q.out_bytes = e.form == 1 ? 2048u : 4096u;
        Q.out_count = e.form == 1 ? 2u : (e.form == 2 && lng ? 2u : 1u);
        const uint32_t out_smem = out_warps * Q.out_bytes * Q.out_count;
        Q.stages = min(kLpMaxStages, (kLpSmemMost - 1024u - out_smem) / kLinStage);
        const uint32_t smem = Q.stages * kLinStage + 1024u + out_smem;
        const PairKernel kernel = pick_act<PickPair>(d.act, e4m3, lng);
        static SmemLimit limit[4 * kActs];
        if (limit[((e4m3 ? 2 : 0) + (lng ? 1 : 0)) * kActs + d.act].raise(reinterpret_cast<const void*>(kernel), kLpSmemMost) != cudaSuccess) { cudaGetLastError(); return CLEAVE_E_CUDA; }
        const uint64_t all = (uint64_t)Q.tiles_m * Q.tiles_n;
        if (all > 0x7FFFFFFFull) return CLEAVE_E_UNSUPPORTED;
        cfg.gridDim = dim3(2u * (unsigned)(all < pairs ? all : pairs));
        cfg.blockDim = dim3(pair_threads(lng));
        cfg.dynamicSmemBytes = smem;
        cfg.numAttrs = 1;                                   // (the cluster size is the kernel's own)
        err = cudaLaunchKernelEx(&cfg, kernel, ma, mb, mc, mz, Q);
    } else {
        P.tiles_n = (uint32_t)tiles_n;
        // K is split while every CTA still finds a place at once (two an SM) and keeps at least four stages of work (16 x 4096 x
        // 4096: 22.8 us whole, 15.7 in two, 11.5 in four, 11.2 in eight; 512 x 1024 x 1024: 9.6, 9.4, 10.6, 11.0)
        P.splits = 1;
        while (P.splits < 8 && tiles * P.splits * 2 <= 2u * (uint32_t)sms && P.K_blocks / (P.splits * 2) >= 4) P.splits *= 2;
        // (K-contiguous rows of A beyond M need not even be zeros: they only reach accumulator rows that nobody reads)
        P.a_rows = g.transA ? kLinTile : std::min(kLinTile, (g.M + 7) / 8 * 8);
        P.stage_bytes = kLinOperand + P.a_rows * 128u;
        P.stages = std::min(kLinMaxStages, (kLinSmem - 1024u - (kLinOperand - P.a_rows * 128u)) / P.stage_bytes);
        rc = g.transA ? encode_operand(&ma, d.A, g.K, g.M, g.lda, 64, e4m3) : encode_operand(&ma, d.A, g.M, g.K, g.lda, P.a_rows, e4m3);
        if (rc || (rc = encode_b(kLinTile))) return rc;
        const bool hand_over = lng && (P.K_blocks + P.splits - 1) / P.splits > kLongBlocks;      // (the cluster's sum is a rounded one)
        const SplitKernel kernel = pick_act<PickSplit>(d.act, e4m3, hand_over);
        static SmemLimit limit[4 * kActs];
        if (limit[((e4m3 ? 2 : 0) + (hand_over ? 1 : 0)) * kActs + d.act].raise(reinterpret_cast<const void*>(kernel), kLinSmem) != cudaSuccess) { cudaGetLastError(); return CLEAVE_E_CUDA; }
        cfg.gridDim = dim3((unsigned)(tiles * P.splits));
        cfg.blockDim = dim3(kLinThreads);
        cfg.dynamicSmemBytes = kLinSmem;
        attr[1].val.clusterDim.x = P.splits;
        err = cudaLaunchKernelEx(&cfg, kernel, ma, mb, mc, mz, P);
    }
    if (err != cudaSuccess) { cudaGetLastError(); return CLEAVE_E_CUDA; }
    return 0;
}

int linear_status(cudaStream_t st) {
    unsigned int s = 0;
    const unsigned int zero = 0;
    if (cudaMemcpyFromSymbolAsync(&s, g_linear_status, sizeof s, 0, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess ||
        (s && (cudaMemcpyToSymbolAsync(g_linear_status, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, st) != cudaSuccess ||
               cudaStreamSynchronize(st) != cudaSuccess))) { cudaGetLastError(); return CLEAVE_E_CUDA; }
    return s & STATUS_TIMEOUT ? CLEAVE_E_TIMEOUT : 0;
}
void linear_set_wait_limit_ns(uint64_t ns) { g_linear_wait_limit.store(ns, std::memory_order_relaxed); }

}  // namespace cleave
