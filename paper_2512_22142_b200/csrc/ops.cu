// C ABI of the operators around the GEMMs (see include/cleave.h): argument checks, the optimizer's device table,
// launches.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "ops.cuh"

using namespace cleave;

struct cleave_adamw_s {
    int device = -1;
    uint32_t state_type = 0, g_type = 0, n_chunks = 0, chunk_blocks = 0;
    std::vector<AdamTensor> host;
    AdamTensor* tensors = nullptr;
    AdamChunk* chunks = nullptr;
};

namespace {

constexpr uint64_t kMaxRows = 0x7FFFFFFFull, kMaxCols = 0x7FFFFFFFull, kMaxLd = 1ull << 40;     // (the kernels count columns in 32 bits)

bool float_type(uint32_t t) { return t == CLEAVE_T_BF16 || t == CLEAVE_T_F32; }
bool aligned(const void* p, uint64_t bytes) { return ((uintptr_t)p % bytes) == 0; }

// A required matrix operand: a pointer aligned to its elements, rows that hold `cols` elements.
bool matrix_ok(const void* p, uint32_t type, uint64_t ld, uint64_t cols) {
    const uint32_t b = type_bytes(type);
    return p && b && aligned(p, b) && ld >= cols && ld <= kMaxLd;
}
// An optional one: absent means type 0 and no pointer.
bool optional_ok(const void* p, uint32_t type, uint64_t ld, uint64_t cols) {
    if (type == CLEAVE_T_NONE) return p == nullptr;
    return float_type(type) && matrix_ok(p, type, ld, cols);
}
int cuda_code(cudaError_t e) {
    if (e == cudaSuccess) return CLEAVE_OK;
    cudaGetLastError();
    return CLEAVE_E_CUDA;
}
// SM count of the current device, or a negative CLEAVE_E_* code (asked for once per device)
int need_device() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0, major = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return CLEAVE_E_CUDA; }
    if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) != 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) { cudaGetLastError(); return CLEAVE_E_CUDA; }
    if (major != 10) n = CLEAVE_E_UNSUPPORTED;
    if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

bool adam_wide(const AdamTensor& t, uint32_t state_type, uint32_t g_type) {
    const uint64_t state = state_type == CLEAVE_T_F32 ? 16 : 4, grad = g_type == CLEAVE_T_F32 ? 16 : 8;
    return aligned(t.p, 16) && aligned(t.w, 8) && aligned(t.g, grad) && aligned(t.m, state) && aligned(t.v, state);
}

}  // namespace

extern "C" {

// ---- AdamW -------------------------------------------------------------------------------------------
int cleave_adamw_create(const cleave_adamw_tensor_t* t, uint32_t n, uint32_t state_type, uint32_t g_type, cleave_adamw_t** out) {
    if (!out) return CLEAVE_E_INVAL;
    *out = nullptr;
    if (!t || !n || !float_type(g_type) || (state_type != CLEAVE_T_F32 && state_type != CLEAVE_T_E4M3)) return CLEAVE_E_INVAL;
    const bool state8 = state_type == CLEAVE_T_E4M3;
    uint64_t n_blocks = 0;
    for (uint32_t i = 0; i < n; ++i) {
        if (t[i].numel == 0) continue;
        if (t[i].numel > (1ull << 40) || !std::isfinite(t[i].weight_decay)) return CLEAVE_E_INVAL;
        const uint64_t sb = state8 ? 1 : 4;
        if (!t[i].p || !aligned(t[i].p, 4) || !aligned(t[i].w, 2) || !t[i].g || !aligned(t[i].g, type_bytes(g_type)) || !t[i].m || !t[i].v ||
            !aligned(t[i].m, sb) || !aligned(t[i].v, sb)) return CLEAVE_E_INVAL;
        if (state8 != (t[i].m_scale != nullptr) || state8 != (t[i].v_scale != nullptr) || !aligned(t[i].m_scale, 4) || !aligned(t[i].v_scale, 4)) return CLEAVE_E_INVAL;
        n_blocks += (t[i].numel + kStateBlock - 1) / kStateBlock;
    }
    if (n_blocks / kChunkWarps > 0x7FFFFFF0ull - n) return CLEAVE_E_UNSUPPORTED;
    const int sms = need_device();
    if (sms < 0) return sms;
    int rc = 0;
    // Blocks a warp takes: long runs keep its copies in flight, but an SM that runs out of chunks early waits, so there are
    // at least two waves of them (a GPT-2-small-shaped layer with 32-bit states: 39.5 us with one wave, 34.7 with two,
    // 34.4 with four, 42 with six; 400 ragged tensors with 8-bit states: 28.3, 26.5, 28.4, 28.4).
    const uint64_t slots = (uint64_t)sms * (state8 ? 3 : 2) * kChunkWarps;
    const uint64_t run = std::max<uint64_t>(1, std::min<uint64_t>(kChunkMost, n_blocks / (2 * slots)));
    const uint32_t chunk_blocks = kChunkWarps * (uint32_t)run;
    cleave_adamw_s* h = new (std::nothrow) cleave_adamw_s();
    if (!h) return CLEAVE_E_NOMEM;
    try {
        std::vector<AdamChunk> chunks;
        chunks.reserve(n_blocks / chunk_blocks + n);
        h->host.resize(n);
        for (uint32_t i = 0; i < n; ++i) {
            AdamTensor& a = h->host[i];
            a = AdamTensor{t[i].numel, t[i].p, static_cast<__nv_bfloat16*>(t[i].w), t[i].g, t[i].m, t[i].v, t[i].m_scale, t[i].v_scale, t[i].weight_decay, 0u, 0u};
            a.wide = adam_wide(a, state_type, g_type) ? 1u : 0u;
            const uint64_t blocks = (t[i].numel + kStateBlock - 1) / kStateBlock;
            for (uint64_t b = 0; b < blocks; b += chunk_blocks) chunks.push_back(AdamChunk{i, (uint32_t)b});
        }
        h->state_type = state_type; h->g_type = g_type; h->n_chunks = (uint32_t)chunks.size(); h->chunk_blocks = chunk_blocks;
        if (cudaGetDevice(&h->device) != cudaSuccess) rc = CLEAVE_E_CUDA;
        if (!rc && (cudaMalloc(&h->tensors, n * sizeof(AdamTensor)) != cudaSuccess ||
                    cudaMalloc(&h->chunks, (chunks.empty() ? 1 : chunks.size()) * sizeof(AdamChunk)) != cudaSuccess)) rc = CLEAVE_E_NOMEM;
        // the table is complete on the device before the call returns, whatever stream the steps run on
        if (!rc && (cudaMemcpy(h->tensors, h->host.data(), n * sizeof(AdamTensor), cudaMemcpyHostToDevice) != cudaSuccess ||
                    (!chunks.empty() && cudaMemcpy(h->chunks, chunks.data(), chunks.size() * sizeof(AdamChunk), cudaMemcpyHostToDevice) != cudaSuccess) ||
                    cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess)) rc = CLEAVE_E_CUDA;
    } catch (const std::bad_alloc&) { rc = CLEAVE_E_NOMEM; }
    if (rc) { cudaGetLastError(); cleave_adamw_destroy(h); return rc; }
    *out = h;
    return 0;
}

int cleave_adamw_set_grads(cleave_adamw_t* h, const void* const* g, void* stream) {
    if (!h || !g) return CLEAVE_E_INVAL;
    for (size_t i = 0; i < h->host.size(); ++i)
        if (h->host[i].numel && (!g[i] || !aligned(g[i], type_bytes(h->g_type)))) return CLEAVE_E_INVAL;
    for (size_t i = 0; i < h->host.size(); ++i) {
        h->host[i].g = g[i];
        h->host[i].wide = adam_wide(h->host[i], h->state_type, h->g_type) ? 1u : 0u;
    }
    // pageable source: the copy is staged before the call returns
    return cuda_code(cudaMemcpyAsync(h->tensors, h->host.data(), h->host.size() * sizeof(AdamTensor), cudaMemcpyHostToDevice, static_cast<cudaStream_t>(stream)));
}

int cleave_adamw_step(cleave_adamw_t* h, const cleave_adamw_step_t* s, void* stream) {
    if (!h || !s || s->step == 0) return CLEAVE_E_INVAL;
    if (!(s->beta1 >= 0.0 && s->beta1 < 1.0) || !(s->beta2 >= 0.0 && s->beta2 < 1.0) || !(s->eps >= 0.0) || !std::isfinite(s->eps) ||
        !std::isfinite(s->lr) || !std::isfinite(s->grad_scale)) return CLEAVE_E_INVAL;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return cuda_code(cudaErrorUnknown);
    if (dev != h->device) return CLEAVE_E_INVAL;             // the table lives on another device
    AdamStep k;
    k.beta1 = (float)s->beta1; k.omb1 = (float)(1.0 - s->beta1);
    k.beta2 = (float)s->beta2; k.omb2 = (float)(1.0 - s->beta2);
    k.step_size = (float)(s->lr / (1.0 - std::pow(s->beta1, (double)s->step)));
    k.root = (float)(1.0 / std::sqrt(1.0 - std::pow(s->beta2, (double)s->step)));
    k.eps = (float)s->eps; k.grad_scale = (float)s->grad_scale;
    k.lr = s->lr;
    k.base = s->seed + (s->step << 32);
    return cuda_code(launch_adamw(h->tensors, h->chunks, h->n_chunks, h->chunk_blocks, k, h->state_type == CLEAVE_T_E4M3, h->g_type == CLEAVE_T_BF16,
                                  static_cast<cudaStream_t>(stream)));
}

void cleave_adamw_destroy(cleave_adamw_t* h) {
    if (!h) return;
    cudaFree(h->tensors);
    cudaFree(h->chunks);
    cudaGetLastError();
    delete h;
}

// ---- norm ----------------------------------------------------------------------------------------------
int cleave_rmsnorm(const cleave_rmsnorm_t* d, void* stream) {
    if (!d || !d->cols || !(d->eps >= 0.f)) return CLEAVE_E_INVAL;
    if (d->rows == 0) return CLEAVE_OK;
    if (d->rows > kMaxRows || d->cols > kMaxCols) return CLEAVE_E_UNSUPPORTED;
    if (!float_type(d->x_type) || !matrix_ok(d->x, d->x_type, d->ldx, d->cols)) return CLEAVE_E_INVAL;
    if (!optional_ok(d->r, d->r_type, d->ldr, d->cols) || !optional_ok(d->w, d->w_type, d->cols, d->cols)) return CLEAVE_E_INVAL;
    if (d->h && (!d->r || !matrix_ok(d->h, d->r_type, d->ldh, d->cols))) return CLEAVE_E_INVAL;
    if (!matrix_ok(d->y, d->y_type, d->ldy, d->cols) || !aligned(d->rstd, 4)) return CLEAVE_E_INVAL;
    if ((d->y_type == CLEAVE_T_E4M3) != (d->scale != nullptr) || !aligned(d->scale, 4)) return CLEAVE_E_INVAL;
    const int sms = need_device();
    return sms < 0 ? sms : cuda_code(launch_rmsnorm(*d, true, sms, static_cast<cudaStream_t>(stream)));
}

int cleave_quantize_rows(const void* x, uint32_t x_type, uint64_t rows, uint32_t cols, uint64_t ldx, void* y, uint64_t ldy,
                         float* scale, void* stream) {
    if (!cols) return CLEAVE_E_INVAL;
    if (rows == 0) return CLEAVE_OK;
    if (rows > kMaxRows || cols > kMaxCols) return CLEAVE_E_UNSUPPORTED;
    if (!float_type(x_type) || !matrix_ok(x, x_type, ldx, cols) || !matrix_ok(y, CLEAVE_T_E4M3, ldy, cols) || !scale || !aligned(scale, 4)) return CLEAVE_E_INVAL;
    cleave_rmsnorm_t d = {};
    d.rows = rows; d.cols = cols; d.x_type = x_type; d.y_type = CLEAVE_T_E4M3;
    d.x = x; d.ldx = ldx; d.y = y; d.ldy = ldy; d.scale = scale;
    const int sms = need_device();
    return sms < 0 ? sms : cuda_code(launch_rmsnorm(d, false, sms, static_cast<cudaStream_t>(stream)));
}

uint64_t cleave_rmsnorm_backward_workspace(uint64_t rows, uint32_t cols) {
    return (uint64_t)rmsnorm_backward_parts(rows, cols) * cols * sizeof(float);
}
int cleave_rmsnorm_backward(const cleave_rmsnorm_backward_t* d, void* workspace, void* stream) {
    if (!d || !d->cols || !aligned(d->dw, 4)) return CLEAVE_E_INVAL;
    if (d->rows > kMaxRows || d->cols > kMaxCols) return CLEAVE_E_UNSUPPORTED;
    if (d->rows) {
        if (!float_type(d->dy_type) || !float_type(d->h_type) || !matrix_ok(d->dy, d->dy_type, d->lddy, d->cols) ||
            !matrix_ok(d->h, d->h_type, d->ldh, d->cols) || !matrix_ok(d->dx, d->h_type, d->lddx, d->cols)) return CLEAVE_E_INVAL;
        if (!optional_ok(d->w, d->w_type, d->cols, d->cols) || (d->dres && !matrix_ok(d->dres, d->h_type, d->lddres, d->cols))) return CLEAVE_E_INVAL;
        if (!d->rstd || !aligned(d->rstd, 4) || (d->dw && (!workspace || !aligned(workspace, 16)))) return CLEAVE_E_INVAL;
    }
    const int sms = need_device();
    return sms < 0 ? sms : cuda_code(launch_rmsnorm_backward(*d, static_cast<float*>(workspace), static_cast<cudaStream_t>(stream)));
}

// ---- product and its epilogue's backward -------------------------------------------------------------------
int cleave_linear(const cleave_linear_t* d, void* stream) {
    if (!d) return CLEAVE_E_INVAL;
    const cleave_gemm_t& g = d->g;
    if (!g.N || !g.K || g.M > 0x7FFFFFFFu || g.N > 0x7FFFFFFFu || g.K > 0x7FFFFFFFu || g.transA > 1 || g.transB > 1) return CLEAVE_E_INVAL;
    if (d->in_type != CLEAVE_T_BF16 && d->in_type != CLEAVE_T_E4M3) return CLEAVE_E_INVAL;
    if (d->act > CLEAVE_ACT_SILU || !float_type(d->c_type)) return CLEAVE_E_INVAL;
    const bool e4m3 = d->in_type == CLEAVE_T_E4M3;
    if (e4m3 && (g.transA || !g.transB)) return CLEAVE_E_UNSUPPORTED;
    if (g.M == 0) return CLEAVE_OK;
    const uint32_t unit = e4m3 ? 16 : 8;
    if (!d->A || !d->B || !aligned(d->A, 16) || !aligned(d->B, 16) || g.lda % unit || g.ldb % unit ||
        g.lda < (g.transA ? g.M : g.K) || g.ldb < (g.transB ? g.K : g.N)) return CLEAVE_E_INVAL;
    if (!aligned(d->scale_a, 4) || !aligned(d->scale_b, 4) || !optional_ok(d->bias, d->bias_type, g.N, g.N)) return CLEAVE_E_INVAL;
    if (!optional_ok(d->z, d->z_type, d->ldz, g.N) || !optional_ok(d->mul, d->mul_type, d->ldmul, g.N) ||
        !optional_ok(d->res, d->res_type, d->ldres, g.N) || !matrix_ok(d->C, d->c_type, d->ldc, g.N)) return CLEAVE_E_INVAL;
    const int sms = need_device();
    return sms < 0 ? sms : launch_linear(*d, sms, static_cast<cudaStream_t>(stream));
}
int cleave_linear_status(void* stream) { return linear_status(static_cast<cudaStream_t>(stream)); }
void cleave_linear_set_wait_limit_ns(uint64_t ns) { linear_set_wait_limit_ns(ns); }

uint64_t cleave_act_backward_workspace(uint64_t rows, uint32_t cols) {
    return (uint64_t)act_backward_parts(rows, cols) * cols * sizeof(float);
}
int cleave_act_backward(const cleave_act_backward_t* d, void* workspace, void* stream) {
    if (!d || !d->cols || d->act > CLEAVE_ACT_SILU || !aligned(d->dbias, 4)) return CLEAVE_E_INVAL;
    if (d->rows > kMaxRows || d->cols > kMaxCols) return CLEAVE_E_UNSUPPORTED;
    if (d->rows) {
        if (!float_type(d->dy_type) || !matrix_ok(d->dy, d->dy_type, d->lddy, d->cols)) return CLEAVE_E_INVAL;
        if (!optional_ok(d->z, d->z_type, d->ldz, d->cols) || !optional_ok(d->mul, d->mul_type, d->ldmul, d->cols) ||
            !optional_ok(d->dz, d->dz_type, d->lddz, d->cols) || !optional_ok(d->dmul, d->dmul_type, d->lddmul, d->cols)) return CLEAVE_E_INVAL;
        if (!d->z && (d->act != CLEAVE_ACT_NONE || d->dmul)) return CLEAVE_E_INVAL;
        if (d->dbias && (!workspace || !aligned(workspace, 16))) return CLEAVE_E_INVAL;
    }
    const int sms = need_device();
    return sms < 0 ? sms : cuda_code(launch_act_backward(*d, static_cast<float*>(workspace), static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
