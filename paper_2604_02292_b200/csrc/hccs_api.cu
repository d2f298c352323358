// C ABI of libhccs: context, parameter-table validation and upload, argument checks, dispatch.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <new>

#include "hccs.h"
#include "hccs_internal.h"

struct hccs_ctx {
    int device = 0;
    hccs::HeadEntry *d_table = nullptr;     // device parameter table
    hccs::HeadEntry *h_table = nullptr;     // pinned staging copy of it
    int32_t *d_mult = nullptr;              // device copy of the fused path's per-head multipliers
    int32_t *h_mult = nullptr;              // pinned staging for them
    int32_t *mult_last = nullptr;           // host copy of what d_mult holds (to skip an unchanged upload)
    int32_t mult_last_heads = 0;            // 0: d_mult holds nothing yet
    int32_t capacity = 0;                   // heads the allocations can hold
    int32_t num_heads = 0;                  // 0 = nothing uploaded
    int32_t n_design = 0;
    int32_t out_shift = 0;
    bool wide = false;                      // the table came from hccs_params_upload_wide
    uint32_t *d_status = nullptr;           // device status word (bounded waits report here)
    uint32_t *h_status = nullptr;           // pinned landing place for it
    cudaEvent_t table_copied = nullptr;     // the staging buffers may be rewritten after this
    cudaEvent_t mult_copied = nullptr;
    cudaStream_t d2h_stream = nullptr;      // hccs_forward_host: output copies
    static constexpr int kMaxPieces = 16;
    cudaEvent_t ev_done[kMaxPieces] = {};
    cudaEvent_t ev_join = nullptr;
    int32_t last_cuda_error = 0;
    uint64_t launches = 0;
};

namespace hccs {

FastDiv make_fastdiv(uint32_t d) {
    // q = (umulhi(n, mul) + n) >> shift is floor(n / d) for every n < 2^31:
    // shift = ceil(log2 d), mul = ceil(2^(32+shift) / d) - 2^32.
    FastDiv f;
    f.d = d;
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    const unsigned __int128 one = 1;
    const unsigned __int128 num = one << (32 + l);
    const unsigned __int128 m = (num + d - 1) / d - (one << 32);
    f.mul = (uint32_t)m;
    f.shift = l;
    return f;
}

}  // namespace hccs

namespace {

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
        if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
    }
};

hccs_status_t cuda_fail(hccs_ctx *ctx, cudaError_t e) {
    if (ctx) ctx->last_cuda_error = (int32_t)e;
    (void)cudaGetLastError();   // clear the sticky-free error so later calls start clean
    return HCCS_ERR_CUDA;
}

#define HCCS_CUDA(ctx, call)                                   \
    do {                                                       \
        cudaError_t e__ = (call);                              \
        if (e__ != cudaSuccess) return cuda_fail((ctx), e__);  \
    } while (0)

// The admissible parameter region (Section "Integer Range Constraints") for row length n.
bool theta_admissible(const hccs_head_params_t &t, int32_t n) {
    const int64_t B = t.B, S = t.S, D = t.Dmax;
    if (D < 1 || D > 127) return false;               // distances stay in signed int8
    if (S < 0 || S > 127) return false;               // S >= 0; int8 MAC operand
    if (B <= 0) return false;
    const int64_t floor_score = (256 + (int64_t)n - 1) / n;
    if (B - S * D < floor_score) return false;        // Z >= 256 (and scores non-negative)
    if ((int64_t)n * B > 32767) return false;         // Z <= 32767, rho >= 1; B <= 32767
    return true;
}

hccs_status_t ensure_capacity(hccs_ctx *ctx, int32_t heads) {
    if (heads <= ctx->capacity) return HCCS_OK;
    // growing the table: wait for everything that may still read the old one
    HCCS_CUDA(ctx, cudaDeviceSynchronize());
    if (ctx->d_table) cudaFree(ctx->d_table);
    if (ctx->h_table) cudaFreeHost(ctx->h_table);
    if (ctx->d_mult) cudaFree(ctx->d_mult);
    if (ctx->h_mult) cudaFreeHost(ctx->h_mult);
    delete[] ctx->mult_last;
    ctx->d_table = nullptr; ctx->h_table = nullptr; ctx->d_mult = nullptr; ctx->h_mult = nullptr;
    ctx->mult_last = nullptr; ctx->mult_last_heads = 0;
    ctx->capacity = 0;
    ctx->num_heads = 0;                     // should an allocation fail, no call launches without a table
    // room for every count of heads that the cache calls take, so that captured launches of theirs never lose their table
    int32_t cap = heads < HCCS_MAX_CACHE_HEADS ? HCCS_MAX_CACHE_HEADS : heads;
    HCCS_CUDA(ctx, cudaMalloc(&ctx->d_table, sizeof(hccs::HeadEntry) * cap));
    HCCS_CUDA(ctx, cudaHostAlloc(&ctx->h_table, sizeof(hccs::HeadEntry) * cap, cudaHostAllocDefault));
    HCCS_CUDA(ctx, cudaMalloc(&ctx->d_mult, sizeof(int32_t) * 8 * cap));
    HCCS_CUDA(ctx, cudaHostAlloc(&ctx->h_mult, sizeof(int32_t) * 8 * cap, cudaHostAllocDefault));
    ctx->mult_last = new (std::nothrow) int32_t[8 * (size_t)cap];
    if (!ctx->mult_last) return HCCS_ERR_CUDA;
    ctx->capacity = cap;
    return HCCS_OK;
}

hccs_status_t check_forward_args(hccs_ctx *ctx, const void *in, const void *out, int32_t B, int32_t H,
                                 int32_t Lq, int32_t Lk, uint32_t flags) {
    if (!ctx) return HCCS_ERR_INVALID_ARG;
    if (B < 0 || H < 0 || Lq < 0 || Lk < 0) return HCCS_ERR_INVALID_ARG;
    if (flags & ~7u) return HCCS_ERR_INVALID_ARG;
    if (ctx->num_heads == 0) return HCCS_ERR_NOT_UPLOADED;
    if (H != ctx->num_heads) return HCCS_ERR_INVALID_ARG;
    if (ctx->wide || Lk > ctx->n_design) return HCCS_ERR_CONSTRAINT;
    const int64_t rows = (int64_t)B * H * Lq;
    if (rows >= (1ll << 31)) return HCCS_ERR_UNSUPPORTED;
    if (rows * Lk != 0 && (!in || !out)) return HCCS_ERR_INVALID_ARG;
    return HCCS_OK;
}

hccs::RowArgs make_row_args(const hccs_ctx *ctx, int32_t rows, int32_t H, int32_t Lq, int32_t Lk, uint32_t flags,
                            const int32_t *key_len) {
    hccs::RowArgs a;
    a.table = ctx->d_table;
    a.status = ctx->d_status;
    a.wait_cycles = hccs::kDefaultWaitCycles;
    a.rows = rows;
    a.H = H;
    a.Lq = Lq;
    a.Lk = Lk;
    a.causal_off = Lk - Lq;
    a.causal = (flags & HCCS_CAUSAL) ? 1 : 0;
    a.key_len = key_len;
    a.out_shift = ctx->out_shift;
    a.slice0 = 0;
    a.div_Lq = hccs::make_fastdiv((uint32_t)Lq);
    a.div_H = hccs::make_fastdiv((uint32_t)H);
    return a;
}

}  // namespace

extern "C" {

hccs_status_t hccs_create(hccs_ctx_t **out, int device) {
    if (!out) return HCCS_ERR_INVALID_ARG;
    *out = nullptr;
    int count = 0;
    if (cudaGetDeviceCount(&count) != cudaSuccess) { (void)cudaGetLastError(); return HCCS_ERR_CUDA; }
    if (device < 0 || device >= count) return HCCS_ERR_INVALID_ARG;
    DeviceGuard g(device);
    if (!g.ok) return HCCS_ERR_CUDA;
    hccs_ctx *ctx = new (std::nothrow) hccs_ctx();
    if (!ctx) return HCCS_ERR_INVALID_ARG;
    ctx->device = device;
    cudaError_t e = cudaMalloc(&ctx->d_status, 64 * sizeof(uint32_t));
    if (e == cudaSuccess) e = cudaMemset(ctx->d_status, 0, 64 * sizeof(uint32_t));
    if (e == cudaSuccess) e = cudaHostAlloc(&ctx->h_status, sizeof(uint32_t), cudaHostAllocDefault);
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&ctx->table_copied, cudaEventDisableTiming);
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&ctx->mult_copied, cudaEventDisableTiming);
    if (e == cudaSuccess) e = cudaStreamCreateWithFlags(&ctx->d2h_stream, cudaStreamNonBlocking);
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&ctx->ev_join, cudaEventDisableTiming);
    for (int i = 0; i < hccs_ctx::kMaxPieces && e == cudaSuccess; ++i) {
        e = cudaEventCreateWithFlags(&ctx->ev_done[i], cudaEventDisableTiming);
    }
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        hccs_destroy(ctx);
        return HCCS_ERR_CUDA;
    }
    *out = ctx;
    return HCCS_OK;
}

hccs_status_t hccs_destroy(hccs_ctx_t *ctx) {
    if (!ctx) return HCCS_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (ctx->d_table) cudaFree(ctx->d_table);
    if (ctx->h_table) cudaFreeHost(ctx->h_table);
    if (ctx->d_mult) cudaFree(ctx->d_mult);
    if (ctx->h_mult) cudaFreeHost(ctx->h_mult);
    delete[] ctx->mult_last;
    if (ctx->d_status) cudaFree(ctx->d_status);
    if (ctx->h_status) cudaFreeHost(ctx->h_status);
    if (ctx->table_copied) cudaEventDestroy(ctx->table_copied);
    if (ctx->mult_copied) cudaEventDestroy(ctx->mult_copied);
    if (ctx->d2h_stream) cudaStreamDestroy(ctx->d2h_stream);
    if (ctx->ev_join) cudaEventDestroy(ctx->ev_join);
    for (int i = 0; i < hccs_ctx::kMaxPieces; ++i) {
        if (ctx->ev_done[i]) cudaEventDestroy(ctx->ev_done[i]);
    }
    (void)cudaGetLastError();
    delete ctx;
    return HCCS_OK;
}

hccs_status_t hccs_params_check(const hccs_head_params_t *params, int32_t num_heads,
                                int32_t n_design, int32_t *bad_head) {
    if (bad_head) *bad_head = -1;
    if (!params || num_heads < 1 || num_heads > (1 << 20)) return HCCS_ERR_INVALID_ARG;
    if (n_design < 1 || n_design > 32767) return HCCS_ERR_INVALID_ARG;
    for (int32_t h = 0; h < num_heads; ++h) {
        if (!theta_admissible(params[h], n_design)) {
            if (bad_head) *bad_head = h;
            return HCCS_ERR_CONSTRAINT;
        }
    }
    return HCCS_OK;
}

// The checked table goes up on `stream`, and the context takes it.
static hccs_status_t upload_table(hccs_ctx_t *ctx, const hccs_head_params_t *params, int32_t num_heads,
                                  int32_t n_design, int32_t out_shift, bool wide, void *cuda_stream) {
    DeviceGuard g(ctx->device);
    if (!g.ok) return cuda_fail(ctx, cudaErrorInvalidDevice);
    hccs_status_t st = ensure_capacity(ctx, num_heads);
    if (st != HCCS_OK) return st;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    // the pinned staging copy may still be in flight from the previous upload
    HCCS_CUDA(ctx, cudaEventSynchronize(ctx->table_copied));
    for (int32_t h = 0; h < num_heads; ++h) {
        hccs::HeadEntry e;
        e.B = params[h].B;
        e.S = params[h].S;
        e.D = params[h].Dmax;
        e.pad = 0;
        ctx->h_table[h] = e;
    }
    HCCS_CUDA(ctx, cudaMemcpyAsync(ctx->d_table, ctx->h_table, sizeof(hccs::HeadEntry) * num_heads,
                                   cudaMemcpyHostToDevice, stream));
    HCCS_CUDA(ctx, cudaEventRecord(ctx->table_copied, stream));
    ctx->num_heads = num_heads;
    ctx->n_design = n_design;
    ctx->out_shift = out_shift;
    ctx->wide = wide;
    return HCCS_OK;
}

hccs_status_t hccs_params_upload(hccs_ctx_t *ctx, const hccs_head_params_t *params,
                                 int32_t num_heads, int32_t n_design, int32_t out_shift,
                                 int32_t *bad_head, void *cuda_stream) {
    if (bad_head) *bad_head = -1;
    if (!ctx) return HCCS_ERR_INVALID_ARG;
    if (out_shift < 0 || out_shift > 8) return HCCS_ERR_INVALID_ARG;
    hccs_status_t chk = hccs_params_check(params, num_heads, n_design, bad_head);
    if (chk != HCCS_OK) return chk;
    return upload_table(ctx, params, num_heads, n_design, out_shift, false, cuda_stream);
}

hccs_status_t hccs_params_upload_wide(hccs_ctx_t *ctx, const hccs_head_params_t *params, int32_t num_heads,
                                      int32_t n_design, int32_t *bad_head, void *cuda_stream) {
    if (bad_head) *bad_head = -1;
    if (!ctx || !params || num_heads < 1 || num_heads > HCCS_MAX_CACHE_HEADS) return HCCS_ERR_INVALID_ARG;
    if (n_design < 1 || n_design > HCCS_MAX_CACHE_KEYS) return HCCS_ERR_INVALID_ARG;
    for (int32_t h = 0; h < num_heads; ++h) {
        const int64_t B = params[h].B, S = params[h].S, D = params[h].Dmax;
        if (D < 1 || D > 127 || S < 0 || S > 127 || B < 1 || B > 32767 || B - S * D < 0) {
            if (bad_head) *bad_head = h;
            return HCCS_ERR_CONSTRAINT;
        }
    }
    return upload_table(ctx, params, num_heads, n_design, 0, true, cuda_stream);
}

hccs_status_t hccs_forward(hccs_ctx_t *ctx, const int8_t *logits, void *probs,
                           int32_t B, int32_t H, int32_t Lq, int32_t Lk,
                           uint32_t flags, void *cuda_stream) {
    hccs_status_t st = check_forward_args(ctx, logits, probs, B, H, Lq, Lk, flags);
    if (st != HCCS_OK) return st;
    const int64_t rows = (int64_t)B * H * Lq;
    if (rows * Lk == 0) return HCCS_OK;
    if ((flags & HCCS_OUT_U16) && (const void *)logits == probs) return HCCS_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (!g.ok) return cuda_fail(ctx, cudaErrorInvalidDevice);
    hccs::RowArgs a = make_row_args(ctx, (int32_t)rows, H, Lq, Lk, flags, nullptr);
    HCCS_CUDA(ctx, hccs::launch_rows(logits, probs, a, flags, (cudaStream_t)cuda_stream, &ctx->launches));
    return HCCS_OK;
}

hccs_status_t hccs_forward_keylen(hccs_ctx_t *ctx, const int8_t *logits, void *probs, const int32_t *key_len,
                                  int32_t B, int32_t H, int32_t Lq, int32_t Lk,
                                  uint32_t flags, void *cuda_stream) {
    hccs_status_t st = check_forward_args(ctx, logits, probs, B, H, Lq, Lk, flags);
    if (st != HCCS_OK) return st;
    const int64_t rows = (int64_t)B * H * Lq;
    if (rows * Lk == 0) return HCCS_OK;
    if (!key_len) return HCCS_ERR_INVALID_ARG;
    if ((flags & HCCS_OUT_U16) && (const void *)logits == probs) return HCCS_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (!g.ok) return cuda_fail(ctx, cudaErrorInvalidDevice);
    hccs::RowArgs a = make_row_args(ctx, (int32_t)rows, H, Lq, Lk, flags, key_len);
    HCCS_CUDA(ctx, hccs::launch_rows(logits, probs, a, flags, (cudaStream_t)cuda_stream, &ctx->launches));
    return HCCS_OK;
}

hccs_status_t hccs_forward_host(hccs_ctx_t *ctx, const int8_t *logits_host, void *probs_host,
                                int8_t *logits_staging, void *probs_staging,
                                int32_t B, int32_t H, int32_t Lq, int32_t Lk,
                                uint32_t flags, void *cuda_stream) {
    hccs_status_t st = check_forward_args(ctx, logits_host, probs_host, B, H, Lq, Lk, flags);
    if (st != HCCS_OK) return st;
    const int64_t rows = (int64_t)B * H * Lq;
    if (rows * Lk == 0) return HCCS_OK;
    if (!logits_staging || !probs_staging || (void *)logits_staging == probs_staging)
        return HCCS_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (!g.ok) return cuda_fail(ctx, cudaErrorInvalidDevice);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const int64_t osz = (flags & HCCS_OUT_U16) ? 2 : 1;
    // Pieces are whole (b, h) slices, so that a piece's first row has query index 0 and its
    // head is a pure function of the slice index.  A piece's input copy and its kernel run in order on
    // the caller's stream (the kernel of one piece delays the next copy by microseconds only); the
    // results come down on a second stream, piece by piece behind an event, so that the two copy
    // directions overlap.  One event hand-over per piece: each costs several microseconds of latency.
    const int64_t slices = (int64_t)B * H;
    const int64_t slice_bytes = (int64_t)Lq * Lk;
    int pieces = 1;
    if (slices * slice_bytes >= (8ll << 20)) pieces = 8;
    if (pieces > slices) pieces = (int)slices;
    for (int p = 0; p < pieces; ++p) {
        const int64_t s0 = slices * p / pieces, s1 = slices * (p + 1) / pieces;
        const int64_t off = s0 * slice_bytes, bytes = (s1 - s0) * slice_bytes;
        HCCS_CUDA(ctx, cudaMemcpyAsync(logits_staging + off, logits_host + off, bytes,
                                       cudaMemcpyHostToDevice, stream));
        // a piece starts at slice s0: the kernel runs on a view whose flat row 0 is that slice, and the
        // row arguments carry the starting slice so that (r / Lq) mod H still gives the head
        hccs::RowArgs a = make_row_args(ctx, (int32_t)((s1 - s0) * Lq), H, Lq, Lk, flags, nullptr);
        a.slice0 = (int32_t)s0;
        HCCS_CUDA(ctx, hccs::launch_rows(logits_staging + off, (char *)probs_staging + off * osz, a,
                                         flags, stream, &ctx->launches));
        HCCS_CUDA(ctx, cudaEventRecord(ctx->ev_done[p], stream));
        HCCS_CUDA(ctx, cudaStreamWaitEvent(ctx->d2h_stream, ctx->ev_done[p], 0));
        HCCS_CUDA(ctx, cudaMemcpyAsync((char *)probs_host + off * osz, (char *)probs_staging + off * osz,
                                       bytes * osz, cudaMemcpyDeviceToHost, ctx->d2h_stream));
    }
    HCCS_CUDA(ctx, cudaEventRecord(ctx->ev_join, ctx->d2h_stream));
    HCCS_CUDA(ctx, cudaStreamWaitEvent(stream, ctx->ev_join, 0));
    return HCCS_OK;
}

// Shared by the int32, fp32 and int8 entry points: out_scale != NULL means fp32 output, out_mult != NULL
// int8 output, neither int32 output.
static hccs_status_t fused_common(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *K, const int8_t *V, void *O,
                                  const float *out_scale, const int32_t *out_mult, int32_t out_shift,
                                  const int32_t *key_len, const int32_t *requant_mult,
                                  int32_t requant_shift, int32_t B, int32_t H, int32_t L, int32_t d,
                                  uint32_t flags, void *cuda_stream) {
    if (!ctx || B < 0 || H < 0 || L < 0 || d < 0) return HCCS_ERR_INVALID_ARG;
    if (flags & ~7u) return HCCS_ERR_INVALID_ARG;
    if (flags & HCCS_OUT_U16) return HCCS_ERR_UNSUPPORTED;
    if (ctx->num_heads == 0) return HCCS_ERR_NOT_UPLOADED;
    if (H != ctx->num_heads || !requant_mult) return HCCS_ERR_INVALID_ARG;
    if (requant_shift < 1 || requant_shift > 31) return HCCS_ERR_INVALID_ARG;
    for (int32_t h = 0; h < H; ++h)
        if (requant_mult[h] < 0 || requant_mult[h] >= (1 << 13)) return HCCS_ERR_INVALID_ARG;
    if (out_mult) {
        if (out_shift < 1 || out_shift > 31) return HCCS_ERR_INVALID_ARG;
        for (int32_t h = 0; h < H; ++h)
            if (out_mult[h] < 0 || out_mult[h] >= (1 << 13)) return HCCS_ERR_INVALID_ARG;
    }
    // the kernel requantises with the multiplier pre-shifted by 32 - requant_shift bits
    for (int32_t h = 0; h < H; ++h)
        if ((int64_t)requant_mult[h] << (32 - requant_shift) >= (1ll << 31)) return HCCS_ERR_UNSUPPORTED;
    if (ctx->wide || L > ctx->n_design) return HCCS_ERR_CONSTRAINT;
    if ((int64_t)B * H * L * d == 0) return HCCS_OK;
    if (!Q || !K || !V || !O) return HCCS_ERR_INVALID_ARG;
    if (!hccs::fused_shape_supported(L, d)) return HCCS_ERR_UNSUPPORTED;
    if ((((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O) & 15u) != 0)
        return HCCS_ERR_UNSUPPORTED;
    DeviceGuard g(ctx->device);
    if (!g.ok) return cuda_fail(ctx, cudaErrorInvalidDevice);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    // Per head: {multiplier, and for shifts up to 24 the constants of the single-multiply
    // requantisation: multiplier << k, offset, -lo, hi - lo} (see hccs_fused.cu, phase 1), then the
    // fp32 output scale, the int8 output multiplier and 1 / multiplier as a double; eight 32-bit words per head.
    // The words are built on the stack and go up only when they differ from what the device table
    // already holds (the usual case is the same multipliers call after call): then nothing is copied
    // and the host never waits for an earlier call's copy.
    constexpr int32_t kStackHeads = 64;
    int32_t stack_words[8 * kStackHeads];
    int32_t *words = H <= kStackHeads ? stack_words : new (std::nothrow) int32_t[8 * (size_t)H];
    if (!words) return HCCS_ERR_INVALID_ARG;
    for (int32_t h = 0; h < H; ++h) {
        const int64_t M = requant_mult[h];
        int32_t *e = words + 8 * h;
        e[0] = (int32_t)M;
        e[1] = e[2] = e[3] = e[6] = e[7] = 0;
        e[5] = out_mult ? out_mult[h] : 0;
        const float scale = out_scale ? out_scale[h] : 1.0f;
        memcpy(&e[4], &scale, sizeof(float));
        const double inv_m = M > 0 ? 1.0 / (double)M : 0.0;      // words 6 and 7
        memcpy(&e[6], &inv_m, sizeof(double));
        if (requant_shift <= 24) {
            const int sh = requant_shift, k = 24 - sh;
            const int64_t R = (int64_t)1 << (sh - 1), lim = (int64_t)1 << 21;   // |acc| <= d*128*128 <= 2^21
            int64_t lo = -lim, hi = lim;
            if (M > 0) {
                lo = -((((int64_t)128 << sh) + R) / M);          // smallest accumulator that gives -128
                hi = (((int64_t)128 << sh) - 1 - R) / M;         // largest accumulator that gives 127
                if (lo < -lim) lo = -lim;
                if (hi > lim) hi = lim;
            }
            e[0] = (int32_t)(uint32_t)((uint64_t)M << k);
            e[1] = (int32_t)(uint32_t)(uint64_t)((lo * M + R) * ((int64_t)1 << k));
            e[2] = (int32_t)-lo;
            e[3] = (int32_t)(hi - lo);
        }
    }
    const bool same = ctx->mult_last_heads == H && memcmp(ctx->mult_last, words, sizeof(int32_t) * 8 * H) == 0;
    if (!same) {
        // the pinned staging copy may still be in flight from the previous upload
        cudaError_t e = cudaEventSynchronize(ctx->mult_copied);
        if (e == cudaSuccess) {
            memcpy(ctx->h_mult, words, sizeof(int32_t) * 8 * H);
            e = cudaMemcpyAsync(ctx->d_mult, ctx->h_mult, sizeof(int32_t) * 8 * H, cudaMemcpyHostToDevice, stream);
        }
        if (e == cudaSuccess) e = cudaEventRecord(ctx->mult_copied, stream);
        if (e == cudaSuccess) {
            memcpy(ctx->mult_last, words, sizeof(int32_t) * 8 * H);
            ctx->mult_last_heads = H;
        } else {
            ctx->mult_last_heads = 0;
        }
        if (words != stack_words) delete[] words;
        if (e != cudaSuccess) return cuda_fail(ctx, e);
    } else {
        if (words != stack_words) delete[] words;
        // the table went up on the stream of an earlier call: order this stream behind that copy
        HCCS_CUDA(ctx, cudaStreamWaitEvent(stream, ctx->mult_copied, 0));
    }
    hccs::FusedArgs a;
    a.Q = Q; a.K = K; a.V = V; a.O = O;
    a.table = ctx->d_table;
    a.requant_mult = ctx->d_mult;
    a.status = ctx->d_status;
    a.wait_cycles = hccs::kDefaultWaitCycles;
    a.out_mode = out_scale ? 1 : (out_mult ? 2 : 0);
    a.out_requant_shift = out_mult ? out_shift : 1;
    a.key_len = key_len;
    a.requant_shift = requant_shift;
    a.B = B; a.H = H; a.L = L; a.d = d;
    a.out_shift = ctx->out_shift;
    a.flags = flags;
    HCCS_CUDA(ctx, hccs::launch_fused(a, stream, &ctx->launches));
    return HCCS_OK;
}

hccs_status_t hccs_attention_fused(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *K,
                                   const int8_t *V, int32_t *O, const int32_t *requant_mult,
                                   int32_t requant_shift, int32_t B, int32_t H, int32_t L, int32_t d,
                                   uint32_t flags, void *cuda_stream) {
    return fused_common(ctx, Q, K, V, O, nullptr, nullptr, 0, nullptr, requant_mult, requant_shift, B, H, L, d, flags, cuda_stream);
}

hccs_status_t hccs_attention_fused_keylen(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *K,
                                          const int8_t *V, int32_t *O, const int32_t *key_len,
                                          const int32_t *requant_mult, int32_t requant_shift,
                                          int32_t B, int32_t H, int32_t L, int32_t d,
                                          uint32_t flags, void *cuda_stream) {
    if (!key_len && (int64_t)B * H * L * d != 0) return HCCS_ERR_INVALID_ARG;
    return fused_common(ctx, Q, K, V, O, nullptr, nullptr, 0, key_len, requant_mult, requant_shift, B, H, L, d, flags, cuda_stream);
}

hccs_status_t hccs_attention_fused_f32(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *K,
                                       const int8_t *V, float *O, const float *out_scale,
                                       const int32_t *requant_mult, int32_t requant_shift,
                                       int32_t B, int32_t H, int32_t L, int32_t d,
                                       uint32_t flags, void *cuda_stream) {
    if (!out_scale) return HCCS_ERR_INVALID_ARG;
    return fused_common(ctx, Q, K, V, O, out_scale, nullptr, 0, nullptr, requant_mult, requant_shift, B, H, L, d, flags, cuda_stream);
}

hccs_status_t hccs_attention_fused_i8(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *K,
                                      const int8_t *V, int8_t *O, const int32_t *out_mult, int32_t out_shift,
                                      const int32_t *requant_mult, int32_t requant_shift,
                                      int32_t B, int32_t H, int32_t L, int32_t d,
                                      uint32_t flags, void *cuda_stream) {
    if (!out_mult) return HCCS_ERR_INVALID_ARG;
    return fused_common(ctx, Q, K, V, O, nullptr, out_mult, out_shift, nullptr, requant_mult, requant_shift, B, H, L, d, flags, cuda_stream);
}

hccs_status_t hccs_device_status(hccs_ctx_t *ctx, uint32_t *word, void *cuda_stream) {
    if (!ctx) return HCCS_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (!g.ok) return cuda_fail(ctx, cudaErrorInvalidDevice);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    HCCS_CUDA(ctx, cudaMemcpyAsync(ctx->h_status, ctx->d_status, sizeof(uint32_t),
                                   cudaMemcpyDeviceToHost, stream));
    HCCS_CUDA(ctx, cudaMemsetAsync(ctx->d_status, 0, sizeof(uint32_t), stream));
    HCCS_CUDA(ctx, cudaStreamSynchronize(stream));
    const uint32_t w = *ctx->h_status;
    if (word) *word = w;
    if (w & (hccs::STATUS_ROW_TMA_TIMEOUT | hccs::STATUS_FUSED_TIMEOUT)) return HCCS_ERR_DEVICE_TIMEOUT;
    return w ? HCCS_ERR_DEVICE_INDEX : HCCS_OK;
}

// ---- generation over an int8 cache

static bool cache_shape(int32_t Hkv, int32_t d, int32_t num_pages, int32_t page_size, int32_t *page_shift) {
    if (Hkv < 1 || Hkv > HCCS_MAX_CACHE_HEADS || num_pages < 1 || page_size < 16 || page_size > 65536) return false;
    if ((page_size & (page_size - 1)) != 0 || (int64_t)num_pages * Hkv >= (1ll << 31)) return false;
    *page_shift = 0;
    while ((1 << *page_shift) < page_size) ++*page_shift;
    return d == 64 || d == 128;
}

static bool steps_ok(const float *s, int32_t n) {
    if (!s) return false;
    for (int32_t i = 0; i < n; ++i)
        if (!(s[i] >= 0x1p-100f) || !(s[i] <= 0x1p100f)) return false;
    return true;
}

static bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

hccs_status_t hccs_rope_frequencies(hccs_rope_t *rope, int32_t rot_dim, int32_t interleaved, double base,
                                    const hccs_rope_scaling_t *scaling) {
    if (!rope || rot_dim < 2 || rot_dim > HCCS_MAX_ROT_DIM || (rot_dim & 1)) return HCCS_ERR_INVALID_ARG;
    if (!(base > 1.0) || !isfinite(base)) return HCCS_ERR_INVALID_ARG;
    const int32_t kind = scaling ? scaling->kind : HCCS_ROPE_NONE;
    const double factor = kind == HCCS_ROPE_NONE ? 1.0 : scaling->factor;
    if (kind < HCCS_ROPE_NONE || kind > HCCS_ROPE_DIMENSION || !(factor >= 1.0) || !isfinite(factor)) return HCCS_ERR_INVALID_ARG;
    if (kind == HCCS_ROPE_BASE && rot_dim <= 2) return HCCS_ERR_INVALID_ARG;
    const bool mixed = kind == HCCS_ROPE_WAVELENGTH || kind == HCCS_ROPE_DIMENSION;
    if (mixed && (!(scaling->low > 0.0) || !(scaling->high > scaling->low) || !isfinite(scaling->high) ||
                  !(scaling->original_len > 0.0) || !isfinite(scaling->original_len)))
        return HCCS_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    if (kind == HCCS_ROPE_BASE) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
    double first = 0.0, last = 0.0;                  // DIMENSION: the pairs between which the mixture changes
    if (kind == HCCS_ROPE_DIMENSION) {
        first = floor(rot_dim * log(scaling->original_len / (scaling->high * two_pi)) / (2.0 * log(base)));
        last = ceil(rot_dim * log(scaling->original_len / (scaling->low * two_pi)) / (2.0 * log(base)));
        first = fmax(first, 0.0);
        last = fmin(last, (double)(rot_dim - 1));
        if (last <= first) last = first + 0.001;
    }
    rope->rot_dim = rot_dim;
    rope->interleaved = interleaved ? 1 : 0;
    rope->scale = kind == HCCS_ROPE_DIMENSION ? 0.1 * log(factor) + 1.0 : 1.0;
    for (int32_t i = 0; i < HCCS_MAX_ROT_DIM / 2; ++i) {
        if (i >= rot_dim / 2) { rope->freq[i] = 0.0; continue; }
        double f = pow(base, -2.0 * i / rot_dim);
        if (kind == HCCS_ROPE_LINEAR) f /= factor;
        if (mixed) {
            double keep;
            if (kind == HCCS_ROPE_WAVELENGTH)
                keep = (scaling->original_len * f / two_pi - scaling->low) / (scaling->high - scaling->low);
            else
                keep = 1.0 - (i - first) / (last - first);
            keep = fmin(fmax(keep, 0.0), 1.0);
            f = f * keep + f / factor * (1.0 - keep);
        }
        rope->freq[i] = f;
    }
    return HCCS_OK;
}

hccs_status_t hccs_rope_axes(hccs_rope_axes_t *axes, int32_t rot_dim, int32_t interleaved, double base,
                             const hccs_rope_scaling_t *scaling, const int32_t *pairs, int32_t num_axes,
                             int32_t order, int32_t restart) {
    if (!axes || !pairs || num_axes < 1 || num_axes > HCCS_MAX_AXES) return HCCS_ERR_INVALID_ARG;
    if (order != HCCS_AXES_SECTIONS && order != HCCS_AXES_TURNS) return HCCS_ERR_INVALID_ARG;
    hccs_rope_axes_t got;
    memset(&got, 0, sizeof(got));
    hccs_status_t st = hccs_rope_frequencies(&got.rope, rot_dim, interleaved, base, scaling);
    if (st != HCCS_OK) return st;
    int64_t sum = 0;
    for (int32_t x = 0; x < num_axes; ++x) {
        if (pairs[x] < 0) return HCCS_ERR_INVALID_ARG;
        sum += pairs[x];
    }
    if (sum != rot_dim / 2) return HCCS_ERR_INVALID_ARG;
    got.num_axes = num_axes;
    hccs_rope_t own[HCCS_MAX_AXES];
    int32_t dealt[HCCS_MAX_AXES] = {0, 0, 0, 0};
    if (restart)
        for (int32_t x = 0; x < num_axes; ++x) {
            if (pairs[x] == 0) continue;
            st = hccs_rope_frequencies(&own[x], 2 * pairs[x], interleaved, base, scaling);
            if (st != HCCS_OK) return st;
        }
    for (int32_t i = 0, x = 0; i < rot_dim / 2; ++i) {
        while (dealt[x] == pairs[x]) x = (x + 1) % num_axes;
        got.axis[i] = (uint8_t)x;
        if (restart) got.rope.freq[i] = own[x].freq[dealt[x]];
        ++dealt[x];
        if (order == HCCS_AXES_TURNS) x = (x + 1) % num_axes;
    }
    *axes = got;
    return HCCS_OK;
}

// Where the new tokens of a write come from and go to, besides the kernel's own arguments.
struct WriteCall {
    const void *q, *k, *v;
    hccs_type_t type;
    int64_t q_stride, k_stride, v_stride;
    const int32_t *positions;
    int64_t axis_stride, token_stride;
    const int64_t *slots;
    const hccs_rope_t *rope;
    const hccs_rope_axes_t *axes;               // NULL: one axis
    const float *q_step, *k_step, *v_step;
    int8_t *q8, *k8, *v8;
    int32_t T, L, Hq, Hkv, d;                   // L: 0 for pages
    int32_t num_pages, page_size;
};

static hccs_status_t write_tokens(hccs_ctx_t *ctx, const WriteCall &w, void *cuda_stream) {
    const int32_t T = w.T, d = w.d;
    const hccs_rope_t *rope = w.rope;
    if (T < 0) return HCCS_ERR_INVALID_ARG;
    if (w.type != HCCS_F32 && w.type != HCCS_BF16 && w.type != HCCS_F16) return HCCS_ERR_INVALID_ARG;
    const bool with_q = w.q != nullptr, with_kv = w.k != nullptr, paged = w.L == 0;
    if ((w.k == nullptr) != (w.v == nullptr)) return HCCS_ERR_INVALID_ARG;
    int32_t page_shift = 0;
    if (d != 64 && d != 128) return HCCS_ERR_UNSUPPORTED;
    if (with_kv && (paged ? !cache_shape(w.Hkv, d, w.num_pages, w.page_size, &page_shift) : w.Hkv < 1 || w.Hkv > HCCS_MAX_CACHE_HEADS))
        return HCCS_ERR_INVALID_ARG;
    if (with_q && (w.Hq < 1 || w.Hq > HCCS_MAX_CACHE_HEADS)) return HCCS_ERR_INVALID_ARG;
    if (with_q && !steps_ok(w.q_step, w.Hq)) return HCCS_ERR_INVALID_ARG;
    if (with_kv && (!steps_ok(w.k_step, w.Hkv) || !steps_ok(w.v_step, w.Hkv))) return HCCS_ERR_INVALID_ARG;
    if (rope) {
        if (rope->rot_dim < 0 || rope->rot_dim > d || (rope->rot_dim & 1)) return HCCS_ERR_INVALID_ARG;
        if (!(fabs(rope->scale) >= 0x1p-64) || !(fabs(rope->scale) <= 0x1p64)) return HCCS_ERR_INVALID_ARG;
        for (int32_t i = 0; i < rope->rot_dim / 2; ++i)
            if (!isfinite(rope->freq[i])) return HCCS_ERR_INVALID_ARG;
    }
    if (w.axes) {
        if (w.axes->num_axes < 1 || w.axes->num_axes > HCCS_MAX_AXES) return HCCS_ERR_INVALID_ARG;
        for (int32_t i = 0; i < rope->rot_dim / 2; ++i)
            if (w.axes->axis[i] >= w.axes->num_axes) return HCCS_ERR_INVALID_ARG;
    }
    const bool turns = rope && rope->rot_dim > 0;
    if (T == 0 || (!with_q && !with_kv)) return ctx ? HCCS_OK : HCCS_ERR_INVALID_ARG;
    if (!paged && (w.L < 1 || T % w.L != 0)) return HCCS_ERR_INVALID_ARG;
    if ((turns && !w.positions) || (with_q && !w.q8) || (with_kv && ((paged && !w.slots) || !w.k8 || !w.v8))) return HCCS_ERR_INVALID_ARG;
    const int64_t esz = w.type == HCCS_F32 ? 4 : 2;
    if (with_q && (!aligned16(w.q) || !aligned16(w.q8) || (w.q_stride * esz) % 16 != 0)) return HCCS_ERR_UNSUPPORTED;
    if (with_kv && (!aligned16(w.k) || !aligned16(w.v) || !aligned16(w.k8) || !aligned16(w.v8) ||
                    (w.k_stride * esz) % 16 != 0 || (w.v_stride * esz) % 16 != 0))
        return HCCS_ERR_UNSUPPORTED;
    if (!ctx) return HCCS_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (!g.ok) return cuda_fail(ctx, cudaErrorInvalidDevice);
    hccs::CacheWriteArgs a;
    memset(&a, 0, sizeof(a));
    a.q = w.q; a.k = w.k; a.v = w.v;
    a.q_stride = w.q_stride; a.k_stride = w.k_stride; a.v_stride = w.v_stride;
    a.positions = w.positions; a.axis_stride = w.axis_stride; a.token_stride = w.token_stride;
    a.slots = w.slots;
    a.q8 = w.q8; a.k_pages = w.k8; a.v_pages = w.v8;
    a.status = ctx->d_status;
    a.num_slots = with_kv && paged ? (int64_t)w.num_pages * w.page_size : 0;
    a.T = T; a.Hq = with_q ? w.Hq : 0; a.Hkv = with_kv ? w.Hkv : 0; a.d = d; a.page_shift = page_shift;
    a.dense_len = w.L;
    if (turns) a.rope = *rope;
    a.axes = w.axes != nullptr;
    if (turns && w.axes) memcpy(a.axis, w.axes->axis, sizeof(a.axis));
    if (with_q) memcpy(a.step, w.q_step, sizeof(float) * w.Hq);
    if (with_kv) {
        memcpy(a.step + HCCS_MAX_CACHE_HEADS, w.k_step, sizeof(float) * w.Hkv);
        memcpy(a.step + 2 * HCCS_MAX_CACHE_HEADS, w.v_step, sizeof(float) * w.Hkv);
    }
    HCCS_CUDA(ctx, hccs::launch_cache_write(a, w.type, (cudaStream_t)cuda_stream, &ctx->launches));
    return HCCS_OK;
}

hccs_status_t hccs_cache_write(hccs_ctx_t *ctx, const void *q, const void *k, const void *v, hccs_type_t type,
                               int64_t q_stride, int64_t k_stride, int64_t v_stride,
                               const int32_t *positions, const int64_t *slots, const hccs_rope_t *rope,
                               const float *q_step, const float *k_step, const float *v_step,
                               int8_t *q8, int8_t *k_pages, int8_t *v_pages,
                               int32_t T, int32_t Hq, int32_t Hkv, int32_t d,
                               int32_t num_pages, int32_t page_size, void *cuda_stream) {
    return write_tokens(ctx, {q, k, v, type, q_stride, k_stride, v_stride, positions, 0, 1, slots, rope, nullptr, q_step, k_step, v_step,
                              q8, k_pages, v_pages, T, 0, Hq, Hkv, d, num_pages, page_size}, cuda_stream);
}

hccs_status_t hccs_cache_write_axes(hccs_ctx_t *ctx, const void *q, const void *k, const void *v, hccs_type_t type,
                                    int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                    const int32_t *positions, int64_t axis_stride, int64_t token_stride,
                                    const int64_t *slots, const hccs_rope_axes_t *axes,
                                    const float *q_step, const float *k_step, const float *v_step,
                                    int8_t *q8, int8_t *k_pages, int8_t *v_pages,
                                    int32_t T, int32_t Hq, int32_t Hkv, int32_t d,
                                    int32_t num_pages, int32_t page_size, void *cuda_stream) {
    return write_tokens(ctx, {q, k, v, type, q_stride, k_stride, v_stride, positions, axis_stride, token_stride, slots,
                              axes ? &axes->rope : nullptr, axes, q_step, k_step, v_step,
                              q8, k_pages, v_pages, T, 0, Hq, Hkv, d, num_pages, page_size}, cuda_stream);
}

hccs_status_t hccs_states_write(hccs_ctx_t *ctx, const void *q, const void *k, const void *v, hccs_type_t type,
                                int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                const int32_t *positions, int64_t axis_stride, int64_t token_stride,
                                const hccs_rope_axes_t *axes,
                                const float *q_step, const float *k_step, const float *v_step,
                                int8_t *q8, int8_t *k8, int8_t *v8,
                                int32_t T, int32_t L, int32_t Hq, int32_t Hkv, int32_t d, void *cuda_stream) {
    if (L < 1) return HCCS_ERR_INVALID_ARG;
    return write_tokens(ctx, {q, k, v, type, q_stride, k_stride, v_stride, positions, axis_stride, token_stride, nullptr,
                              axes ? &axes->rope : nullptr, axes, q_step, k_step, v_step,
                              q8, k8, v8, T, L, Hq, Hkv, d, 0, 0}, cuda_stream);
}

hccs_status_t hccs_cache_read(hccs_ctx_t *ctx, const int8_t *k_pages, const int8_t *v_pages,
                              const int32_t *page_table, const int32_t *out_start,
                              const float *k_step, const float *v_step, void *k_out, void *v_out, hccs_type_t type,
                              int32_t B, int32_t max_pages, int32_t max_len, int32_t rows, int32_t Hkv, int32_t d,
                              int32_t num_pages, int32_t page_size, void *cuda_stream) {
    if (B < 0 || max_pages < 0 || max_len < 0 || rows < 0) return HCCS_ERR_INVALID_ARG;
    if (type != HCCS_F32 && type != HCCS_BF16 && type != HCCS_F16) return HCCS_ERR_INVALID_ARG;
    if (d != 64 && d != 128) return HCCS_ERR_UNSUPPORTED;
    int32_t page_shift = 0;
    if (!cache_shape(Hkv, d, num_pages, page_size, &page_shift)) return HCCS_ERR_INVALID_ARG;
    if ((k_out && (!k_pages || !steps_ok(k_step, Hkv))) || (v_out && (!v_pages || !steps_ok(v_step, Hkv)))) return HCCS_ERR_INVALID_ARG;
    if (B > 65535) return HCCS_ERR_UNSUPPORTED;
    if (B == 0 || max_len == 0 || rows == 0 || (!k_out && !v_out)) return ctx ? HCCS_OK : HCCS_ERR_INVALID_ARG;
    if ((!page_table && max_pages > 0) || !out_start) return HCCS_ERR_INVALID_ARG;
    if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned16(k_out) || !aligned16(v_out)) return HCCS_ERR_UNSUPPORTED;
    if (!ctx) return HCCS_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (!g.ok) return cuda_fail(ctx, cudaErrorInvalidDevice);
    hccs::CacheReadArgs a;
    memset(&a, 0, sizeof(a));
    a.k_pages = k_pages; a.v_pages = v_pages;
    a.page_table = page_table; a.out_start = out_start;
    a.k_out = k_out; a.v_out = v_out;
    a.status = ctx->d_status;
    a.B = B; a.max_pages = max_pages; a.max_len = max_len; a.rows = rows;
    a.Hkv = Hkv; a.d = d; a.num_pages = num_pages; a.page_shift = page_shift;
    if (k_out) memcpy(a.step, k_step, sizeof(float) * Hkv);
    if (v_out) memcpy(a.step + HCCS_MAX_CACHE_HEADS, v_step, sizeof(float) * Hkv);
    HCCS_CUDA(ctx, hccs::launch_cache_read(a, type, (cudaStream_t)cuda_stream, &ctx->launches));
    return HCCS_OK;
}

// What the two calls of attention to int8 states check alike: first what needs no context, then the context.
static hccs_status_t states_attention_shape(const int32_t *requant_mult, int32_t requant_shift, const float *out_scale, int32_t B, int32_t Hq,
                                            int32_t Hkv, int32_t max_q, int32_t max_kv) {
    if (Hq > HCCS_MAX_CACHE_HEADS || B > 65535 || max_kv > HCCS_MAX_CACHE_KEYS) return HCCS_ERR_UNSUPPORTED;
    if ((int64_t)max_q * (Hq / Hkv) > (1ll << 30)) return HCCS_ERR_UNSUPPORTED;
    if (requant_shift < 1 || requant_shift > 24) return HCCS_ERR_INVALID_ARG;
    for (int32_t h = 0; h < Hq; ++h)
        if (requant_mult[h] < 0 || requant_mult[h] >= (1 << 13)) return HCCS_ERR_INVALID_ARG;
    for (int32_t h = 0; h < Hq; ++h)      // the steps of the requantisation stay below one
        if ((int64_t)requant_mult[h] >= (1ll << (requant_shift - 1))) return HCCS_ERR_UNSUPPORTED;
    if (out_scale)
        for (int32_t h = 0; h < Hq; ++h)
            if (!isfinite(out_scale[h])) return HCCS_ERR_INVALID_ARG;
    return HCCS_OK;
}
static hccs_status_t states_attention_context(const hccs_ctx_t *ctx, int32_t Hq, int32_t max_kv, uint32_t flags) {
    if (!ctx) return HCCS_ERR_INVALID_ARG;
    if (ctx->num_heads == 0) return HCCS_ERR_NOT_UPLOADED;
    if (Hq != ctx->num_heads) return HCCS_ERR_INVALID_ARG;
    if ((ctx->wide && flags != HCCS_RECIP_REAL) || max_kv > ctx->n_design) return HCCS_ERR_CONSTRAINT;
    return HCCS_OK;
}
static bool states_attention_types(hccs_type_t out_type, const float *out_scale, uint32_t flags) {
    if (flags != HCCS_RECIP_DIV && flags != HCCS_RECIP_CLB && flags != HCCS_RECIP_REAL) return false;
    if (out_type != HCCS_I32 && out_type != HCCS_F32 && out_type != HCCS_BF16 && out_type != HCCS_F16) return false;
    return out_type == HCCS_I32 ? flags != HCCS_RECIP_REAL && !out_scale : out_scale != nullptr;
}
static void states_attention_args(hccs::CachedAttnArgs &a, const hccs_ctx_t *ctx, const int32_t *requant_mult, int32_t requant_shift,
                                  const float *out_scale, hccs_type_t out_type, int32_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t d,
                                  int32_t max_q, int32_t max_kv, uint32_t flags) {
    a.table = ctx->d_table;
    a.status = ctx->d_status;
    a.wait_cycles = hccs::kDefaultWaitCycles;
    a.out_type = out_type; a.recip = (int32_t)flags;
    a.T = T; a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.group = Hq / Hkv; a.d = d;
    a.max_q = max_q; a.max_kv = max_kv; a.requant_shift = requant_shift;
    for (int32_t h = 0; h < Hq; ++h) {
        a.mult[h] = (uint16_t)requant_mult[h];
        a.scale[h] = out_scale ? out_scale[h] : 1.0f;
    }
}

hccs_status_t hccs_attention_cached(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *k_pages, const int8_t *v_pages,
                                    const int32_t *page_table, const int32_t *q_start, const int32_t *kv_len,
                                    const int32_t *tree_mask, int32_t tree_words,
                                    const int32_t *requant_mult, int32_t requant_shift, const float *out_scale,
                                    void *O, hccs_type_t out_type,
                                    int32_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t d, int32_t max_pages,
                                    int32_t num_pages, int32_t page_size, int32_t max_q, int32_t max_kv,
                                    uint32_t flags, void *cuda_stream) {
    // what needs no context first
    if (T < 0 || B < 0 || max_pages < 0 || max_q < 0 || max_kv < 0) return HCCS_ERR_INVALID_ARG;
    if (!states_attention_types(out_type, out_scale, flags)) return HCCS_ERR_INVALID_ARG;
    if (d != 64 && d != 128) return HCCS_ERR_UNSUPPORTED;
    int32_t page_shift = 0;
    if (!requant_mult || Hq < 1 || !cache_shape(Hkv, d, num_pages, page_size, &page_shift) || Hq % Hkv != 0) return HCCS_ERR_INVALID_ARG;
    hccs_status_t st = states_attention_shape(requant_mult, requant_shift, out_scale, B, Hq, Hkv, max_q, max_kv);
    if (st != HCCS_OK) return st;
    if (tree_mask && (tree_words < 1 || (int64_t)tree_words * 32 < max_q)) return HCCS_ERR_INVALID_ARG;
    const bool empty = T == 0 || B == 0 || max_q == 0;
    if (!empty && (!Q || !k_pages || !v_pages || (!page_table && max_pages > 0) || !q_start || !kv_len || !O)) return HCCS_ERR_INVALID_ARG;
    if (!aligned16(Q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(O)) return HCCS_ERR_UNSUPPORTED;
    st = states_attention_context(ctx, Hq, max_kv, flags);
    if (st != HCCS_OK || empty) return st;
    DeviceGuard g(ctx->device);
    if (!g.ok) return cuda_fail(ctx, cudaErrorInvalidDevice);
    hccs::CachedAttnArgs a;
    memset(&a, 0, sizeof(a));
    states_attention_args(a, ctx, requant_mult, requant_shift, out_scale, out_type, T, B, Hq, Hkv, d, max_q, max_kv, flags);
    a.Q = Q; a.k_pages = k_pages; a.v_pages = v_pages;
    a.page_table = page_table; a.q_start = q_start; a.kv_len = kv_len; a.tree_mask = tree_mask;
    a.O = O;
    a.tree_words = tree_words;
    a.max_pages = max_pages; a.num_pages = num_pages; a.page_shift = page_shift;
    HCCS_CUDA(ctx, hccs::launch_cached_attention(a, (cudaStream_t)cuda_stream, &ctx->launches));
    return HCCS_OK;
}

hccs_status_t hccs_attention_cross(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *K, const int8_t *V,
                                   int64_t k_stride, int64_t v_stride, const int32_t *q_start,
                                   const int32_t *k_start, const int32_t *k_len, const int32_t *key_range,
                                   const int32_t *requant_mult, int32_t requant_shift, const float *out_scale,
                                   void *O, hccs_type_t out_type,
                                   int32_t T, int32_t S, int32_t B, int32_t Hq, int32_t Hkv, int32_t d,
                                   int32_t max_q, int32_t max_kv, uint32_t flags, void *cuda_stream) {
    if (T < 0 || S < 0 || B < 0 || max_q < 0 || max_kv < 0) return HCCS_ERR_INVALID_ARG;
    if (!states_attention_types(out_type, out_scale, flags)) return HCCS_ERR_INVALID_ARG;
    if (d != 64 && d != 128) return HCCS_ERR_UNSUPPORTED;
    if (!requant_mult || Hq < 1 || Hkv < 1 || Hkv > HCCS_MAX_CACHE_HEADS || Hq % Hkv != 0) return HCCS_ERR_INVALID_ARG;
    hccs_status_t st = states_attention_shape(requant_mult, requant_shift, out_scale, B, Hq, Hkv, max_q, max_kv);
    if (st != HCCS_OK) return st;
    const bool empty = T == 0 || B == 0 || max_q == 0;
    if (!empty && (!Q || (S > 0 && (!K || !V)) || !q_start || !k_start || !k_len || !O)) return HCCS_ERR_INVALID_ARG;
    if (S > 0 && (k_stride < (int64_t)Hkv * d || v_stride < (int64_t)Hkv * d)) return HCCS_ERR_INVALID_ARG;
    if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || ((uintptr_t)key_range & 7u) != 0) return HCCS_ERR_UNSUPPORTED;
    if (S > 0 && (k_stride % 16 != 0 || v_stride % 16 != 0 || k_stride >= (1ll << 36) || v_stride >= (1ll << 36))) return HCCS_ERR_UNSUPPORTED;
    st = states_attention_context(ctx, Hq, max_kv, flags);
    if (st != HCCS_OK || empty) return st;
    DeviceGuard g(ctx->device);
    if (!g.ok) return cuda_fail(ctx, cudaErrorInvalidDevice);
    hccs::CachedAttnArgs a;
    memset(&a, 0, sizeof(a));
    states_attention_args(a, ctx, requant_mult, requant_shift, out_scale, out_type, T, B, Hq, Hkv, d, max_q, max_kv, flags);
    a.Q = Q; a.k_pages = K; a.v_pages = V;
    a.k_stride = k_stride; a.v_stride = v_stride;
    a.q_start = q_start; a.k_start = k_start; a.kv_len = k_len; a.key_range = key_range;
    a.states = S;
    a.O = O;
    HCCS_CUDA(ctx, hccs::launch_cross_attention(a, (cudaStream_t)cuda_stream, &ctx->launches));
    return HCCS_OK;
}

hccs_status_t hccs_debug_wait_timeout(hccs_ctx_t *ctx, int32_t mode, int64_t limit_cycles, void *cuda_stream) {
    if (!ctx || (mode != 0 && mode != 1)) return HCCS_ERR_INVALID_ARG;
    if (limit_cycles < 1 || limit_cycles > 10000000) return HCCS_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (!g.ok) return cuda_fail(ctx, cudaErrorInvalidDevice);
    HCCS_CUDA(ctx, hccs::launch_wait_probe(ctx->d_status, mode, (long long)limit_cycles, (cudaStream_t)cuda_stream));
    ctx->launches += 1;
    return HCCS_OK;
}

int32_t hccs_last_cuda_error(const hccs_ctx_t *ctx) { return ctx ? ctx->last_cuda_error : 0; }

uint64_t hccs_launch_count(const hccs_ctx_t *ctx) { return ctx ? ctx->launches : 0; }

const char *hccs_status_string(hccs_status_t status) {
    switch (status) {
        case HCCS_OK: return "HCCS_OK";
        case HCCS_ERR_INVALID_ARG: return "HCCS_ERR_INVALID_ARG";
        case HCCS_ERR_CONSTRAINT: return "HCCS_ERR_CONSTRAINT";
        case HCCS_ERR_NOT_UPLOADED: return "HCCS_ERR_NOT_UPLOADED";
        case HCCS_ERR_UNSUPPORTED: return "HCCS_ERR_UNSUPPORTED";
        case HCCS_ERR_CUDA: return "HCCS_ERR_CUDA";
        case HCCS_ERR_DEVICE_TIMEOUT: return "HCCS_ERR_DEVICE_TIMEOUT";
        case HCCS_ERR_DEVICE_INDEX: return "HCCS_ERR_DEVICE_INDEX";
    }
    return "HCCS_<unknown status>";
}

}  // extern "C"
