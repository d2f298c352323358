/*
 * hccs.h -- C ABI of libhccs: the inference step of the Head-Calibrated
 * Clipped-Linear Softmax (HCCS) on NVIDIA B200 (sm_100a).
 *
 * HCCS maps a row of int8 attention logits x to scaled integer probabilities
 * using only integer arithmetic (paper, Section III and Algorithm 1):
 *
 *   m       = max_j x_j                                   (Eq. 1)
 *   delta_j = min(m - x_j, Dmax_h)                        (Eq. 2)
 *   s_j     = B_h - S_h * delta_j            (>= 0)       (Eq. 3, Eq. 4)
 *   Z       = sum_j s_j                                   (Eq. 5)
 *   int16 output:  rho = floor(32767 / Z),      p_j = s_j * rho           (Eq. 6, 7)
 *   int8 output:   rho = floor(255 * 2^15 / Z), p_j = (s_j * rho) >> (15 + OUT_SHIFT)   (Eq. 8)
 *   leading-bit reciprocal (CLB): k = floor(log2 Z), rho = T' >> k        (Eq. 9)
 *
 * with one parameter triple theta_h = (B_h, S_h, Dmax_h) per attention head.
 *
 * Conventions for every entry point
 *   - Tensors are contiguous, row-major, innermost dimension last.
 *   - "device" pointers are CUDA device memory of the context's device, owned by
 *     the caller; "host" pointers are ordinary (preferably pinned) host memory.
 *   - Work is enqueued on `cuda_stream` (a cudaStream_t passed as void*, NULL =
 *     the default stream) and the call returns without synchronising, unless
 *     stated otherwise.
 *   - Errors are return codes only.  On any error nothing is launched.
 *   - A context is not thread-safe: one host call at a time per context (different contexts, also
 *     on the same device, are independent).  On the GPU, hccs_forward, hccs_forward_keylen,
 *     hccs_forward_host, hccs_attention_cached and hccs_attention_cross calls of one context only read the context's parameter
 *     table (hccs_cache_write, hccs_cache_write_axes, hccs_states_write and hccs_cache_read not even that) and may overlap each other freely
 *     (different streams, back to back on one stream).  Calls that rewrite device memory the context
 *     owns do so on their own `cuda_stream`: hccs_params_upload and hccs_params_upload_wide (the
 *     parameter table) and the hccs_attention_fused* calls (a small per-head multiplier table,
 *     rewritten only when the multipliers, the shift or the output scales differ from the previous
 *     fused call's).  Order such a call against other work of the same context that may still be
 *     running on another stream yourself (an event, or one stream per context).
 *   - There is no CPU implementation behind this interface.
 */
#ifndef HCCS_H
#define HCCS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hccs_ctx hccs_ctx_t;   /* opaque; owns the device parameter table and a status word */

/* theta_h of the paper's Section "Offline Calibration": fixed at inference. */
typedef struct {
    int32_t B;      /* B_h    > 0  : score of the row maximum                     */
    int32_t S;      /* S_h    >= 0 : slope per unit of clamped distance           */
    int32_t Dmax;   /* Dmax_h in [1,127] : clamp bound of the distance (Eq. 2)    */
} hccs_head_params_t;

typedef enum {
    HCCS_OK = 0,
    HCCS_ERR_INVALID_ARG    = 1,  /* NULL pointer, negative size, unknown flag, wrong H          */
    HCCS_ERR_CONSTRAINT     = 2,  /* theta outside the admissible region, or Lk > n_design       */
    HCCS_ERR_NOT_UPLOADED   = 3,  /* hccs_forward before hccs_params_upload                      */
    HCCS_ERR_UNSUPPORTED    = 4,  /* shape the kernels cannot take (documented per call)         */
    HCCS_ERR_CUDA           = 5,  /* a CUDA runtime call failed; see hccs_last_cuda_error        */
    HCCS_ERR_DEVICE_TIMEOUT = 6,  /* a bounded device-side wait gave up (hccs_device_status)     */
    HCCS_ERR_DEVICE_INDEX   = 7   /* a page, slot or length in device memory was out of range (hccs_device_status) */
} hccs_status_t;

/* flags of hccs_forward / hccs_attention_fused (bitwise OR) */
enum {
    HCCS_OUT_U8    = 0,   /* uint8 probabilities, T = 255 (int8 output path, Eq. 8)             */
    HCCS_OUT_U16   = 1,   /* uint16 probabilities, T = 32767 (Eq. 6, 7)                         */
    HCCS_RECIP_DIV = 0,   /* exact integer divide                                               */
    HCCS_RECIP_CLB = 2,   /* leading-bit reciprocal (Eq. 9); uint8 results saturate at 255      */
    HCCS_CAUSAL    = 4    /* key j of query i takes part iff j <= i + (Lk - Lq); others give 0  */
};

/* a further reciprocal, of hccs_attention_cached and hccs_attention_cross only: the scores are divided by their sum as real numbers */
enum { HCCS_RECIP_REAL = 8 };

/* element types of the cache entry points */
typedef enum {
    HCCS_I32  = 0,
    HCCS_F32  = 1,
    HCCS_BF16 = 2,
    HCCS_F16  = 3
} hccs_type_t;

/* Creates a context on CUDA device `device` (allocates a small parameter table lazily and a
 * 4-byte device status word).  *out receives the context.  Synchronous. */
hccs_status_t hccs_create(hccs_ctx_t **out, int device);

/* Frees the context's device memory.  The caller must have synchronised its streams. */
hccs_status_t hccs_destroy(hccs_ctx_t *ctx);

/*
 * Uploads the per-head parameter table (Section "Offline Calibration"; looked up per row by the
 * row's head, Section "Multi-tile scaling").
 *   params     host array of num_heads triples
 *   n_design   the row length n the table was calibrated for (1..32767)
 *   out_shift  OUT_SHIFT of the int8 output path (Eq. 8), 0..8; 0 unless you know better
 *   bad_head   may be NULL; receives the first offending head on HCCS_ERR_CONSTRAINT, else -1
 * Every item of the paper's Section "Integer Range Constraints" is checked on the host for
 * n = n_design:  Dmax <= 127;  S >= 0;  B - S*Dmax >= ceil(256/n);  n*B <= 32767 (hence
 * B <= 32767).  Two more bounds are this library's own additions, not the paper's: Dmax >= 1 (a
 * clamp bound of 0 would make every row uniform) and S <= 127 (the paper describes the score as a
 * single int8 multiply-accumulate, so S is kept an int8 operand).  On a violation nothing is
 * uploaded and the previous table stays in force.
 * The table is copied from an internal pinned staging buffer on `cuda_stream`; `params` may be
 * reused as soon as the call returns.  The first upload makes room for 256 heads; it, and one with more
 * heads than there is room for, allocates device memory and therefore synchronises the device.
 * Uploads do not belong into a stream capture.  Captured launches read the table that is in force when they
 * are replayed; one that is uploaded meanwhile has to have as many heads.  An upload that needs more room
 * moves the table: graphs captured before it must not be replayed any more.  Should that allocation
 * fail, the context has no table (HCCS_ERR_NOT_UPLOADED) until an upload succeeds.
 */
hccs_status_t hccs_params_upload(hccs_ctx_t *ctx, const hccs_head_params_t *params,
                                 int32_t num_heads, int32_t n_design, int32_t out_shift,
                                 int32_t *bad_head, void *cuda_stream);

/* The host-side admissibility check of hccs_params_upload on its own (no context, no CUDA call):
 * HCCS_OK, or HCCS_ERR_CONSTRAINT with *bad_head (may be NULL) = first offending head, or
 * HCCS_ERR_INVALID_ARG for a NULL table, num_heads < 1 or n_design outside 1..32767. */
hccs_status_t hccs_params_check(const hccs_head_params_t *params, int32_t num_heads,
                                int32_t n_design, int32_t *bad_head);

/*
 * HCCS over every row of a logit tensor (Algorithm 1 applied to B*H*Lq independent rows,
 * Section "Vectorization and Parallelism Across Rows").
 *   logits  device int8  [B, H, Lq, Lk]
 *   probs   device uint8 [B, H, Lq, Lk] (HCCS_OUT_U8) or uint16 (HCCS_OUT_U16); may equal
 *           `logits` for uint8 output (each row is read completely before it is written)
 *   H       must equal the uploaded num_heads; the head of flat row r is (r / Lq) mod H
 *   Lk      1..n_design (HCCS_ERR_CONSTRAINT beyond: the admissible band only narrows with n)
 * Rows shorter than n_design, and causal rows with few valid keys, are computed with the same
 * formulas in 32-bit integers (rho is not narrowed to int16).  Masked positions take no part in
 * the max or the sum and produce 0; a row without any valid key produces all zeros.
 * Any Lk and any pointer alignment is accepted; the fast kernels need Lk % 16 == 0 and
 * 16-byte-aligned pointers, everything else runs in a slower CUDA kernel.  Empty tensors
 * (B*H*Lq*Lk == 0) return HCCS_OK without a launch.  B*H*Lq must be below 2^31.
 */
hccs_status_t hccs_forward(hccs_ctx_t *ctx, const int8_t *logits, void *probs,
                           int32_t B, int32_t H, int32_t Lq, int32_t Lk,
                           uint32_t flags, void *cuda_stream);

/*
 * hccs_forward with a padding mask: key j of batch entry b takes part iff j < key_len[b] (and,
 * with HCCS_CAUSAL, iff the causal rule holds as well).  This is the mask of the paper's encoder
 * workloads, whose sequences are padded to 64 or 128 tokens (Section "Models and tasks"); the
 * paper itself does not define masking: masked keys are left out of the max (Eq. 1) and the sum
 * (Eq. 5) and produce 0, a row without valid keys produces zeros.
 *   key_len  device int32 [B]; values are clamped to [0, Lk]
 * Everything else as hccs_forward.
 */
hccs_status_t hccs_forward_keylen(hccs_ctx_t *ctx, const int8_t *logits, void *probs,
                                  const int32_t *key_len, int32_t B, int32_t H, int32_t Lq, int32_t Lk,
                                  uint32_t flags, void *cuda_stream);

/*
 * The same operation for HOST tensors: copies `logits_host` to `logits_staging`, runs
 * hccs_forward, copies the result back to `probs_host`, all on `cuda_stream`, in pieces so that
 * the two copy directions and the kernel overlap.  The caller provides both device staging
 * buffers (same sizes as the tensors; the library allocates nothing here).  Host buffers should
 * be pinned (cudaHostAlloc / torch pin_memory), otherwise the copies serialise.  The result is
 * complete once `cuda_stream` has been synchronised.
 */
hccs_status_t hccs_forward_host(hccs_ctx_t *ctx, const int8_t *logits_host, void *probs_host,
                                int8_t *logits_staging, void *probs_staging,
                                int32_t B, int32_t H, int32_t Lq, int32_t Lk,
                                uint32_t flags, void *cuda_stream);

/*
 * Fused integer attention (not in the paper, which only notes that the integer outputs stay
 * compatible with fixed-point attention pipelines): per (b, h)
 *   acc_ij = sum_c Q[i,c] * K[j,c]                         (int32)
 *   x_ij   = clamp((acc_ij * requant_mult[h] + 2^(requant_shift-1)) >> requant_shift, -128, 127)
 *   P_i.   = HCCS(x_i.) with theta_h, uint8 output         (Algorithm 1, Eq. 8)
 *   O[i,:] = sum_j P_ij * V[j,:]                           (int32)
 *   Q, K, V       device int8  [B, H, L, d]
 *   O             device int32 [B, H, L, d]
 *   requant_mult  HOST int32 [H], each in [0, 2^13) and below 2^(requant_shift-1); requant_shift in 1..31
 *   flags         HCCS_RECIP_CLB and HCCS_CAUSAL are honoured; HCCS_OUT_U16 is HCCS_ERR_UNSUPPORTED
 * Supported shapes: d == 64 or d == 128 with 1 <= L <= 1024 (the 128 x L probability panel stays in
 * one SM's shared memory; for d == 128 beyond 512 keys K and V stream through a ring of buffers
 * beside it); L <= n_design, pointers 16-byte aligned; anything else returns HCCS_ERR_UNSUPPORTED.
 * The logits and probabilities never leave the chip.
 */
hccs_status_t hccs_attention_fused(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *K,
                                   const int8_t *V, int32_t *O, const int32_t *requant_mult,
                                   int32_t requant_shift, int32_t B, int32_t H, int32_t L, int32_t d,
                                   uint32_t flags, void *cuda_stream);

/*
 * hccs_attention_fused with a key-padding mask: key_len is a DEVICE int32 [B] array; keys at and
 * beyond key_len[b] (clamped to 0..L) of batch entry b are padding: like causally masked keys they
 * take no part in the row maximum and the row sum and get probability 0, so O is the attention over
 * the first key_len[b] keys alone; a batch entry with key length 0 gets O = 0.  Key blocks that
 * hold padding only are not computed at all.  Combines with HCCS_CAUSAL.  Everything else as hccs_attention_fused.  (Masking is not in the paper, whose
 * encoder workloads are padded to a fixed length, Section "Models and tasks".)
 */
hccs_status_t hccs_attention_fused_keylen(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *K,
                                          const int8_t *V, int32_t *O, const int32_t *key_len,
                                          const int32_t *requant_mult, int32_t requant_shift,
                                          int32_t B, int32_t H, int32_t L, int32_t d,
                                          uint32_t flags, void *cuda_stream);

/*
 * hccs_attention_fused with a dequantised fp32 output: O[b,h,i,:] = float(int32 accumulator) *
 * out_scale[h] (HOST float [H]; e.g. the V quantisation step divided by 255).  The integer result
 * is exact; the two fp32 roundings keep the relative error below 2^-23.  O is device float
 * [B, H, L, d]; everything else as hccs_attention_fused.  (Not in the paper.)
 */
hccs_status_t hccs_attention_fused_f32(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *K,
                                       const int8_t *V, float *O, const float *out_scale,
                                       const int32_t *requant_mult, int32_t requant_shift,
                                       int32_t B, int32_t H, int32_t L, int32_t d,
                                       uint32_t flags, void *cuda_stream);

/*
 * hccs_attention_fused with an int8 output, for pipelines that stay in int8 after the attention:
 * O[b,h,i,c] = clamp((acc * out_mult[h] + 2^(out_shift-1)) >> out_shift, -128, 127), acc the int32
 * accumulator of P.V, i.e. the rounding rule of the logit requantisation applied to the output
 * (round half up, arithmetic shift, then clamp; exact: computed in 64 bits).
 *   O          device int8 [B, H, L, d]
 *   out_mult   HOST int32 [H], each in [0, 2^13);  out_shift in 1..31
 * Everything else as hccs_attention_fused.  (Not in the paper.)
 */
hccs_status_t hccs_attention_fused_i8(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *K,
                                      const int8_t *V, int8_t *O, const int32_t *out_mult, int32_t out_shift,
                                      const int32_t *requant_mult, int32_t requant_shift,
                                      int32_t B, int32_t H, int32_t L, int32_t d,
                                      uint32_t flags, void *cuda_stream);

/* A bounded grid of candidates for hccs_calibrate: D = D_lo, D_lo + D_step, ... <= D_hi (clipped to
 * 1..127), S likewise (clipped to 0..127), and for each (D, S) the values B = S*D + ceil(256/n),
 * + B_step, ... <= floor(32767/n): every candidate lies in the admissible band (Eq. 11). */
typedef struct {
    int32_t D_lo, D_hi, D_step;
    int32_t S_lo, S_hi, S_step;
    int32_t B_step;
} hccs_calib_grid_t;

/*
 * Offline per-head calibration (Section "Offline Calibration", Eq. 10): scans the grid and returns,
 * for each head, the theta that minimises the mean over the head's rows of
 * KL( softmax(alpha * x) || q ), q the int16-path HCCS row renormalised to sum one (the paper
 * recommends the int16 space; the renormalisation and the logit scale alpha are readings).
 *   logits   device int8 [B, H, Lq, Lk], the calibration rows; n_design = Lk
 *   best     HOST array of H triples (output);  best_kl  HOST double [H] (output, may be NULL)
 * Ties go to the smallest (Dmax, S, B).  Needs no context.  Offline tooling: allocates and frees
 * its work space (128 * B * H * Lq * 4 bytes plus small tables) and synchronises `cuda_stream`.
 * fp64 throughout.  HCCS_ERR_CONSTRAINT when the grid holds no admissible candidate.
 */
hccs_status_t hccs_calibrate(const int8_t *logits, int32_t B, int32_t H, int32_t Lq, int32_t Lk,
                             double alpha, const hccs_calib_grid_t *grid, hccs_head_params_t *best,
                             double *best_kl, void *cuda_stream);

/*
 * ---- Generation over an int8 key/value cache (not in the paper: its models are encoders) ----
 *
 * The cache is two pools of pages, int8 [num_pages, Hkv, page_size, d] each, one for keys and one for
 * values; page_size is a power of two from 16 to 65536, d is 64 or 128,
 * num_pages * Hkv is below 2^31.  A sequence is a row of a page
 * table: its token j lives in page table[j / page_size], at place j % page_size.  A slot is
 * page * page_size + place.  Codes stand for code * step with one step per head.  The pools, tables and
 * every workspace belong to the caller.  hccs_cache_write, hccs_cache_write_axes, hccs_states_write, hccs_cache_read and hccs_attention_cached do not
 * allocate, copy from pageable memory or synchronise, so they can be captured into a CUDA graph (host
 * arrays are taken by value).  hccs_params_upload_wide allocates and synchronises like hccs_params_upload:
 * it comes before a capture.  No upload that these calls can use moves the table that they read.
 * At most HCCS_MAX_CACHE_HEADS query heads and HCCS_MAX_CACHE_KEYS keys per sequence.
 */
#define HCCS_MAX_CACHE_HEADS 256
#define HCCS_MAX_CACHE_KEYS 131072
#define HCCS_MAX_ROT_DIM 128

/* Rotary positions: the pair i of a head, (a, b) = dims (i, i + rot_dim/2), or (2i, 2i+1) where
 * interleaved, becomes (a*c - b*s, b*c + a*s) with c = scale*cos(t), s = scale*sin(t) and
 * t = position * freq[i], one rounding to fp64.  Dims from rot_dim on are left as they are. */
typedef struct {
    int32_t rot_dim;                          /* even, 0..d */
    int32_t interleaved;                      /* 0: halves, 1: neighbours */
    double  scale;                            /* magnitude 2^-64 .. 2^64 */
    double  freq[HCCS_MAX_ROT_DIM / 2];       /* radians per position, finite */
} hccs_rope_t;

/* How frequencies f_i = base^(-2i/rot_dim) are changed for contexts longer than a model was trained on.
 *   NONE        as they are
 *   LINEAR      f / factor
 *   BASE        base * factor^(rot_dim / (rot_dim - 2)) in the place of base (rot_dim > 2)
 *   WAVELENGTH  with n = original_len * f / (2 pi), the turns over the original length:
 *               keep = clamp((n - low) / (high - low), 0, 1), f*keep + (f/factor)*(1 - keep)
 *   DIMENSION   the same mixture, keep falling linearly over the pair index from the pair that makes
 *               `high` turns (rounded down) to the one that makes `low` (rounded up), both kept within
 *               0 .. rot_dim - 1; scale = 0.1 ln(factor) + 1 (the other kinds: scale = 1)
 */
enum { HCCS_ROPE_NONE = 0, HCCS_ROPE_LINEAR = 1, HCCS_ROPE_BASE = 2, HCCS_ROPE_WAVELENGTH = 3, HCCS_ROPE_DIMENSION = 4 };
typedef struct {
    int32_t kind;
    double factor;                            /* >= 1 */
    double low, high;                         /* WAVELENGTH, DIMENSION: 0 < low < high */
    double original_len;                      /* WAVELENGTH, DIMENSION: > 0 */
} hccs_rope_scaling_t;

/* Fills *rope (host only, no CUDA call).  `scaling` may be NULL (NONE).  HCCS_ERR_INVALID_ARG for a NULL
 * rope, an odd rot_dim or one outside 2..HCCS_MAX_ROT_DIM, base <= 1, or a scaling outside its ranges. */
hccs_status_t hccs_rope_frequencies(hccs_rope_t *rope, int32_t rot_dim, int32_t interleaved, double base,
                                    const hccs_rope_scaling_t *scaling);

/*
 * Rotates and quantises new tokens: queries to q8, keys and values into the cache.
 *   q, k, v      device [T, Hq | Hkv, d] of `type` (HCCS_F32, HCCS_BF16 or HCCS_F16); head and dim are
 *                contiguous, tokens are q_stride, k_stride, v_stride ELEMENTS apart (views of one fused
 *                projection, for instance); 16-byte aligned, and so are the strides
 *                (HCCS_ERR_UNSUPPORTED otherwise).  q may be NULL (Hq is then ignored), or both k and v
 *   positions    device int32 [T], any values; may be NULL without rope
 *   slots        device int64 [T]: where the token's key and value go; a negative slot skips them (padding
 *                tokens); the others of one call must differ (where two are
 *                the same, the slot holds a mixture of both).  A slot at or beyond num_pages * page_size is
 *                skipped as well and reported (hccs_device_status).  May be NULL where k and v are
 *   rope         HOST, or NULL for none; applied to q and k
 *   *_step       HOST float [Hq], [Hkv], [Hkv], each in 2^-100 .. 2^100: the value of one code
 *   q8           device int8 [T, Hq, d];  k_pages, v_pages  the pools; 16-byte aligned
 * A code is clamp(round(y / step), -128, 127), the exact quotient rounded to nearest, ties to even: the
 * kernel works in fp32 and repeats exactly (rotated dims: in fp64) what lies next to a border, so the codes
 * are those of a computation in fp64.  NaN gives 0.  Nothing else in the pools is touched.
 */
hccs_status_t hccs_cache_write(hccs_ctx_t *ctx, const void *q, const void *k, const void *v, hccs_type_t type,
                               int64_t q_stride, int64_t k_stride, int64_t v_stride,
                               const int32_t *positions, const int64_t *slots, const hccs_rope_t *rope,
                               const float *q_step, const float *k_step, const float *v_step,
                               int8_t *q8, int8_t *k_pages, int8_t *v_pages,
                               int32_t T, int32_t Hq, int32_t Hkv, int32_t d,
                               int32_t num_pages, int32_t page_size, void *cuda_stream);

/* Rotary positions with several axes (time, rows and columns of a video, rows and columns of an image): pair i turns
 * by positions of axis[i] alone, t = position[axis[i]] * freq[i]; the rest as in hccs_rope_t. */
#define HCCS_MAX_AXES 4
typedef struct {
    hccs_rope_t rope;
    int32_t num_axes;                         /* 1..HCCS_MAX_AXES */
    uint8_t axis[HCCS_MAX_ROT_DIM / 2];       /* of each pair, below num_axes */
} hccs_rope_axes_t;

/* How the pairs are dealt out: the first pairs[0] of them to axis 0, the next pairs[1] to axis 1, and so on; or
 * one to each axis in turn, axes that have theirs being left out. */
enum { HCCS_AXES_SECTIONS = 0, HCCS_AXES_TURNS = 1 };

/* Fills *axes (host only, no CUDA call).  pairs[x] >= 0 is the number of pairs of axis x; they sum to rot_dim / 2.
 * Frequencies are those of hccs_rope_frequencies for rot_dim, or, with `restart`, each axis has those for its own
 * 2 * pairs[x] dims, from the fastest on.  HCCS_ERR_INVALID_ARG as there, for a NULL axes or pairs, num_axes outside
 * 1..HCCS_MAX_AXES, an order that is none, or pairs that do not sum up. */
hccs_status_t hccs_rope_axes(hccs_rope_axes_t *axes, int32_t rot_dim, int32_t interleaved, double base,
                             const hccs_rope_scaling_t *scaling, const int32_t *pairs, int32_t num_axes,
                             int32_t order, int32_t restart);

/*
 * hccs_cache_write with positions of several axes: that of token t on axis x is
 * positions[x*axis_stride + t*token_stride] (device int32, any values; strides in elements, of any sign).  `axes` is a
 * HOST pointer or NULL for no rotation.  All else as there.
 */
hccs_status_t hccs_cache_write_axes(hccs_ctx_t *ctx, const void *q, const void *k, const void *v, hccs_type_t type,
                                    int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                    const int32_t *positions, int64_t axis_stride, int64_t token_stride,
                                    const int64_t *slots, const hccs_rope_axes_t *axes,
                                    const float *q_step, const float *k_step, const float *v_step,
                                    int8_t *q8, int8_t *k_pages, int8_t *v_pages,
                                    int32_t T, int32_t Hq, int32_t Hkv, int32_t d,
                                    int32_t num_pages, int32_t page_size, void *cuda_stream);

/*
 * The same into dense tensors, for states that are no cache: an encoder's own (hccs_attention_fused reads
 * [B, H, L, d]) or those that a decoder looks at (hccs_attention_cross reads [T, Hkv, d]).
 *   q8, k8, v8   device int8 [T/L, Hq | Hkv, L, d]: token t is number t % L of entry t / L.  L = 1 makes it [T, Hq | Hkv, d].
 *                L in 1..T divides T (HCCS_ERR_INVALID_ARG otherwise).  16-byte aligned
 * q may be NULL (with q8 and q_step; Hq is then ignored), or both k and v.  Codes, types, strides, positions and steps as in
 * hccs_cache_write_axes.
 */
hccs_status_t hccs_states_write(hccs_ctx_t *ctx, const void *q, const void *k, const void *v, hccs_type_t type,
                                int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                const int32_t *positions, int64_t axis_stride, int64_t token_stride,
                                const hccs_rope_axes_t *axes,
                                const float *q_step, const float *k_step, const float *v_step,
                                int8_t *q8, int8_t *k8, int8_t *v8,
                                int32_t T, int32_t L, int32_t Hq, int32_t Hkv, int32_t d, void *cuda_stream);

/*
 * Reads sequences back: token j of sequence b goes to row out_start[b] + j of the outputs.
 *   page_table   device int32 [B, max_pages]; may be NULL where max_pages is 0
 *   out_start    device int32 [B+1], not falling; sequence b has out_start[b+1] - out_start[b] tokens, at
 *                most max_len (host) and max_pages * page_size of which are read; more is reported, and so
 *                is a page outside 0..num_pages-1, whose rows become zeros
 *   k_out, v_out device [rows, Hkv, d] of `type`; rows (host) is the size of the outputs: sequences that
 *                reach beyond it are cut there and reported.  Rows no sequence has are left as they are.
 *                16-byte aligned.  Either may be NULL
 * Values are code * step in fp32, rounded to `type`.
 */
hccs_status_t hccs_cache_read(hccs_ctx_t *ctx, const int8_t *k_pages, const int8_t *v_pages,
                              const int32_t *page_table, const int32_t *out_start,
                              const float *k_step, const float *v_step, void *k_out, void *v_out, hccs_type_t type,
                              int32_t B, int32_t max_pages, int32_t max_len, int32_t rows, int32_t Hkv, int32_t d,
                              int32_t num_pages, int32_t page_size, void *cuda_stream);

/*
 * hccs_params_upload for caches longer than the paper's int16 row sums allow (n*B <= 32767 leaves a table
 * of constants at 16384 keys): Dmax in 1..127, S in 0..127, 1 <= B <= 32767, B - S*Dmax >= 0, n_design in
 * 1..HCCS_MAX_CACHE_KEYS.  Such a table serves hccs_attention_cached and hccs_attention_cross with HCCS_RECIP_REAL alone; the other
 * calls return HCCS_ERR_CONSTRAINT until hccs_params_upload puts an ordinary table in its place.
 */
hccs_status_t hccs_params_upload_wide(hccs_ctx_t *ctx, const hccs_head_params_t *params, int32_t num_heads,
                                      int32_t n_design, int32_t *bad_head, void *cuda_stream);

/*
 * HCCS attention of new tokens over the cache, which already holds their keys and values.  Sequence b has
 * nq = q_start[b+1] - q_start[b] queries, the last nq of its kv_len[b] keys being their own.  For query i of
 * head h and the keys j it sees, kv head h / (Hq/Hkv):
 *   acc = sum_c Q[i,c] K[j,c];  x = clamp((acc*M_h + 2^(shift-1)) >> shift, -128, 127)
 *   s_j = B_h - S_h * min(max x - x_j, Dmax_h);  Z = sum s_j                               (Eq. 1 to 5)
 *   HCCS_RECIP_DIV, HCCS_RECIP_CLB   O = rho * sum s_j V[j,:], rho of the int16 path       (Eq. 6, 7, 9)
 *   HCCS_RECIP_REAL                  O = (sum s_j V[j,:] / Z) * out_scale[h]
 * The sums are exact integers whatever the split over the GPU, so results do not depend on it.
 * Which keys: all before the new ones; of the new ones those at or before the query itself, or, with
 * tree_mask, those whose bit is set: bit j % 32 of word j / 32 of row i for the j-th new key of the
 * sequence (a tree of drafted tokens: itself and its ancestors).  A query that sees no key gives zeros.
 *   Q            device int8 [T, Hq, d], 16-byte aligned
 *   page_table   device int32 [B, max_pages] (may be NULL where max_pages is 0);  q_start  device int32 [B+1], not falling;  kv_len  device int32 [B]
 *   tree_mask    device int32 [T, tree_words], or NULL
 *   requant_mult HOST int32 [Hq], each in [0, 2^13) and below 2^(shift-1) (HCCS_ERR_UNSUPPORTED beyond);
 *                requant_shift in 1..24
 *   out_scale    HOST float [Hq]; NULL for HCCS_I32 output, whose O is the exact integer
 *   O            device [T, Hq, d] of out_type; float types hold the fp32 product with out_scale[h], rounded
 *                once more to the type; HCCS_I32 goes with DIV and CLB only.  16-byte aligned
 *   max_q, max_kv (host)  bounds of the lengths of this call, which choose kernel and grid for all its
 *                sequences (chunks and single tokens are faster in calls of their own): queries beyond
 *                max_q are not computed (nor are their keys seen by a tree), and keys beyond max_kv are not seen, both reported.  max_kv beyond
 *                n_design is HCCS_ERR_CONSTRAINT, beyond HCCS_MAX_CACHE_KEYS HCCS_ERR_UNSUPPORTED
 *   flags        one HCCS_RECIP_*; nothing else
 * kv_len outside 0 .. max_pages * page_size is cut and reported; a page outside 0..num_pages-1 is reported
 * and its keys are not seen; q_start is cut to 0..T.  Rows behind the last sequence are left as they are.
 */
hccs_status_t hccs_attention_cached(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *k_pages, const int8_t *v_pages,
                                    const int32_t *page_table, const int32_t *q_start, const int32_t *kv_len,
                                    const int32_t *tree_mask, int32_t tree_words,
                                    const int32_t *requant_mult, int32_t requant_shift, const float *out_scale,
                                    void *O, hccs_type_t out_type,
                                    int32_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t d, int32_t max_pages,
                                    int32_t num_pages, int32_t page_size, int32_t max_q, int32_t max_kv,
                                    uint32_t flags, void *cuda_stream);

/*
 * HCCS attention of queries to states of another length (cross attention: an encoder's states, an image's, a
 * video's).  Sequence b has the queries q_start[b] .. q_start[b+1] - 1 and the keys k_start[b] .. k_start[b] + k_len[b] - 1
 * (sequences may share states, in whole or in part).  A query sees all keys of its sequence, or with key_range those
 * numbered key_range[t][0] .. key_range[t][1] - 1 of them (cut to the sequence's; the image that a token follows, for
 * instance).  Logits, scores, normalisation and outputs as in hccs_attention_cached; a query that sees no key gives
 * zeros.  Does not allocate or synchronise, and can be captured.
 *   Q            device int8 [T, Hq, d], 16-byte aligned
 *   K, V         device int8 [S, Hkv, d]; heads and dims are contiguous, keys are k_stride, v_stride BYTES apart: multiples of 16,
 *                Hkv*d or more, below 2^36 (halves of one tensor, for instance); 16-byte aligned.  May be NULL where S is 0
 *   q_start      device int32 [B+1], not falling;  k_start, k_len  device int32 [B]
 *   key_range    device int32 [T, 2], 8-byte aligned, or NULL
 *   requant_mult, requant_shift, out_scale, O, out_type, flags   as in hccs_attention_cached
 *   max_q, max_kv (host)  bounds of the lengths of this call, which choose kernel and grid: queries beyond max_q are not
 *                computed and keys beyond max_kv are not seen, both reported.  max_kv beyond n_design is
 *                HCCS_ERR_CONSTRAINT, beyond HCCS_MAX_CACHE_KEYS HCCS_ERR_UNSUPPORTED
 * Keys from S on are not seen and reported (bit 4 of the status word); where k_start is not in 0..S none of the sequence's keys is seen, which is
 * reported unless k_len is 0.  q_start is cut to 0..T.  Rows no sequence has are left as they are.
 */
hccs_status_t hccs_attention_cross(hccs_ctx_t *ctx, const int8_t *Q, const int8_t *K, const int8_t *V,
                                   int64_t k_stride, int64_t v_stride, const int32_t *q_start,
                                   const int32_t *k_start, const int32_t *k_len, const int32_t *key_range,
                                   const int32_t *requant_mult, int32_t requant_shift, const float *out_scale,
                                   void *O, hccs_type_t out_type,
                                   int32_t T, int32_t S, int32_t B, int32_t Hq, int32_t Hkv, int32_t d,
                                   int32_t max_q, int32_t max_kv, uint32_t flags, void *cuda_stream);

/* Reads (and clears) the device status word: 0 = no kernel gave up a bounded wait or met an index out of
 * range.  Synchronises `cuda_stream`.  Returns HCCS_ERR_DEVICE_TIMEOUT when a wait was given up (bits 0
 * and 1), else HCCS_ERR_DEVICE_INDEX when the word was non-zero (bit 2: slot, bit 3: page, bit 4: length);
 * *word (may be NULL) receives it.  A launch that gave up a wait leaves its output incomplete: some rows as
 * they were, some from part of their sums; none of it is to be used. */
hccs_status_t hccs_device_status(hccs_ctx_t *ctx, uint32_t *word, void *cuda_stream);

/*
 * Self-test of the device-side wait limits.  (The paper has no counterpart.)  Every wait of the
 * TMA-staged kernels (on a bulk copy, on a tensor-core commit) gives up after a limit of SM clock
 * cycles -- about a second in production -- sets a bit of the status word and lets the kernel return
 * instead of hanging the GPU.  This call runs that give-up path on purpose and harmlessly: one small
 * CTA waits, through the same wait routines, on a barrier that nothing will ever complete, with the
 * limit given here.
 *   mode          0: the wait of the long-row kernel (sets bit 0 of the status word);
 *                 1: the abort-flag wait of the fused kernel (sets bit 1; a second thread gives up
 *                    because it sees the flag, not because its own, longer limit ran out)
 *   limit_cycles  1 .. 10 000 000
 * Afterwards hccs_device_status returns HCCS_ERR_DEVICE_TIMEOUT once and clears the word.
 */
hccs_status_t hccs_debug_wait_timeout(hccs_ctx_t *ctx, int32_t mode, int64_t limit_cycles, void *cuda_stream);

/* The cudaError_t of the last failing CUDA call made through this context (0 = none). */
int32_t hccs_last_cuda_error(const hccs_ctx_t *ctx);

/* Static, human-readable name of a status code. */
const char *hccs_status_string(hccs_status_t status);

/* Number of kernels launched through this context since creation (for launch accounting). */
uint64_t hccs_launch_count(const hccs_ctx_t *ctx);

/*
 * hccs_forward for callers that are not allowed to allocate device memory.  (The paper has no
 * counterpart to this entry point; it exists for deployment reasons only.)
 *
 * Who needs it: code that runs where cudaMalloc is off limits -- inside a memory pool's or a
 * framework's allocator callback, in a process whose device memory was handed out in full at
 * start-up (a serving engine that pre-claims the whole GPU), or in a latency-critical loop where
 * an allocation (which may synchronise the whole device) cannot be tolerated.  Such a caller
 * cannot create an hccs_ctx_t, because the context allocates its parameter table.
 *
 * What it does: the same result as hccs_forward, computed by the shared-memory-staged
 * one-CTA-per-row kernel, with all of the library's working memory (the parameter table and the
 * status word that device-side waits report to) in one fixed 4.25 KB array that is part of the
 * loaded library image on every GPU.  No context, no cudaMalloc/cudaFree, no allocating library
 * call, no host-to-device copy; the tensors are the caller's.
 *   params, num_heads, n_design, out_shift   HOST table, checked exactly as hccs_params_upload
 *        does; it travels to the GPU as a kernel argument, so it may be reused or freed as soon as
 *        the call returns.  num_heads above 256 does not fit the fixed array: HCCS_ERR_UNSUPPORTED
 *   logits, probs, B, H, Lq, Lk, flags       as hccs_forward, on the CURRENT device; this entry
 *        point needs Lk % 16 == 0 and 16-byte aligned pointers (else HCCS_ERR_UNSUPPORTED)
 *   timed_out   NULL: two kernels are enqueued on `cuda_stream` (one that fills the array, then the
 *        row kernel) and the call returns without waiting for them.  Non-NULL (host): the call
 *        also synchronises `cuda_stream` and stores the status word there; non-zero returns
 *        HCCS_ERR_DEVICE_TIMEOUT as well.
 * The first call on each device looks up the device address of the fixed array
 * (cudaGetSymbolAddress); make that first call before any stream capture begins.  All calls on a
 * device share the array and it keeps the previous call's contents: each call rewrites the table
 * and clears the status word on `cuda_stream` before its row kernel.  Two calls whose work
 * overlaps on the GPU (different streams, no dependency between them) therefore race on it --
 * serialise them.
 */
hccs_status_t hccs_forward_static_scratch(const hccs_head_params_t *params, int32_t num_heads,
                                          int32_t n_design, int32_t out_shift,
                                          const int8_t *logits, void *probs,
                                          int32_t B, int32_t H, int32_t Lq, int32_t Lk,
                                          uint32_t flags, uint32_t *timed_out, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* HCCS_H */
