/*
 * libsolo — the SOLO low-bit AdamW optimizer step for AMD MI355X (gfx950).
 *
 * One call performs, in a single pass over HBM, the whole quantized-state
 * update of "Pushing the Limits of Low-Bit Optimizers: A Focus on EMA
 * Dynamics" (SOLO) for one flat buffer of parameters:
 *
 *   dequantize both moments  ->  EMA update  ->  AdamW parameter update
 *   ->  per-block scale / quantile / log base  ->  re-quantize  ->  re-pack
 *
 *   1st moment  m : b_m-bit signed linear codes, or the signed dynamic-
 *                   exponent codes of the paper's own variants (App. A, Eq. 1)
 *   2nd moment  v : b_v-bit unsigned logarithmic codes, levels alpha^k,
 *                   log-domain stochastic rounding, per-block base alpha
 *                   from the p-quantile                     (Sec. 3.2.2)
 *   block-wise quantization, one scale per block            (Sec. 3.4)
 *
 * Conventions for every entry point
 *   - Pointers named param / grad / *_codes / *_scale / v_base are DEVICE
 *     pointers; `cfg` is a HOST pointer, read during the call only.
 *   - All buffers are owned by the caller.  The library never allocates,
 *     frees or keeps a pointer, and never synchronises: work is enqueued on
 *     `stream` (a hipStream_t passed as void*; NULL = the default stream) and
 *     the call returns at once.
 *   - Return value: SOLO_OK (0) or a negative error code; nothing is enqueued
 *     when an error is returned.  n == 0 is a successful no-op.
 *   - The library uses the HIP runtime it finds in the process.  A process
 *     that brings one of its own (a PyTorch wheel does) loads that first, so
 *     that the streams it passes and the launches belong to the same runtime.
 *
 * State layout for n elements, block size B, nb = ceil(n / B) blocks
 *   m_codes  uint32[solo_code_words(n, bits_m)]   element i lives in word
 *   v_codes  uint32[solo_code_words(n, bits_v)]   i / c at bit bits*(i mod c),
 *            c = 16 (2-bit), 10 (3-bit, two pad bits), 8 (4-bit); unused bits 0
 *   m_scale  float[nb]   Delta_m = max |m| of the block
 *   v_scale  float[nb]   Delta_v = max v of the block
 *   v_base   float[nb]   alpha of the block, in (0, 1]
 *   A 1st-moment code c in [0, 2L], L = 2^(bits_m-1)-1, stands for the level
 *   (c - L) / L; with SOLO_FLAG_M_DYNAMIC_EXPONENT a code in [0, 2L+1] indexes the
 *   increasing signed dynamic-exponent levels (code L is 0, code 2L+1 is +1, there
 *   is no level -1).  A 2nd-moment code q in [0, 2^bits_v - 1] stands for alpha^q.
 *   param, grad and the code buffers must be 16-byte aligned, the scale
 *   buffers 4-byte aligned.
 *   The unused bits of the code words (the two pad bits of every 3-bit word, the
 *   fields behind element n-1 of the last word) must be zero on entry to a step;
 *   solo_state_init and every step leave them zero.
 */
#ifndef SOLO_H
#define SOLO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    SOLO_OK = 0,
    SOLO_E_INVALID = -1,      /* null/misaligned pointer, value out of range   */
    SOLO_E_UNSUPPORTED = -2,  /* legal value this build has no kernel for      */
    SOLO_E_HIP = -3           /* the HIP runtime refused the launch            */
};

enum { SOLO_GRAD_FP32 = 0, SOLO_GRAD_BF16 = 1 };
enum { SOLO_FP32 = 0, SOLO_BF16 = 1 };     /* element types of the operators around the step */

/* flags */
#define SOLO_FLAG_STOCHASTIC 1u   /* xi ~ U(-0.5, 0.5); clear = xi = 0 */
#define SOLO_FLAG_M_DYNAMIC_EXPONENT 2u /* 1st moment uses the signed dynamic-exponent levels of
                                          App. A (the paper's own 4/2-bit and 2-bit AdamW, Sec. 3.4)
                                          instead of the signed linear ones */

#define SOLO_FLAG_ADABELIEF 4u     /* AdaBelief instead of Adam (Sec. 4.2, "Generalizability"): the
                                     unsigned EMA follows (g - m^)^2, m^ the fresh 1st moment, and
                                     eps is added to that EMA itself at every step */
#define SOLO_FLAG_COUPLED_DECAY 8u /* plain Adam: weight_decay * p is added to the gradient before
                                     both EMAs and the parameter is not decayed separately */

typedef struct solo_config {
    uint32_t bits_m;       /* 2, 3 or 4: signed linear or dynamic-exponent codes (App. A) */
    uint32_t bits_v;       /* 2, 3 or 4: logarithmic codes (Sec. 3.2.2)                */
    uint32_t block_size;   /* 64, 128 or 2048 elements per block (Sec. 3.4 uses 128;   */
                           /* 2048 is the large-block setting of Sec. 4.2)             */
    uint32_t grad_dtype;   /* SOLO_GRAD_FP32 or SOLO_GRAD_BF16                         */
    float lr;              /* learning rate                                            */
    float beta1;           /* momentum of the signed EMA, in [0,1); use the precision- */
                           /* specific value of Sec. 3.3 (solo_beta1_default)          */
    float beta2;           /* momentum of the unsigned EMA, in [0,1)                   */
    float eps;             /* added to the bias-corrected root, >= 0                   */
    float weight_decay;    /* decoupled decay                                          */
    float quantile_p;      /* p of the quantile that sets alpha, in [0,1); paper: 0.1  */
    uint32_t flags;        /* SOLO_FLAG_*                                              */
    uint32_t reserved;     /* must be 0                                                */
    uint64_t seed;         /* key of the xi stream                                     */
    uint64_t index_offset; /* global index of element 0 of this buffer; multiple of 8. */
                           /* xi is a function of (seed, step, index_offset + i), so a */
                           /* shard of a larger buffer reproduces the unsharded result */
} solo_config;

/* Number of uint32 words that hold n codes of the given width (2, 3 or 4);
 * 0 for an unsupported width.  Sec. 3.4 packs several low-bit codes into one
 * storage element (two 4-bit or four 2-bit codes per byte; a word of this library
 * is four such bytes, little-endian); 3-bit codes, which Sec. 3.4 leaves out for
 * lack of a packing, go ten to a word with two unused bits. */
size_t solo_code_words(uint64_t n, uint32_t bits);

/* Number of quantization blocks of n elements, ceil(n / block_size) (block-wise
 * quantization, Sec. 3.4: every block of block_size consecutive elements has its
 * own scale; a shorter last block is a block of its own); 0 if block_size is 0. */
size_t solo_num_blocks(uint64_t n, uint32_t block_size);

/* Bytes of optimizer state for n elements: both code buffers plus three
 * floats per block (Sec. 4.2: the scale costs 32/B bits per element and the
 * buffered log base doubles that). 0 if cfg is invalid. */
size_t solo_state_bytes(uint64_t n, const solo_config *cfg);

/* Default momentum of the signed EMA for a code width (Sec. 3.4): 4-bit 0.8
 * (fine-tuning) / 0.3 (from scratch), 2-bit 0.5 / 0.1; 3-bit, which the paper
 * does not list, takes 0.6 / 0.2 by the same rule.  Other widths: 0.9. */
float solo_beta1_default(uint32_t bits_m, int from_scratch);

/* Largest beta' with beta'/(1-beta') * r_median(b') <= beta/(1-beta) * r_median(b)
 * (Sec. 3.3, Eq. "beta-prime"), given the two median radii. */
float solo_beta1_bound(float beta, float r_median_b, float r_median_bprime);

/* Write the zero state m = v = 0 of a fresh optimizer.  The paper does not say how
 * the zero state is encoded; this library's reading: every 1st-moment code = L (the
 * code of level 0 of either codebook, not a zero byte), every 2nd-moment code = 0,
 * Delta_m = Delta_v = 0, alpha = 1 (a block whose maximum is zero has no levels to
 * tell apart; the step treats Delta = 0 as "all elements are exactly 0").  Unused
 * bits of the code words are written as zeros. */
int solo_state_init(uint32_t *m_codes, float *m_scale,
                    uint32_t *v_codes, float *v_scale, float *v_base,
                    uint64_t n, const solo_config *cfg, void *stream);

/* One optimizer step (Sec. 3.1 Eqs. 2-4 for both moments, Sec. 3.2.2 for the
 * 2nd-moment quantizer, Sec. 3.4 for blocks), in place:
 *   param   float[n], read and written
 *   grad    float[n] or bf16[n] per cfg->grad_dtype, read only
 *   states  as laid out above, read and written
 *   step    1-based count of this update (bias correction and xi stream)
 * Gradients must be finite and so must their squares in binary32 (|g| < 1.8e19);
 * the result for other inputs is unspecified for the blocks that hold them and
 * unchanged for every other block (no call hangs or faults: every loop of the
 * kernels is bounded and every table index is clamped).  A block whose new
 * maximum is below 2^-100 is stored as a zero block.
 * Performance note: on MI355X the 288 GiB of HBM behave as three regions of 96 GiB of physical
 * memory (a third of every stack).  The step of a large buffer is about 2 % slower when the two
 * code buffers lie in the same region as `param` (the one large stream that is both read and
 * written) than when they lie in another one; where `grad` and the three scale buffers lie does
 * not matter.  A process that starts on an idle GPU receives physical memory in allocation order:
 * a long-lived optimizer does well to allocate its state so that it does not end up in the
 * third of HBM that holds the parameters (python -m paper_2505_00347_amd.hbm_regions measures
 * the effect; state_region of the Python binding does it, and bench.py allocates that way). */
int solo_adamw_step(float *param, const void *grad,
                    uint32_t *m_codes, float *m_scale,
                    uint32_t *v_codes, float *v_scale, float *v_base,
                    uint64_t n, uint64_t step,
                    const solo_config *cfg, void *stream);

/* The same step with the two extras of a mixed-precision training loop (Sec. 1: 16-bit weights
 * and gradients beside the 32-bit parameters) fused into the one pass:
 *   param_bf16  bf16[n] DEVICE, 16-byte aligned, or NULL: receives every new parameter rounded
 *               to bfloat16 (nearest, ties to even), so the 16-bit weights of the next forward
 *               pass need no second sweep over the parameters
 *   grad_scale  DEVICE pointer to one float, or NULL (= 1): every gradient is multiplied by it,
 *               rounded to binary32, before anything else (reciprocal of the loss scale, a
 *               clipping coefficient computed on the GPU); must be finite
 * All other arguments, the return value and the state are those of solo_adamw_step, which is
 * this call with both pointers NULL. */
int solo_adamw_step_mp(float *param, uint16_t *param_bf16, const void *grad, const float *grad_scale,
                       uint32_t *m_codes, float *m_scale,
                       uint32_t *v_codes, float *v_scale, float *v_base,
                       uint64_t n, uint64_t step,
                       const solo_config *cfg, void *stream);

/* ---- many tensors in one launch ------------------------------------------------------------
 * A model is a set of tensors, each quantized on its own (Sec. 3.4: block-wise, small tensors
 * included), and most of them are small: one launch per tensor is bound by launch latency.
 * solo_adamw_step_multi runs the step of the same configuration over all tensors of a table in
 * one launch.  The table is built on the host from `count` descriptors of DEVICE buffers and
 * copied to device memory by the caller (who owns it, like every other buffer):
 *
 *   units = solo_multi_units(tensors, count, cfg);
 *   bytes = solo_multi_table_bytes(count, units);
 *   solo_multi_table_build(tensors, count, cfg, host_buffer, bytes, &table_flags);   // host -> host
 *   copy host_buffer to a 16-byte aligned device buffer `table`
 *   solo_adamw_step_multi(table, count, units, table_flags, grad_scale, step, cfg, stream);   // every step
 *
 * A tensor's buffers are laid out and aligned like those of solo_adamw_step (state sized by
 * solo_code_words / solo_num_blocks for its own n); param_bf16 may be NULL per tensor; tensors
 * with n == 0 are allowed.  Tensor k uses the xi stream of the flat step at
 * index_offset = cfg->index_offset + sum over the tensors before it of n rounded up to a multiple
 * of 2560, so its result is that of solo_adamw_step_mp on the tensor alone with that
 * index_offset.  The table depends on the pointers, the sizes, cfg's state format (code widths,
 * block size, codebook), grad_dtype and index_offset; it need not be rebuilt when only scalars of
 * cfg or the step change. */
typedef struct solo_tensor {
    float *param;          /* fp32[n], read and written                      */
    void *param_bf16;      /* bf16[n] or NULL: bf16 copy of the new parameters */
    const void *grad;      /* fp32[n] or bf16[n] per cfg->grad_dtype          */
    uint32_t *m_codes;
    float *m_scale;
    uint32_t *v_codes;
    float *v_scale;
    float *v_base;
    uint64_t n;            /* elements                                       */
} solo_tensor;

/* Number of work units the tensors are cut into for cfg's state format and gradient type: one per
 * full 5120 elements (2560 for the wider formats) plus one per 512 elements of a tensor's ragged end;
 * with fp32 gradients and the linear codebook one per 2560 elements, a tensor's shorter end
 * included.  0 if cfg is invalid.  At most 2^24 tensors per table.  With blocks of 2048 elements
 * a unit is one block. */
uint64_t solo_multi_units(const solo_tensor *tensors, uint32_t count, const solo_config *cfg);

/* Bytes of the table for `count` tensors and `units` units. */
size_t solo_multi_table_bytes(uint32_t count, uint64_t units);

/* Fill `table_host` (HOST memory, table_bytes >= solo_multi_table_bytes) from `tensors` (HOST
 * array of descriptors holding DEVICE pointers) and set *table_flags (SOLO_TABLE_*), which
 * solo_adamw_step_multi takes back.  Checks every pointer's alignment. */
#define SOLO_TABLE_BF16_COPY 1u   /* some tensor has a bf16 copy to write */
#define SOLO_TABLE_SHORT_BLOCK 2u /* blocks of 2048: some tensor ends in a shorter block (for the caller; the
                                     launch does not depend on it) */
#define SOLO_TABLE_PIECES_SHIFT 2 /* blocks of 64 and 128: table_flags >> 2 is the number of pieces of the
                                     tensors (one wavefront each), which sizes the launch; 0 where the
                                     units do, which is right for every table but larger than need be */
int solo_multi_table_build(const solo_tensor *tensors, uint32_t count, const solo_config *cfg,
                           void *table_host, size_t table_bytes, uint32_t *table_flags);

/* One optimizer step over every tensor of `table_device` (DEVICE copy of a built table, 16-byte
 * aligned; `count`, `units` and `table_flags` as at build time).  grad_scale as in solo_adamw_step_mp. */
int solo_adamw_step_multi(const void *table_device, uint32_t count, uint64_t units,
                          uint32_t table_flags, const float *grad_scale, uint64_t step,
                          const solo_config *cfg, void *stream);

/* ==== around the step ============================================================================
 * The operators of a training loop that lie next to the optimizer step: the gradients' global norm
 * and clipping, the embedding and its gradient, the log probabilities of given tokens and their
 * gradient, layer norm and its gradient, distillation from a teacher's alternatives and its
 * gradient, sampling.  The conventions of the step hold: device pointers owned by the caller, a host struct
 * read during the call, work enqueued on `stream`, no allocation, no synchronisation, SOLO_OK or a
 * negative code with nothing enqueued (but SOLO_E_HIP of a call of several launches: those before the
 * one that the runtime refused are enqueued, and the outputs are then not specified).  A workspace needs no initialisation, holds nothing between
 * calls and serves one call at a time (calls on one stream follow each other).  Tensors need the
 * alignment of their elements only.  Every call gives the same bits for the same inputs: no sum of
 * floating-point numbers is made by atomic additions.  All calls can be captured into a HIP graph. */

/* ---- global norm and clipping ---------------------------------------------------------------
 * Over the tensors g_k of a table, with u = *unscale (the reciprocal of a loss scale; NULL: 1):
 *
 *   N_k = |u| sqrt(sum g_k^2)     N = sqrt(sum N_k^2)     c = u * (N > max_norm ? max_norm / N : 1)
 *
 * *norm = N, *grad_scale = c (what solo_adamw_step_mp and _multi take as grad_scale), tensor_norm[k] =
 * N_k.  Squares and sums are binary64, so N is that of the exact sum to about one rounding, for every
 * finite gradient.  Where N is not finite (a gradient is not, or N exceeds binary32), c is 0.
 * solo_grad_clip also writes clipped_k = c * g_k, the binary32 product rounded to the gradient's type;
 * where c is 0, zeros, whatever the gradient holds.  The table is built like that of the multi-tensor step:
 *
 *   units = solo_norm_units(grads, count);
 *   solo_norm_table_build(grads, count, host_buffer, solo_norm_table_bytes(count, units));
 *   copy host_buffer to a 16-byte aligned device buffer `table`
 *   solo_grad_norm(table, count, units, unscale, max_norm, norm, grad_scale, tensor_norm, workspace, stream);
 */
typedef struct solo_grad {
    const void *grad;      /* fp32[n] or bf16[n], DEVICE                                        */
    void *clipped;         /* the same type: where solo_grad_clip writes; may be grad itself, or
                              NULL (not written); must not overlap another tensor               */
    uint64_t n;            /* elements, up to 2^40; 0 is allowed                                */
    uint32_t dtype;        /* SOLO_FP32 or SOLO_BF16                                            */
    uint32_t reserved;     /* must be 0                                                         */
} solo_grad;

/* Work units of the table: 0 if grads is NULL, all tensors are empty or one is too long. */
uint64_t solo_norm_units(const solo_grad *grads, uint32_t count);
size_t solo_norm_table_bytes(uint32_t count, uint64_t units);
size_t solo_norm_workspace_bytes(uint64_t units);
int solo_norm_table_build(const solo_grad *grads, uint32_t count, void *table_host, size_t table_bytes);

/* max_norm >= 0 (infinity: no clipping); workspace: solo_norm_workspace_bytes, 16-byte aligned;
 * tensor_norm: float[count] or NULL.  norm, grad_scale: one float each. */
int solo_grad_norm(const void *table_device, uint32_t count, uint64_t units, const float *unscale, float max_norm,
                   float *norm, float *grad_scale, float *tensor_norm, void *workspace, void *stream);
int solo_grad_clip(const void *table_device, uint32_t count, uint64_t units, const float *unscale, float max_norm,
                   float *norm, float *grad_scale, float *tensor_norm, void *workspace, void *stream);

/* ---- embedding --------------------------------------------------------------------------------
 *   rows[i] = scale * table[t_i]            grad_table[v] = scale * sum over i with t_i = v of grad_rows[i]
 *
 * A token outside [0, vocab) (padding) gives a row of zeros and has no gradient.  Sums are binary32 in
 * an order that the tokens alone determine; one rounding to bf16 at the end.  Every row of grad_table is
 * written, those without a token with zeros; with SOLO_EMBEDDING_ACCUMULATE the sums are added to what
 * is there (a table that is also the head of the model, a second micro-batch) and other rows are not
 * touched. */
#define SOLO_EMBEDDING_ACCUMULATE 1u
typedef struct solo_embedding_shape {
    uint64_t vocab, dim;        /* rows and columns of the table; below 2^30 and 2^24            */
    uint64_t tokens;            /* below 2^28                                                    */
    uint64_t table_stride;      /* elements from row to row, >= dim, below 2^31                  */
    uint64_t rows_stride;       /* the same of rows / grad_rows                                  */
    uint32_t table_dtype;       /* of table / grad_table                                         */
    uint32_t rows_dtype;        /* of rows / grad_rows                                           */
    uint32_t token_bits;        /* 32 or 64: signed whole numbers                                */
    uint32_t flags;             /* 0 or SOLO_EMBEDDING_ACCUMULATE (gradient only)                */
    float scale;                /* finite                                                        */
    uint32_t reserved;          /* must be 0                                                     */
} solo_embedding_shape;

int solo_embedding(const void *table, const void *tokens, void *rows, const solo_embedding_shape *shape, void *stream);
/* Bytes of workspace of solo_embedding_grad (16-byte aligned), no fewer for more tokens; 0 if the shape is invalid. */
size_t solo_embedding_workspace_bytes(const solo_embedding_shape *shape);
int solo_embedding_grad(const void *grad_rows, const void *tokens, void *grad_table, void *workspace, size_t workspace_bytes,
                        const solo_embedding_shape *shape, void *stream);

/* ---- log probabilities ------------------------------------------------------------------------
 * For every row x of logits, with z = scale * x (scale: the reciprocal of a temperature), L = ln sum e^z
 * and p = e^(z - L):
 *
 *   logprob = z_t - L             of the row's target t
 *   entropy = -sum p ln p
 *   rank = number of columns whose logit is larger than the target's
 *   top_logprob, top_token [rows, top]: z - L of the `top` largest logits and their columns, larger ones
 *            first, ties by the lower column; places behind the last column are -inf and -1
 *   stats [rows, 2]: what solo_logprob_grad takes: the row's largest logit, and the sum of e^z relative to it
 *
 * and for a loss with d loss / d logprob = a, d loss / d entropy = b (one float per row each):
 *
 *   grad_logits_j = scale * (a (delta_jt - p_j) - b p_j (ln p_j + entropy))
 *
 * (the alternatives carry no gradient).  Logits of -inf have probability 0; in a row that has no other,
 * logprob is -inf, entropy and gradient are 0.  A target outside [0, cols) means none (a padding
 * position): the row is not read, logprob and entropy are 0, rank is -1, the alternatives are -inf and -1,
 * the gradient is 0.  Sums are binary32 and relative to the row's largest logit: logprob <= 0, with an error of some 1e-7 of
 * 1 + the distance of the target's z from the largest.  A NaN or +inf in a row makes its logprob, entropy and gradient NaN and its alternatives
 * and rank unspecified.  solo_logprob_with_grad does both for weights that are known beforehand (a mean over
 * tokens), reading the logits from HBM once. */
#define SOLO_TOP_MAX 32
typedef struct solo_logits {
    uint64_t rows, cols;        /* cols below 2^29                                               */
    uint64_t stride;            /* elements from row to row of logits, >= cols                   */
    uint64_t grad_stride;       /* the same of grad_logits                                       */
    uint32_t dtype;             /* of logits and grad_logits                                     */
    uint32_t target_bits;       /* 32 or 64: signed whole numbers                                */
    uint32_t top;               /* alternatives, 0 .. SOLO_TOP_MAX                               */
    uint32_t reserved;          /* must be 0                                                     */
    float scale;                /* > 0, finite                                                   */
    uint32_t reserved2;         /* must be 0                                                     */
} solo_logits;

/* targets may be NULL (no logprob, no rank: both NULL then); every output may be NULL, the alternatives if top is 0. */
int solo_logprob(const void *logits, const void *targets, float *logprob, float *entropy, int32_t *rank,
                 float *top_logprob, int32_t *top_token, float *stats, const solo_logits *shape, void *stream);
/* entropy, stats: of solo_logprob on the same logits, targets and scale.  grad_logprob or grad_entropy may be NULL (0).
 * grad_logits may be the logits themselves (same stride); it must not overlap them in another way. */
int solo_logprob_grad(const void *logits, const void *targets, const float *entropy, const float *stats,
                      const float *grad_logprob, const float *grad_entropy, void *grad_logits,
                      const solo_logits *shape, void *stream);
int solo_logprob_with_grad(const void *logits, const void *targets, const float *grad_logprob, const float *grad_entropy,
                           float *logprob, float *entropy, void *grad_logits, const solo_logits *shape, void *stream);

/* ---- layer norm -------------------------------------------------------------------------------
 * For every row x of `cols` elements
 *
 *   mean = sum x / cols (SOLO_LAYERNORM_RMS: 0)      rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps)
 *   h = (x - mean) rstd       y = h w + b
 *
 * weight NULL is 1, bias NULL 0.  stats [rows, 2], NULL or what solo_layernorm_grad takes: mean and rstd.  With g = grad_y w
 *
 *   grad_x = rstd (g - sum g / cols - h sum(g h) / cols)          (SOLO_LAYERNORM_RMS: without the term in sum g)
 *   grad_weight = sum over the rows of grad_y h                   grad_bias = sum over the rows of grad_y
 *
 * grad_weight and grad_bias have the weights' type; with SOLO_LAYERNORM_ACCUMULATE the sums are added to what is there (a second
 * micro-batch).  Sums are binary32, over the rows in an order that the shape alone determines; one rounding at the end.  The squares
 * are those of the differences from the mean; a row whose mean is many deviations away from zero keeps the digits of its differences, in the gradients, too.  A row with a NaN or an infinity, or whose squares overflow binary32, has unspecified
 * results in that row (NaN behind a NaN) and in the sums over the rows, no others.  y may be x, grad_x may be x or grad_y, where types and
 * strides are the same; otherwise outputs must not overlap inputs. */
#define SOLO_LAYERNORM_RMS 1u
#define SOLO_LAYERNORM_ACCUMULATE 2u
typedef struct solo_layernorm_shape {
    uint64_t rows, cols;        /* below 2^31 and 2^24                                           */
    uint64_t x_stride;          /* elements from row to row of x, >= cols, below 2^31            */
    uint64_t y_stride;          /* the same of y / grad_y                                        */
    uint64_t grad_stride;       /* the same of grad_x                                            */
    uint32_t x_dtype;           /* of x and grad_x                                               */
    uint32_t y_dtype;           /* of y and grad_y                                               */
    uint32_t weight_dtype;      /* of weight, bias and their gradients                           */
    uint32_t flags;             /* SOLO_LAYERNORM_*; ACCUMULATE for the gradient only            */
    float eps;                  /* > 0, finite                                                   */
    uint32_t reserved;          /* must be 0                                                     */
} solo_layernorm_shape;

int solo_layernorm(const void *x, const void *weight, const void *bias, void *y, float *stats, const solo_layernorm_shape *shape, void *stream);
/* Bytes of workspace of solo_layernorm_grad (16-byte aligned), no fewer for more rows; 0 if the shape is invalid. */
size_t solo_layernorm_workspace_bytes(const solo_layernorm_shape *shape);
/* stats: of solo_layernorm on the same x.  grad_x may be NULL, and grad_weight or grad_bias or both (no workspace is needed then), not all three. */
int solo_layernorm_grad(const void *grad_y, const void *x, const void *weight, const float *stats, void *grad_x, void *grad_weight, void *grad_bias,
                        void *workspace, size_t workspace_bytes, const solo_layernorm_shape *shape, void *stream);

/* ---- distillation -----------------------------------------------------------------------------
 * For every row x of a student's logits, with z = scale * x and q = softmax of z, and `top` alternatives of a teacher, values v_k at
 * columns t_k (what solo_logprob writes as top_logprob and top_token, or stored logits):
 *
 *   p_k = softmax of teacher_scale * v over the row's alternatives, r = 0
 *   SOLO_DISTILL_REST: p_k = e^(v_k), and what they leave of 1 is one more alternative, r = 1 - sum p_k (0 where that is below 2^-20:
 *            the values' rounding), against the student's q_r = sum of q_j over the columns that are not among the t_k
 *
 *   loss = sum p_k (ln p_k - ln q_(t_k)) + r (ln r - ln q_r)            (terms with p_k = 0 or r = 0 are 0)
 *   stats [rows, 3]: what solo_distill_grad takes: the row's largest logit, and the sums of e^z relative to it, of all columns and of
 *            those that are not among the t_k.  Where the latter is below 2^-64 and r > 0, another three: the largest logit of those columns,
 *            the sum of all columns negated, and that of those columns relative to their own largest logit
 *
 * and with d loss / d z times scale, for a = grad_loss of the row and T = sum p_k + r:
 *
 *   grad_logits_j = scale * a * (T q_j - sum over the k with t_k = j of p_k)        j among the t_k
 *   grad_logits_j = scale * a * q_j (T - r / q_r)                                   elsewhere (0 where q_r is)
 *
 * A place whose token lies outside [0, cols) or whose value is -inf is none (solo_logprob writes -1 and -inf behind the last column); a
 * column may occur more than once.  What a row without alternatives holds is of no account (a padding position): loss and gradient are 0; its memory
 * has to be readable, like any row's, since logits are read before the alternatives are known.  Where the student
 * gives no probability to an alternative that has some (-inf), the loss is +inf and the gradient the formula's; in a row of -inf alone the loss is +inf, the gradient 0.  A NaN or
 * +inf among the logits or values of a row makes its results NaN or unspecified, no other row's.  q_r is summed by itself, not taken from 1.  Sums
 * are binary32 and relative to the row's largest logit, q_r's to that of its columns where the two lie far apart (1 - sum p_k: binary64).  solo_distill_with_grad does both for weights that are known beforehand,
 * reading the logits from HBM once. */
#define SOLO_DISTILL_REST 1u
#define SOLO_DISTILL_MAX 128
typedef struct solo_distill_shape {
    uint64_t rows, cols;        /* below 2^35 and 2^29                                           */
    uint64_t stride;            /* elements from row to row of logits, >= cols                   */
    uint64_t grad_stride;       /* the same of grad_logits                                       */
    uint64_t value_stride;      /* the same of teacher_value, >= top                             */
    uint64_t token_stride;      /* the same of teacher_token, >= top                             */
    uint32_t top;               /* alternatives, 1 .. SOLO_DISTILL_MAX                           */
    uint32_t dtype;             /* of logits and grad_logits                                     */
    uint32_t value_dtype;       /* of teacher_value                                              */
    uint32_t token_bits;        /* 32 or 64: signed whole numbers                                */
    uint32_t flags;             /* 0 or SOLO_DISTILL_REST                                        */
    uint32_t reserved;          /* must be 0                                                     */
    float scale;                /* > 0, finite                                                   */
    float teacher_scale;        /* > 0, finite; 1 with SOLO_DISTILL_REST                         */
} solo_distill_shape;

/* loss and stats may be NULL. */
int solo_distill(const void *logits, const void *teacher_value, const void *teacher_token, float *loss, float *stats,
                 const solo_distill_shape *shape, void *stream);
/* stats: of solo_distill on the same logits, teacher and scales.  grad_logits may be the logits themselves (same stride); it must not overlap them in another way. */
int solo_distill_grad(const void *logits, const void *teacher_value, const void *teacher_token, const float *stats, const float *grad_loss,
                      void *grad_logits, const solo_distill_shape *shape, void *stream);
int solo_distill_with_grad(const void *logits, const void *teacher_value, const void *teacher_token, const float *grad_loss, float *loss,
                           void *grad_logits, const solo_distill_shape *shape, void *stream);

/* ---- sampling ---------------------------------------------------------------------------------
 * For every row x of logits one column, by a given number u of [0, 1) (greater numbers count as the one next to 1, smaller ones as 0):
 *
 *   w_j = e^((x_j - max x) / temperature)        the columns in the order of their logits, larger ones first, ties by the lower column
 *   kept: the first top_k of the columns with w_j >= min_p, and of these the shortest beginning whose sum of w is
 *            at least top_p times that of them all; one column at least
 *   token = the first column, in that order, at which the running sum of the kept w exceeds u times their sum
 *   logprob = ln of the token's share of the kept w
 *
 * temperature 0, or min_p above 1: the largest logit's column (lowest of several), logprob 0.  top_k <= 0, top_p >= 1, min_p <= 0: no limit by it.  A
 * logit of -inf is never chosen; in a row that has no other the token is -1 and logprob -inf.  A row with a NaN or +inf among its
 * logits, or with a NaN or a negative temperature among its parameters, gives -1 and NaN.
 * Weights are computed in binary64 (off by 2e-13 of themselves) and rounded to whole multiples of 2^-k of the largest, whose sums are exact in any order.  Up to 2^19
 * columns k is 62 - log2 cols (rounded up), 51 at most: a sum is off by no more than cols 2^-(k + 1) of the largest weight, 3.6e-10 for 50257 columns and 2^-25 for
 * 2^19.  In longer rows k follows the sum of the row's weights: off by no more than cols 2^-52 of the largest weight or cols 2^-61 of the sum, whichever is more
 * (2^-23 for 2^29 columns).  The token is that of exact arithmetic unless u times the kept sum, or a limit, lies nearer than that to a border; columns below half
 * a multiple are never chosen. */
typedef struct solo_sample_shape {
    uint64_t rows, cols;        /* below 2^35 and 2^29                                           */
    uint64_t stride;            /* elements from row to row of logits, >= cols                   */
    uint32_t dtype;             /* of logits                                                     */
    uint32_t token_bits;        /* of token, 32 or 64                                            */
    int32_t top_k;              /* where top_k is NULL                                           */
    uint32_t reserved;          /* must be 0                                                     */
    float temperature;          /* where temperature is NULL, >= 0                               */
    float top_p, min_p;         /* where these are NULL, not NaN                                 */
    uint32_t reserved2;         /* must be 0                                                     */
} solo_sample_shape;

/* uniform: float[rows]; temperature, top_k, top_p, min_p [rows]: of the rows' own, each may be NULL (all rows take the shape's); token [rows];
 * logprob: float[rows] or NULL. */
int solo_sample(const void *logits, const float *uniform, const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                void *token, float *logprob, const solo_sample_shape *shape, void *stream);

/* Static, human-readable text for a return code. */
const char *solo_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* SOLO_H */
