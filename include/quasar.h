/*
 * quasar.h -- C ABI of the GB300 (sm_103a) QUASAR reconstruction library.
 *
 * QUASAR ("QUASAR: Lowering the Loss Floor of Quantization-Aware Training
 * with Loss-Aware Reconstruction") rebuilds, at every training step, the
 * quantized weights r that the forward pass uses from the latent weights w:
 * for each group it updates the saliency EMA of squared gradients, searches
 * a small grid of clipping ranges, assigns codes for each range, fits the
 * dequantizer by saliency-weighted least squares, and keeps the range whose
 * weighted reconstruction error is lowest (Algorithm 1; Sec. 4.2 for NVFP4).
 *
 * Conventions shared by every entry point:
 *  - All tensor arguments are DEVICE pointers into memory owned by the caller
 *    (cudaMalloc / a framework allocator).  The library allocates nothing on
 *    these paths and keeps no per-call state.
 *  - Calls are asynchronous on `stream` (NULL = legacy default stream).
 *    Arguments are validated on the host first; on any error a status is
 *    returned and nothing is launched.  A failed launch returns
 *    QUASAR_ERR_CUDA.
 *  - Tensors are row-major [rows, cols].  Groups of `group_size` consecutive
 *    elements of a row share one dequantizer (rows of an nn.Linear weight
 *    [out, in] are split along `in`), so the tensor is a flat sequence of
 *    rows*cols/group_size groups.
 *  - Device pointers to tensors must be 16-byte aligned.  Outputs must not
 *    overlap the inputs w, g or v (checked by address range).
 *  - Inputs holding NaN or Inf give unspecified outputs but never fault.
 *  - A device-side wait that runs out (a shared-memory pipeline stage that
 *    never arrives) does not hang: the kernel records QUASAR_ERR_TIMEOUT in
 *    a per-device status word and returns; quasar_get_device_status reports
 *    and clears it.
 */
#ifndef QUASAR_H
#define QUASAR_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Same type as cudaStream_t; declared here so C callers need no CUDA headers. */
struct CUstream_st;
typedef struct CUstream_st* quasar_stream_t;

typedef enum {
    QUASAR_OK = 0,
    QUASAR_ERR_INVALID_ARG = 1, /* a NULL, out-of-range, misaligned or aliasing argument */
    QUASAR_ERR_UNSUPPORTED = 2, /* a valid request this build has no kernel for           */
    QUASAR_ERR_CUDA = 3,        /* a CUDA runtime call or a launch failed                */
    QUASAR_ERR_TIMEOUT = 4      /* a device-side wait ran out (see quasar_get_device_status) */
} quasar_status;

typedef enum { QUASAR_F32 = 0, QUASAR_BF16 = 1 } quasar_dtype;

/*
 * quasar_options -- variants of the reconstruction, for the *_ex batch entry
 * points and quasar_adamw_recon_int_batch (NULL = all defaults).
 *
 *   saliency      the weights h of the fit (Eq. 4) and the error (Eq. 3):
 *     QUASAR_SALIENCY_EMA          h = v', the EMA of squared gradients
 *                                  (Sec. 4.1.1; the default);
 *     QUASAR_SALIENCY_EMA_SQUARED  h = v'^2 (fp32 square), the alternative
 *                                  weighting the paper compares against
 *                                  (App. A.3);
 *     QUASAR_SALIENCY_UNIFORM      h = 1: scale search and least-squares fit
 *                                  without saliency (the "scale search only"
 *                                  ablation, Sec. 6.5).
 *                 In every mode v is still updated to v' when g is given.
 *   codes_layout  the codes output, when a codes pointer is given:
 *     QUASAR_CODES_U8      one code per byte, [rows, cols] (the default);
 *     QUASAR_CODES_PACKED  the deployment format.  Integer codes: each group
 *                          is one little-endian bitstream of `bits` bits a
 *                          code (code j of the group in bits [j*bits,
 *                          (j+1)*bits) of the group's group_size*bits/8
 *                          bytes), groups in order: rows*cols*bits/8 bytes.
 *                          NVFP4: two E2M1 codes a byte, the even element in
 *                          the low nibble: rows*cols/2 bytes.  (The paper
 *                          deploys real NVFP4 checkpoints, Sec. 6.1, but
 *                          prints no byte layout: these are the usual
 *                          little-endian conventions.)
 *   grid          integer codes only (quasar_recon_int_batch_ex):
 *     QUASAR_GRID_ASYMMETRIC  Eq. 1 and Eq. 4 (the default);
 *     QUASAR_GRID_SYMMETRIC   the offset-free closed form of Sec. 4.1.2:
 *                             Q = 2^(bits-1) - 1 (bits >= 2), step
 *                             s_f = f * max|w| / Q per group, codes
 *                             q = clamp(round_half_even(w / s_f), -Q, Q)
 *                             stored as q + Q, fit s* = sum h q w / sum h q^2
 *                             (s_f when every h > 0 element has q = 0), and
 *                             r = s* q; a = s*, b = -s* Q, so r = a*code + b
 *                             as for asymmetric codes.  A group with
 *                             max|w| = 0 gives codes Q, a = b = 0, r = 0.
 *                             Not available with the fused AdamW step
 *                             (QUASAR_ERR_UNSUPPORTED); NVFP4 and the lookup
 *                             table take only the default
 *                             (QUASAR_ERR_INVALID_ARG).
 * The "Adam weighting only" ablation (no scale search) is F = {1}: clip =
 * {1.0}, n_clip = 1.
 */
typedef enum {
    QUASAR_SALIENCY_EMA = 0,
    QUASAR_SALIENCY_EMA_SQUARED = 1,
    QUASAR_SALIENCY_UNIFORM = 2
} quasar_saliency;

typedef enum { QUASAR_CODES_U8 = 0, QUASAR_CODES_PACKED = 1 } quasar_codes_layout;

typedef enum { QUASAR_GRID_ASYMMETRIC = 0, QUASAR_GRID_SYMMETRIC = 1 } quasar_int_grid;

typedef struct {
    quasar_saliency saliency;
    quasar_codes_layout codes_layout;
    quasar_int_grid grid;
} quasar_options;

/*
 * quasar_recon_int -- QUASAR reconstruction with asymmetric b-bit integer
 * codes (Algorithm 1; code assignment Eq. 1; dequantizer fit Eq. 4; error
 * Eq. 3; saliency EMA Sec. 4.1.1 / App. A.2).
 *
 * For every group of `group_size` consecutive elements:
 *   1. v' = beta2*v + (1-beta2)*g^2 is written back to v, and h = v' is the
 *      saliency.  g == NULL skips the update (h = v, v untouched).
 *   2. c = (min w + max w)/2, rho = (max w - min w)/2.
 *   3. For each factor f = clip[k]: codes q = clamp(round_half_even((w - z)/s),
 *      0, 2^bits - 1) with z = c - f*rho, s = 2*f*rho/(2^bits - 1); the
 *      weighted least-squares (a_k, b_k) minimising sum h (a q + b - w)^2;
 *      its error.
 *   4. The candidate with the lowest error is kept (ties: lowest k);
 *      r = a*q + b.
 *   Degenerate groups: zero range gives q = 0, a = 0, b = w[0], r = w,
 *   k = 0.  All h = 0 in a group: the group is fitted with h = 1.  If every
 *   h > 0 element of a candidate shares one code, that candidate's error is
 *   sum h (w - mean_h(w))^2 and a = its grid step, b = mean_h(w) - a*code.
 *
 * Arguments:
 *   w          [rows, cols] fp32 latent weights (read).
 *   g          [rows, cols] gradient, dtype g_dtype (read), or NULL.
 *   v          [rows, cols] fp32 EMA state (read; overwritten with v').
 *   beta2      EMA decay, 0 <= beta2 < 1.
 *   bits       1..8.
 *   group_size 32, 64, 128 or 256; cols % group_size == 0.
 *   clip       HOST array of n_clip factors, each in (0, 1], in search order;
 *              copied before the call returns.  1 <= n_clip <= 32.
 *   r          [rows, cols] reconstruction, dtype r_dtype (written).
 *   codes      [rows, cols] uint8 codes of the kept candidate, or NULL.
 *   a, b       [rows*cols/group_size] fp32 scale and offset (written).
 *   cand_idx   [rows*cols/group_size] uint8 index into clip[] of the kept
 *              candidate, or NULL.
 * Returns QUASAR_OK, or INVALID_ARG / UNSUPPORTED / CUDA with nothing done
 * (CUDA: a launch failure after validation).  rows*cols == 0 is a no-op.
 */
quasar_status quasar_recon_int(const float* w, const void* g, quasar_dtype g_dtype, float* v,
                               float beta2, int bits, int group_size, const float* clip,
                               int n_clip, int64_t rows, int64_t cols, void* r,
                               quasar_dtype r_dtype, uint8_t* codes, float* a, float* b,
                               uint8_t* cand_idx, quasar_stream_t stream);

/*
 * quasar_int_tensor / quasar_recon_int_batch -- quasar_recon_int over many
 * tensors in one launch (Algorithm 1 applied to every linear weight of a
 * model at each step), with the same quantization settings for all of them.
 * The units of work of all tensors are numbered consecutively and shared by
 * one persistent grid, so small tensors cost no launch of their own and the
 * step has a single tail.
 *
 * Each descriptor holds one tensor's arguments exactly as quasar_recon_int
 * takes them (same meaning, layout and rules); either every non-empty tensor
 * has a gradient g or none does.  The descriptor array is a HOST array read before
 * the call returns; tensors may be listed in any order and may differ in
 * shape.  More than 256 tensors are processed 256 per launch.
 * Returns as quasar_recon_int; every tensor is validated before anything is
 * launched.  The paper has no batched form: this entry point only removes
 * per-tensor launches.
 */
typedef struct {
    const float* w;
    const void* g;
    float* v;
    void* r;
    uint8_t* codes;
    float* a;
    float* b;
    uint8_t* cand_idx;
    int64_t rows;
    int64_t cols;
} quasar_int_tensor;

quasar_status quasar_recon_int_batch(const quasar_int_tensor* tensors, int n_tensors,
                                     quasar_dtype g_dtype, float beta2, int bits, int group_size,
                                     const float* clip, int n_clip, quasar_dtype r_dtype,
                                     quasar_stream_t stream);

/* quasar_recon_int_batch with variant options (see quasar_options; NULL =
 * defaults).  With packed codes, each descriptor's codes buffer holds
 * rows*cols*bits/8 bytes (16-byte aligned).  An invalid option value gives
 * QUASAR_ERR_INVALID_ARG. */
quasar_status quasar_recon_int_batch_ex(const quasar_int_tensor* tensors, int n_tensors,
                                        quasar_dtype g_dtype, float beta2, int bits,
                                        int group_size, const float* clip, int n_clip,
                                        quasar_dtype r_dtype, const quasar_options* options,
                                        quasar_stream_t stream);

/*
 * quasar_adamw_tensor / quasar_adamw_recon_int_batch -- one AdamW step fused
 * with the integer-code reconstruction of the updated weights.  The paper
 * trains with AdamW and takes AdamW's second moment as the saliency h
 * (Sec. 4.1.1; training setup in Sec. 6.1); the reconstruction of Algorithm 1
 * follows every optimizer step.  Here both run in one pass over the weights:
 * each element of w, g, m, v is read once and w', m', v', r written once.
 *
 * Per element (t = step, decoupled weight decay, bias-corrected moments):
 *   m' = beta1*m + (1-beta1)*g           written back to m
 *   v' = beta2*v + (1-beta2)*g^2         written back to v
 *   w' = w*(1 - lr*wd) - (lr/(1-beta1^t)) * m' / (sqrt(v')/sqrt(1-beta2^t) + eps)
 *                                        written back to w
 * then quasar_recon_int of w' with saliency h = v' (steps 2-4 there).
 * Arithmetic is fp32: m', v' within one rounding of each product; the
 * decrement w*lr*wd + step_size*m'/den is formed to a few ulps (root and
 * quotient by the fast reciprocal-square-root and reciprocal, 2 ulps each)
 * and added to w once, so w' is the correctly rounded result up to those
 * ulps of the decrement.
 *
 * Descriptor fields as in quasar_int_tensor, plus m (fp32 first moment,
 * [rows, cols], read and overwritten), and w is overwritten with w'.  g is
 * required for every non-empty tensor.  w, m, v, g must not overlap one
 * another; the outputs r, codes, a, b, cand_idx must not overlap any of
 * them.  Hyper-parameters: lr >= 0, 0 <= beta1 < 1, 0 <= beta2 < 1,
 * eps > 0, weight_decay >= 0 (all finite), step >= 1.  options as in
 * quasar_recon_int_batch_ex (NULL = defaults).
 * Returns as quasar_recon_int_batch.
 */
typedef struct {
    float* w;
    const void* g;
    float* m;
    float* v;
    void* r;
    uint8_t* codes;
    float* a;
    float* b;
    uint8_t* cand_idx;
    int64_t rows;
    int64_t cols;
} quasar_adamw_tensor;

quasar_status quasar_adamw_recon_int_batch(const quasar_adamw_tensor* tensors, int n_tensors,
                                           quasar_dtype g_dtype, float lr, float beta1,
                                           float beta2, float eps, float weight_decay,
                                           int64_t step, int bits, int group_size,
                                           const float* clip, int n_clip, quasar_dtype r_dtype,
                                           const quasar_options* options, quasar_stream_t stream);

/*
 * quasar_recon_nvfp4 -- QUASAR for NVFP4 (Sec. 4.2): E2M1 codes, one FP8
 * (E4M3) scale per 16 consecutive elements, one FP32 scale per tensor.
 *
 *   s_T = amax / (6*448) from the tensor absmax (amax = 0 gives s_T = 1);
 *   the tensor scale is not optimised.  For each 16-element block and each
 *   factor f = clip[k]: search scale sigma = f*max|w_block|/6; codes
 *   q = sign(w) * E2M1_rne(min(|w|/sigma, 6)); least-squares slope
 *   a* = sum h q w / sum h q^2; E4M3 scale e = E4M3_rne_satfinite(a* / s_T);
 *   error sum h (s_T*e*q - w)^2.  The candidate with the lowest error is
 *   kept (ties: lowest k) and r = s_T*e*q.  The saliency update is the same
 *   as in quasar_recon_int.  A zero block gives q = 0, e = 0, r = 0; a
 *   candidate whose weighted codes are all zero takes e = E4M3(sigma/s_T).
 *
 * Arguments as in quasar_recon_int, plus:
 *   cols        cols % 16 == 0.
 *   tensor_amax device pointer to max|w| of this tensor (fp32), or NULL to
 *               have the library compute it (one extra read of w).
 *   codes       [rows, cols] uint8, one E2M1 nibble per byte
 *               (sign << 3 | magnitude index 0..7; magnitude 0 is +0), or NULL.
 *   block_scale [rows*cols/16] uint8 E4M3 bit patterns (written).
 *   tensor_scale device pointer to one fp32, receives s_T (written).
 *   cand_idx    [rows*cols/16] uint8, or NULL.
 */
quasar_status quasar_recon_nvfp4(const float* w, const void* g, quasar_dtype g_dtype, float* v,
                                 float beta2, const float* clip, int n_clip, int64_t rows,
                                 int64_t cols, const float* tensor_amax, void* r,
                                 quasar_dtype r_dtype, uint8_t* codes, uint8_t* block_scale,
                                 float* tensor_scale, uint8_t* cand_idx,
                                 quasar_stream_t stream);

/*
 * quasar_nvfp4_tensor / quasar_recon_nvfp4_batch -- quasar_recon_nvfp4 over
 * many tensors with the same settings: one absmax pass over the tensors
 * whose amax is not supplied, one scale pass, and one persistent
 * reconstruction launch whose units are numbered across the tensors.
 * Each descriptor holds one tensor's arguments as quasar_recon_nvfp4 takes
 * them (same meaning and rules; each tensor has its own tensor_scale slot and
 * optional tensor_amax); either every non-empty tensor has a gradient or none
 * does.  HOST array, read before the call returns; more than 256 tensors are
 * processed 256 per launch.  Returns as quasar_recon_nvfp4; every tensor is
 * validated before anything is launched.  The paper has no batched form.
 */
typedef struct {
    const float* w;
    const void* g;
    float* v;
    const float* tensor_amax;
    void* r;
    uint8_t* codes;
    uint8_t* block_scale;
    float* tensor_scale;
    uint8_t* cand_idx;
    int64_t rows;
    int64_t cols;
} quasar_nvfp4_tensor;

quasar_status quasar_recon_nvfp4_batch(const quasar_nvfp4_tensor* tensors, int n_tensors,
                                       quasar_dtype g_dtype, float beta2, const float* clip,
                                       int n_clip, quasar_dtype r_dtype, quasar_stream_t stream);

/* quasar_recon_nvfp4_batch with variant options (see quasar_options; NULL =
 * defaults).  With packed codes, each descriptor's codes buffer holds
 * rows*cols/2 bytes (16-byte aligned).  An invalid option value gives
 * QUASAR_ERR_INVALID_ARG. */
quasar_status quasar_recon_nvfp4_batch_ex(const quasar_nvfp4_tensor* tensors, int n_tensors,
                                          quasar_dtype g_dtype, float beta2, const float* clip,
                                          int n_clip, quasar_dtype r_dtype,
                                          const quasar_options* options, quasar_stream_t stream);

/*
 * quasar_adamw_nvfp4_tensor / quasar_adamw_recon_nvfp4_batch -- one AdamW
 * step (as quasar_adamw_recon_int_batch) followed by the NVFP4
 * reconstruction (as quasar_recon_nvfp4_batch) of the updated weights with
 * saliency h = v'.  The NVFP4 tensor scale needs the absmax of w' before any
 * block is reconstructed, so the step is two passes: one over w, g, m, v
 * that writes w', m', v' and takes max |w'| per tensor (no separate absmax
 * pass), and the reconstruction pass over w', v' (no gradient: v is not
 * updated twice).  Reads 14 + 8 and writes 12 + 2 bytes a weight.
 *
 * Descriptor fields as in quasar_nvfp4_tensor without tensor_amax, plus m
 * (fp32 first moment, read and overwritten); w is overwritten with w'.  g
 * and m are required for every non-empty tensor; w, g, m, v pairwise
 * disjoint; outputs disjoint from all of them.  Hyper-parameters and
 * options as quasar_adamw_recon_int_batch.
 */
typedef struct {
    float* w;
    const void* g;
    float* m;
    float* v;
    void* r;
    uint8_t* codes;
    uint8_t* block_scale;
    float* tensor_scale;
    uint8_t* cand_idx;
    int64_t rows;
    int64_t cols;
} quasar_adamw_nvfp4_tensor;

quasar_status quasar_adamw_recon_nvfp4_batch(const quasar_adamw_nvfp4_tensor* tensors,
                                             int n_tensors, quasar_dtype g_dtype, float lr,
                                             float beta1, float beta2, float eps,
                                             float weight_decay, int64_t step, const float* clip,
                                             int n_clip, quasar_dtype r_dtype,
                                             const quasar_options* options, quasar_stream_t stream);

/*
 * quasar_lut_tensor / quasar_recon_lut_batch -- QUASAR for the Rubin INT3
 * lookup-table format (App. B): 3-bit indices and a table of 8 E4M3 entries
 * per block of 8 rows x 64 columns (512 weights, 3.125 bits a weight).
 *
 * For every block (rows 8i..8i+7, columns 64j..64j+63; blocks in row-major
 * order):
 *   1. v' and h as in quasar_recon_int (step 1; options.saliency applies).
 *   2. c = (min w + max w)/2, rho = (max w - min w)/2 over the block.
 *   3. For each f = clip[k]: indices q = clamp(round_half_even((w - z)/s),
 *      0, 7) with z = c - f*rho, s = 2*f*rho/7 (Eq. 1 with qmax = 7); entry
 *      C_j = E4M3(sum_{q=j} h w / sum_{q=j} h) (Eq. rubin-fit), or
 *      E4M3(z + j*s) for an index whose elements carry no saliency; the error
 *      sum h (C_q - w)^2.
 *   4. The candidate with the lowest error is kept (ties: lowest k);
 *      r = C_q.
 *   E4M3 entries are signed, round to nearest even, saturate at 448, and a
 *   magnitude 0 is stored as +0.  A zero-range block: indices 0, every entry
 *   E4M3(c), k = 0.  All h = 0 in a block: h = 1.
 *
 * Descriptor fields as in quasar_int_tensor, except:
 *   book      [rows/8 * cols/64, 8] uint8 E4M3 entries, required (written).
 *   codes     one index a byte, [rows, cols]; or, with packed codes
 *             (options), 192 bytes a block: the block's 512 indices in
 *             row-major block order, 3 bits each, little-endian.
 *   cand_idx  [rows/8 * cols/64] uint8, or NULL.
 * rows % 8 == 0 and cols % 64 == 0, and fewer than 2^32 blocks a tensor,
 * else QUASAR_ERR_INVALID_ARG.  Other rules, options and returns as
 * quasar_recon_int_batch_ex.
 */
typedef struct {
    const float* w;
    const void* g;
    float* v;
    void* r;
    uint8_t* codes;
    uint8_t* book;
    uint8_t* cand_idx;
    int64_t rows;
    int64_t cols;
} quasar_lut_tensor;

quasar_status quasar_recon_lut_batch(const quasar_lut_tensor* tensors, int n_tensors,
                                     quasar_dtype g_dtype, float beta2, const float* clip,
                                     int n_clip, quasar_dtype r_dtype, const quasar_options* options,
                                     quasar_stream_t stream);

/*
 * quasar_tensor_amax -- amax_out[0] = max |w[i]| over n fp32 elements (the
 * NVFP4 tensor statistic of Sec. 4.2).  amax_out is a device pointer; it is
 * overwritten.  n == 0 writes 0.
 */
quasar_status quasar_tensor_amax(const float* w, int64_t n, float* amax_out,
                                 quasar_stream_t stream);

/*
 * Operators around the reconstruction.  A training step reads the
 * reconstructed weights r in matrix products, compares the student's logits
 * with a teacher's (the forward KL the paper distils with, Sec. 6.1), and
 * differentiates both; the weight gradient is the g the next reconstruction
 * reads.  The conventions at the top of this file hold, with these
 * differences: matrices are row-major with a row stride (`ld`, in elements,
 * at least the row's length), and only pointers that are said to be are
 * 16-byte aligned; the others need their element's alignment.  Sums and
 * softmax statistics are fp32; an output of fewer bits is rounded once.
 */

/* y = z (none), max(z, 0), z / (1 + e^-z), z Phi(z) */
typedef enum {
    QUASAR_ACT_NONE = 0,
    QUASAR_ACT_RELU = 1,
    QUASAR_ACT_SILU = 2,
    QUASAR_ACT_GELU = 3
} quasar_activation;

/*
 * quasar_linear -- z = x r^T + bias, y = activation(z) + residual.
 *
 *   x         [tokens, inputs] bf16, 16-byte aligned, ld_x % 8 == 0.
 *   r         [features, inputs] bf16 (a reconstruction with bf16 r), 16-byte
 *             aligned, ld_r % 8 == 0.
 *   bias      [features] fp32, or NULL.
 *   residual  [tokens, features] of y's dtype, or NULL; it may be y itself
 *             (same pointer and stride).
 *   y         [tokens, features], dtype y_dtype (written).
 *   pre       [tokens, features] bf16, receives z (what the activation's
 *             gradient needs), or NULL.
 * Any number of tokens, from one up; features may be odd, rows of y, pre and
 * residual may start anywhere.  tokens or features 0 is a no-op; inputs 0
 * gives z = bias.  Products are exact bf16 x bf16, accumulated in fp32.
 * Outputs must share no byte with inputs, but for the residual; columns of one
 * buffer share none.
 */
quasar_status quasar_linear(const void* x, int64_t ld_x, const void* r, int64_t ld_r,
                            const float* bias, quasar_activation activation, const void* residual,
                            int64_t ld_residual, int64_t tokens, int64_t features, int64_t inputs,
                            void* y, quasar_dtype y_dtype, int64_t ld_y, void* pre, int64_t ld_pre,
                            quasar_stream_t stream);

/*
 * quasar_linear_grad_input -- dx = (dz r) * activation_in'(pre_in) + residual.
 *
 *   dz        [tokens, features] bf16, the gradient at z, 16-byte aligned,
 *             ld_dz % 8 == 0.
 *   r         as in quasar_linear.
 *   pre_in    [tokens, inputs] bf16: the z that the layer's input was
 *             activated from, with activation_in; NULL (with
 *             QUASAR_ACT_NONE) if the input was not an activation.  Then dx
 *             is the gradient at that z: the dz of the layer below.
 *   residual  [tokens, inputs] of dx's dtype, added last, or NULL.
 *   dx        [tokens, inputs], dtype dx_dtype (written); it may be residual
 *             or a bf16 pre_in itself.
 */
quasar_status quasar_linear_grad_input(const void* dz, int64_t ld_dz, const void* r, int64_t ld_r,
                                       const void* pre_in, int64_t ld_pre_in,
                                       quasar_activation activation_in, const void* residual,
                                       int64_t ld_residual, int64_t tokens, int64_t features,
                                       int64_t inputs, void* dx, quasar_dtype dx_dtype,
                                       int64_t ld_dx, quasar_stream_t stream);

/*
 * quasar_linear_grad_weight -- dr = dz^T x and dbias = the column sums of dz.
 *
 *   dz, x     as above (x is not read when dr is NULL).
 *   dr        [features, inputs], dtype dr_dtype (written), or NULL: the g of
 *             the reconstruction entry points.
 *   dbias     [features] fp32 (written), or NULL.
 * tokens 0 gives zeros.  The order of every sum is fixed: the same inputs
 * give the same bits.
 */
quasar_status quasar_linear_grad_weight(const void* dz, int64_t ld_dz, const void* x, int64_t ld_x,
                                        int64_t tokens, int64_t features, int64_t inputs, void* dr,
                                        quasar_dtype dr_dtype, int64_t ld_dr, float* dbias,
                                        quasar_stream_t stream);

/*
 * quasar_activation_grad -- dz = dy * activation'(pre) in bf16 (all bf16,
 * [rows, cols]): the gradient at z of a layer whose own output was activated.
 * With QUASAR_ACT_NONE pre is not read and dz is a copy, which brings dy to
 * the row stride the products need.  dz may be dy or pre itself.
 */
quasar_status quasar_activation_grad(const void* dy, int64_t ld_dy, const void* pre, int64_t ld_pre,
                                     quasar_activation activation, int64_t rows, int64_t cols,
                                     void* dz, int64_t ld_dz, quasar_stream_t stream);

/*
 * quasar_top_logits -- each row's k largest logits, largest first.
 *
 *   logits       [rows, vocab] bf16 or fp32 (dtype); rows may start anywhere.
 *   k            1 .. min(256, vocab).
 *   temperature  1e-6 .. 1e6.
 *   values       [rows, k] fp32: the logits themselves (not scaled).
 *   indices      [rows, k] int32.  Equal values rank by the lowest index.
 *   lse          [rows] fp32: log sum exp(logits / temperature) over the
 *                vocabulary (-inf for a row of -inf, inf for one with an inf,
 *                NaN for one with a NaN), or NULL.
 * -inf logits are ordinary values (masked entries), and a NaN ranks above
 * everything.  Rows as long as in quasar_distill_top.
 */
quasar_status quasar_top_logits(const void* logits, quasar_dtype dtype, int64_t ld, int64_t rows,
                                int64_t vocab, int k, float temperature, float* values,
                                int32_t* indices, float* lse, quasar_stream_t stream);

/*
 * quasar_distill_top -- forward KL divergence of the student from a teacher
 * of whom each row keeps k logits, with its gradient if asked.
 *
 * With z = logits / temperature and q = softmax(z):
 *   teacher_lse given: p_k = exp(values_k / temperature - teacher_lse) and
 *     everything not listed is one further outcome, the rest, of teacher mass
 *     p_r = max(0, 1 - sum p_k) and student mass q_r;
 *   teacher_lse NULL: p = softmax of the listed values / temperature, p_r = 0.
 *   loss = sum_k p_k log(p_k / q_k) + p_r log(p_r / q_r)
 *   grad = row_weight * d loss / d logits
 * The loss is summed as p log(p/q) - p + q, which is the same where p sums to
 * one.  teacher_lse may leave it at another sum (above one, or below with the
 * whole vocabulary listed; by its rounding, some 1e-7, or because it belongs
 * to other values): the loss is then larger by 1 - sum p, the gradient is that
 * of the formula.
 *
 *   logits       [rows, vocab] bf16 or fp32; rows may start anywhere.
 *   indices      [rows, k] int32, distinct within a row.  An index outside
 *                [0, vocab) marks an absent entry (a row with fewer than k).
 *   values       [rows, k] fp32, 1 <= k <= 256; temperature 1e-6 .. 1e6.
 *   row_weight   [rows] fp32 (what the row counts in the total), or NULL for
 *                1.  A row of weight 0 is not read: loss, statistics and
 *                gradient 0, whatever its logits hold.
 *   loss         [rows] fp32, not weighted (written).
 *   stats        [rows, 2] fp32: log sum exp z over the vocabulary and over
 *                the unlisted entries, for the backward call; or NULL.
 *   grad         [rows, vocab] of the logits' dtype, or NULL; it may be the
 *                logits themselves (same pointer and stride).
 * -inf logits are ordinary values (q = 0; a listed one with p > 0 makes the
 * loss inf; a row of nothing else has loss inf and gradient 0).  A teacher
 * without mass gives loss and gradient 0: not a single entry of mass with
 * teacher_lse NULL, or a teacher_lse of -inf (a row of -inf).  A NaN logit
 * makes loss, statistics and gradient of its row NaN, a +inf loss and
 * gradient.  A NaN among a row's listed values or in its teacher_lse makes
 * loss and gradient NaN, and so does a listed +inf (teacher_lse +inf or NULL).
 * Up to 6.4 million fp32 or 12.8 million bf16 logits a row (UNSUPPORTED
 * beyond).
 */
quasar_status quasar_distill_top(const void* logits, quasar_dtype dtype, int64_t ld, int64_t rows,
                                 int64_t vocab, const int32_t* indices, const float* values, int k,
                                 const float* teacher_lse, const float* row_weight,
                                 float temperature, float* loss, float* stats, void* grad,
                                 int64_t ld_grad, quasar_stream_t stream);

/* quasar_distill_top_backward -- the gradient alone, from the statistics a
 * forward call kept, where the rows' weights (the gradient that reaches each
 * row's loss) are known only later.  Arguments as above; stats is read.  The
 * statistics are fp32: where all of a row's unlisted logits (or all of its
 * logits) over the temperature lie beyond some 2^20 from zero, their spacing
 * there is what this gradient is good to in the exponent; the forward call's
 * own has no such limit. */
quasar_status quasar_distill_top_backward(const void* logits, quasar_dtype dtype, int64_t ld,
                                          int64_t rows, int64_t vocab, const int32_t* indices,
                                          const float* values, int k, const float* teacher_lse,
                                          const float* stats, const float* row_weight,
                                          float temperature, void* grad, int64_t ld_grad,
                                          quasar_stream_t stream);

/*
 * The layers between the products: embedding, layer norm and attention, with
 * their gradients.  The conventions of the operators above hold: row-major
 * matrices with a row stride, rows that may start anywhere unless said
 * otherwise, fp32 sums and statistics, one rounding of an output of fewer
 * bits, and sums in a fixed order (the same inputs give the same bits).  Calls
 * that need scratch memory say how much in a call of their own; it is the
 * caller's, 16-byte aligned, holds nothing before or after, and must not be
 * used by another call until this one's work is done (calls on one stream may
 * share it).
 */

typedef enum { QUASAR_I32 = 0, QUASAR_I64 = 1 } quasar_index_type;

/*
 * quasar_embedding -- y[t] = scale table[ids[t]] + residual[t].
 *
 *   ids       [tokens] int32 or int64 (ids_type).  One outside [0, vocab)
 *             takes zeros for its row (padding).
 *   table     [vocab, width] bf16 or fp32.
 *   residual  [tokens, width] of y's dtype, or NULL; it may be y itself.
 *   y         [tokens, width], dtype y_dtype (written).
 */
quasar_status quasar_embedding(const void* ids, quasar_index_type ids_type, int64_t tokens, const void* table,
                               quasar_dtype table_dtype, int64_t ld_table, int64_t vocab, int64_t width, float scale,
                               const void* residual, int64_t ld_residual, void* y, quasar_dtype y_dtype, int64_t ld_y,
                               quasar_stream_t stream);

/*
 * quasar_embedding_backward -- dtable[v] = scale times the sum of the rows of
 * dy (bf16 or fp32 [tokens, width]) whose id is v: the g of the reconstruction
 * entry points.  Every row of dtable ([vocab, width], dtype dtable_dtype) is
 * written, with zeros where no token has its id; with accumulate 1 the sums are
 * added to what it holds, and rows without tokens are not touched.  Ids outside
 * [0, vocab) count nowhere.
 */
quasar_status quasar_embedding_backward_workspace(int64_t tokens, int64_t width, int64_t* bytes);
quasar_status quasar_embedding_backward(const void* dy, quasar_dtype dy_dtype, int64_t ld_dy, const void* ids,
                                        quasar_index_type ids_type, int64_t tokens, int64_t vocab, int64_t width,
                                        float scale, void* dtable, quasar_dtype dtable_dtype, int64_t ld_dtable,
                                        int accumulate, void* workspace, int64_t workspace_bytes,
                                        quasar_stream_t stream);

/*
 * quasar_layer_norm -- y = (x - mean) rstd weight + bias for each row, with
 * rstd = (mean((x - mean)^2) + eps)^-1/2.  With center 0 the mean is taken as
 * 0 (the root-mean-square norm).
 *
 *   x         [rows, cols] bf16 or fp32.
 *   weight, bias  [cols] fp32; NULL: 1 and 0.
 *   eps       finite, at least 0.  (A row without variance and eps 0 give NaN.)
 *   y         [rows, cols], dtype y_dtype (written); it may be x itself (same
 *             pointer, stride and dtype).
 *   stats     [rows, 2] fp32: mean and rstd, for the backward call; or NULL.
 * rows 0 is a no-op; cols 0 with rows is INVALID_ARG.
 */
quasar_status quasar_layer_norm(const void* x, quasar_dtype x_dtype, int64_t ld_x, const float* weight,
                                const float* bias, int64_t rows, int64_t cols, int center, float eps, void* y,
                                quasar_dtype y_dtype, int64_t ld_y, float* stats, quasar_stream_t stream);

/*
 * quasar_layer_norm_backward -- from dy (bf16 or fp32 [rows, cols]), x and the
 * forward call's stats, with xh = (x - mean) rstd and u = dy weight:
 *
 *   dx       rstd (u - mean(u) - xh mean(u xh)) + residual (without mean(u)
 *            where center is 0), dtype dx_dtype, or NULL; it may be dy, x or
 *            the residual itself (same pointer, stride and dtype).
 *   residual [rows, cols] of dx's dtype: the gradient that goes around the
 *            layer, or NULL.
 *   dweight  [cols] fp32: the sum over the rows of dy xh, or NULL.
 *   dbias    [cols] fp32: the sum over the rows of dy, or NULL.
 * rows 0 gives dweight and dbias of zeros.
 */
quasar_status quasar_layer_norm_backward_workspace(int64_t rows, int64_t cols, int64_t* bytes);
quasar_status quasar_layer_norm_backward(const void* dy, quasar_dtype dy_dtype, int64_t ld_dy, const void* x,
                                         quasar_dtype x_dtype, int64_t ld_x, const float* weight, const float* stats,
                                         int64_t rows, int64_t cols, int center, const void* residual,
                                         int64_t ld_residual, void* dx, quasar_dtype dx_dtype, int64_t ld_dx,
                                         float* dweight, float* dbias, void* workspace, int64_t workspace_bytes,
                                         quasar_stream_t stream);

/*
 * quasar_attention -- y = softmax(scale q k^T) v for each head, over sequences
 * packed along the rows.
 *
 *   q         [tokens, heads x head_dim] bf16.
 *   k, v      [keys, kv_heads x head_dim] bf16; heads / kv_heads consecutive
 *             heads of q share one of k and v.
 *   starts    [sequences + 1] int32: sequence i has the rows starts[i] ..
 *             starts[i + 1] - 1 of q, key_starts alike for k and v.  Both are
 *             read on the device and must not decrease or leave the tensors
 *             (rows outside are not accessed, whatever they hold).  NULL with
 *             sequences 1: every row.
 *   causal    1: a sequence's last token sees its last key, the token before it
 *             one key less, and so on (so one token sees every key); 0: every
 *             token sees every key of its sequence.
 *   scale     above 0, and finite times log2(e) too.
 *   y         [tokens, heads x head_dim] bf16 (written).
 *   lse       [tokens, heads] fp32: log sum exp of the scaled scores, for the
 *             backward call; or NULL.
 * q, k, v and y are 16-byte aligned with row strides of a multiple of 8, and so
 * is head_dim, at most 128 (UNSUPPORTED beyond; at most 128 heads that share
 * keys).  Columns of one buffer (a projection's result) are fine.  A token that
 * sees no key, and a row of no sequence, has y 0 and lse -inf.  A value that is
 * not finite reaches the rows of its sequence alone; in v it may reach those
 * that see other keys and not its own, as 0 times it does in the formula.  Sums
 * over keys (and over rows, for the gradients) are fp32, made by the matrix cores
 * up to 131072 terms at a time, which cuts off at most 2^-10 of their sizes.
 */
quasar_status quasar_attention(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                               int64_t tokens, int64_t keys, int64_t heads, int64_t kv_heads, int64_t head_dim,
                               const int32_t* starts, const int32_t* key_starts, int64_t sequences, int causal,
                               float scale, void* y, int64_t ld_y, float* lse, quasar_stream_t stream);

/*
 * quasar_attention_backward -- the gradients of quasar_attention in q, k and v
 * from dy (the gradient at y), with the y and lse that the forward call wrote.
 *
 *   dy, y     [tokens, heads x head_dim] bf16, as q.
 *   lse       [tokens, heads] fp32.
 *   dq        [tokens, heads x head_dim] bf16 (written), or NULL.
 *   dk, dv    [keys, kv_heads x head_dim] bf16 (written), or both NULL: sums
 *             over the heads that share them.
 * dq, dk and dv are aligned as q; columns of one buffer (what the projection's
 * own backward pass reads) are fine.  Rows of no sequence, tokens that see no
 * key and keys that no token sees have gradients 0.
 */
quasar_status quasar_attention_backward_workspace(int64_t tokens, int64_t heads, int64_t* bytes);
quasar_status quasar_attention_backward(const void* dy, int64_t ld_dy, const void* q, int64_t ld_q, const void* k,
                                        int64_t ld_k, const void* v, int64_t ld_v, const void* y, int64_t ld_y,
                                        const float* lse, int64_t tokens, int64_t keys, int64_t heads, int64_t kv_heads,
                                        int64_t head_dim, const int32_t* starts, const int32_t* key_starts,
                                        int64_t sequences, int causal, float scale, void* dq, int64_t ld_dq, void* dk,
                                        int64_t ld_dk, void* dv, int64_t ld_dv, void* workspace,
                                        int64_t workspace_bytes, quasar_stream_t stream);

/*
 * quasar_get_device_status -- synchronises `stream`, then returns
 * QUASAR_ERR_TIMEOUT if any kernel of this library on the current device
 * recorded a timed-out wait since the previous query (and clears the record),
 * QUASAR_ERR_CUDA if the synchronisation failed, else QUASAR_OK.
 */
quasar_status quasar_get_device_status(quasar_stream_t stream);

/*
 * quasar_debug_force_timeout -- testing hook for the failure path.  While
 * set (nanoseconds > 0), the next kernels of this library on the calling
 * host thread's current device also wait, for that many nanoseconds, on a
 * pipeline barrier that nothing ever signals; the wait runs out, the kernel
 * records QUASAR_ERR_TIMEOUT, drains its own copies in flight and returns.
 * 0 turns the hook off.  Never needed in normal use.
 */
void quasar_debug_force_timeout(int64_t nanoseconds);

/*
 * quasar_debug_set_stats -- tuning hook.  While device_counters (a device
 * array of at least 8 unsigned ints owned by the caller) is set, the
 * reconstruction kernels atomically count [0] the groups/blocks whose
 * candidates were re-evaluated exactly because of a near tie, [1] the
 * integer groups whose kept fit was recomputed in compensated (float-float)
 * arithmetic, [2] the integer groups with near-tie contenders or
 * equal-sum candidates, [3] the thread blocks of the integer kernel whose
 * code-clamp sets hold more than one candidate (see quasar_debug_set_hoist),
 * [4] the candidates whose error was recomputed from a two-pass fit, [5] those
 * whose error was recomputed from their own moment sums and [6] the
 * equal-sum candidates checked code by code.  NULL turns counting off.
 * Process-wide; never needed in normal use.
 */
void quasar_debug_set_stats(unsigned int* device_counters);

/*
 * quasar_debug_set_hoist -- tuning hook.  Where the clip factors allow it,
 * the integer entry points pick a kernel that clamps |w - c| once per set of
 * consecutive candidates instead of every candidate's code: sets of 4 or 2,
 * and with at most 8 candidates also one set of 8 or the runs 3, 3 and 2
 * (the codes are the same bit for bit).  While enable is 0 they always take
 * the per-candidate clamp; 1 (the default, or the environment variable
 * QUASAR_HOIST at load) restores the automatic choice.  Process-wide; never
 * needed in normal use.
 */
void quasar_debug_set_hoist(int enable);

/* Static, human-readable name of a status code. */
const char* quasar_status_string(quasar_status status);

/* Library version as major*10000 + minor*100 + patch. */
int quasar_version(void);

#ifdef __cplusplus
}
#endif

#endif /* QUASAR_H */
