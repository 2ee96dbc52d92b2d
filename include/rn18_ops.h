/* rn18_ops.h - single-operator entry points of the gfx950 ResNet-18 library.
 *
 * These expose the kernels the training step is built from, on the library's
 * internal layouts, so each can be checked against a reference on its own.
 * The operators are those of the ResNet-18 training step (the unit of work of
 * the paper's Sec. 3 and 4 schemes); the paper itself gives no operator
 * formulas, so each follows the textbook definition stated below.
 *
 * Common rules: device pointers, caller-owned, 16-byte aligned; `prec` is
 * RN18_FP32 (float elements) or RN18_BF16 (bf16 elements as uint16 bit
 * patterns); activations are NHWC; channel counts of activation tensors must
 * be multiples of 4 (fp32) or 8 (bf16). Work is enqueued on `hip_stream`.
 * Invalid arguments return RN18_EINVAL before any launch, among them any
 * tensor of more than 2^31 - 2^24 bytes (32-bit byte offsets in the kernels).
 */
#ifndef RN18_OPS_H
#define RN18_OPS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Convolution, no bias, zero padding, square kernel k, stride s, pad p:
 *   y[n,i,j,o] = sum_{c,kh,kw} w[o,kh,kw,c] * x[n, i*s-p+kh, j*s-p+kw, c]
 * x [N][H][W][Cin], w [Cout][k][k][Cin] (OHWI), y [N][Ho][Wo][Cout] with
 * Ho = (H+2p-k)/s + 1. Implicit GEMM on MFMA, fp32 accumulation. */
int rn18op_conv2d_fwd(int prec, const void* x, const void* w_ohwi, void* y, int N, int H, int W, int Cin, int Cout,
                      int k, int s, int p, void* hip_stream);

/* Data gradient (adjoint of the above in x):
 *   dx[n,h,w,c] = sum over (i,j,kh,kw) with i*s-p+kh = h, j*s-p+kw = w of
 *                 w[o,kh,kw,c] * dy[n,i,j,o]
 * dy [N][Ho][Wo][Cout], w_ihwo [Cin][k][k][Cout] (the forward weights with
 * the channel axes exchanged), dx [N][H][W][Cin]. Stride 2 runs as four
 * parity-phase sub-convolutions (no multiplications by inserted zeros). */
int rn18op_conv2d_dgrad(int prec, const void* dy, const void* w_ihwo, void* dx, int N, int H, int W, int Cin,
                        int Cout, int k, int s, int p, void* hip_stream);

/* Weight gradient: dw[o,c,kh,kw] = sum_{n,i,j} dy[n,i,j,o] * x[n,i*s-p+kh,j*s-p+kw,c]
 * written fp32 in OIHW order for the first cin_real of the Cin channels.
 * Needs `workspace` of rn18op_conv2d_wgrad_workspace(...) bytes for the
 * deterministic split-K partial sums. */
size_t rn18op_conv2d_wgrad_workspace(int prec, int N, int H, int W, int Cin, int Cout, int k, int s, int p);
int rn18op_conv2d_wgrad(int prec, const void* dy, const void* x, float* dw_oihw, int N, int H, int W, int Cin,
                        int cin_real, int Cout, int k, int s, int p, void* workspace, size_t workspace_bytes,
                        void* hip_stream);

/* Allocation-free variant of rn18op_conv2d_wgrad, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid allocation): the same kernels and the same result,
 * with the split-K partial sums in a static device array of the library
 * (rn18op_conv2d_wgrad_noalloc_limit() bytes, 48 MiB; each GPU the library
 * runs on holds its own copy until the process ends) instead of a caller
 * workspace. Nothing is allocated or freed. A shape whose partials need more
 * than the limit returns RN18_EINVAL before any launch (every ResNet-18
 * layer of the library's split rule fits). Every call on one GPU shares that
 * GPU's array: calls that overlap on one GPU (different streams, or
 * different threads on one stream's queue without ordering) race. */
size_t rn18op_conv2d_wgrad_noalloc_limit(void);
int rn18op_conv2d_wgrad_noalloc(int prec, const void* dy, const void* x, float* dw_oihw, int N, int H, int W,
                                int Cin, int cin_real, int Cout, int k, int s, int p, void* hip_stream);

/* Max pool 3x3, stride 2, padding 1 (padding never wins):
 *   y[n,i,j,c] = max over the window; arg[n,i,j,c] = kh*3+kw of the FIRST
 *   maximum in row-major (kh,kw) order (uint8).
 * Backward: dx[n,h,w,c] = sum of dy over the outputs whose argmax is (h,w). */
int rn18op_maxpool_fwd(int prec, const void* x, void* y, uint8_t* arg, int N, int H, int W, int C,
                       void* hip_stream);
int rn18op_maxpool_bwd(int prec, const void* dy, const uint8_t* arg, void* dx, int N, int H, int W, int C,
                       void* hip_stream);

/* fp32 -> bf16 storage rounding exactly as every bf16 kernel stores values:
 * round to nearest, ties to even (binary32 -> bfloat16; a NaN stays a NaN).
 * x: n fp32, y: n uint16 bf16 bit patterns, n a multiple of 8, 16-byte
 * aligned device pointers. The oracle's rounding points assume this rule. */
int rn18op_round_bf16(const float* x, uint16_t* y, size_t n, void* hip_stream);

/* ---- Row operators -------------------------------------------------------
 * Layer norm, RMS norm, dropout, a teacher's top logits and the distillation
 * loss work on R rows of a matrix whose rows are `ld` elements apart (ld >=
 * the width; any ld, any width from 1 to 2^30). Their tensors of the storage
 * type need only the alignment of one element, their fp32 and int32 arrays
 * that of 4 bytes; rows may be of any number whose tensors span at most 2^46
 * elements, R = 0 included. `prec` may be RN18_FP16 too. Sums, statistics and
 * the loss are fp32 or wider, and what is stored in 16 bits is rounded once,
 * to nearest even. An output of the storage type may be an input itself (the
 * same pointer and row stride); tensors must not overlap otherwise. Results
 * do not depend on the order in which blocks run: the same inputs give the
 * same bits. A workspace is scratch of one call (16-byte aligned, NULL where
 * 0 bytes are needed): calls that may overlap need one each. RN18_ENOMEM if
 * it is too small. */

/* Layer norm over the D channels of each row (one pixel of an NHWC tensor):
 *   mean = sum x / D,  rstd = 1 / sqrt(sum (x - mean)^2 / D + eps),
 *   y = (x - mean) * rstd * gamma + beta
 * gamma, beta fp32 [D] (NULL: 1 and 0); mean, rstd fp32 [R], kept for the
 * backward pass (NULL in inference). A row that holds a NaN or an infinity
 * gives NaN. The sums are fp32's: where the squares of x - mean pass its range
 * (from 1.8e19 on) rstd is 0, and where a row's sum does the row is NaN. */
int rn18op_layernorm_fwd(int prec, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                         float* rstd, int64_t R, int D, int64_t ldx, int64_t ldy, float eps, void* hip_stream);

/* Its backward pass, from the forward pass's input and statistics:
 *   g = dy * gamma, xh = (x - mean) * rstd,
 *   dx = rstd * (g - sum g / D - xh * sum(g * xh) / D),
 *   dgamma = sum over rows of dy * xh, dbeta = sum over rows of dy
 * dgamma, dbeta fp32 [D], overwritten (zeros for R = 0; either may be NULL,
 * and without both no workspace is needed). dx may be dy or x itself. */
size_t rn18op_layernorm_bwd_workspace(int prec, int64_t R, int D);
int rn18op_layernorm_bwd(int prec, const void* dy, const void* x, const float* gamma, const float* mean,
                         const float* rstd, void* dx, float* dgamma, float* dbeta, int64_t R, int D, int64_t lddy,
                         int64_t ldx, int64_t lddx, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Dropout of the rows of x, with a residual's addition:
 *   y = res + m x,  m = keep / (1 - p)
 * keep(r, j) iff (w >> 8) >= floor(p 2^24), w = word j mod 4 of Philox4x32-10
 * (Salmon et al., SC'11) with key (seed mod 2^32, seed div 2^32) and counter
 * (q mod 2^32, q div 2^32, t mod 2^32, t div 2^32), q = r ceil(D/4) + j div 4,
 * t = step + *step_add mod 2^64, and kept elements are multiplied by
 * (float)(1 / (1 - p)): rn18_set_dropout's mask where D is a multiple of 4.
 * No mask is stored: the gradient of x is the same call on dy without res,
 * that of res is dy. What is dropped is 0 whatever x holds there. res may be
 * NULL; p in [0, 1). step_add (NULL: 0) points to a 64-bit count on the
 * device that is read when the kernel runs, so that a replayed graph takes
 * the step that stands there then. y may be x or res itself. */
int rn18op_dropout(int prec, const void* x, const void* res, void* y, int64_t R, int D, int64_t ldx, int64_t ldres,
                   int64_t ldy, float p, uint64_t seed, uint64_t step, const uint64_t* step_add, void* hip_stream);

/* Root-mean-square norm over the D elements of each row, with the branch's
 * dropout and the residual's addition in the same pass:
 *   h = res + m x (m as above, 1 for p = 0; rounded to the storage type),
 *   rstd = 1 / sqrt(sum h^2 / D + eps),  y = h rstd gamma
 * h is written for the residual stream and the backward pass; the norm takes
 * it as it is stored. res may be NULL (0), gamma fp32 [D] too (1), rstd fp32
 * [R] too (in inference); h may be NULL where it would be x itself (no res,
 * p = 0). h and y may each be x or res, but not the same. The sum of squares
 * is fp32's: beyond its range (elements from 1.8e19 on) rstd is 0, and below it
 * (for eps = 0 a row of elements below 1e-19 alone) inexact or infinite; a row
 * that holds a NaN gives NaN, and one that holds an infinity NaN there and 0
 * elsewhere. */
int rn18op_rmsnorm_fwd(int prec, const void* x, const void* res, const float* gamma, void* h, void* y, float* rstd,
                       int64_t R, int D, int64_t ldx, int64_t ldres, int64_t ldh, int64_t ldy, float eps, float p,
                       uint64_t seed, uint64_t step, const uint64_t* step_add, void* hip_stream);

/* The same with y in 8 bits (OCP e4m3, one byte an element, rows ldy8 bytes
 * apart) and a scale a row, for products in 8 bits:
 *   a = max(max_j |y_j|, 1e-30),  scale = a / 448,  y8 = e4m3(y / scale)
 * to nearest even, y in fp32. A row with a NaN in y has a NaN scale and NaN
 * codes. scale fp32 [R]; y8 overlaps no other tensor. */
int rn18op_rmsnorm_fwd_q8(int prec, const void* x, const void* res, const float* gamma, void* h, uint8_t* y8,
                          float* scale, float* rstd, int64_t R, int D, int64_t ldx, int64_t ldres, int64_t ldh,
                          int64_t ldy8, float eps, float p, uint64_t seed, uint64_t step, const uint64_t* step_add,
                          void* hip_stream);

/* Its backward pass, from the stored h and rstd:
 *   g = dy gamma, xh = h rstd,
 *   dh = rstd (g - xh sum(g xh) / D) + dr,  dx = m dh,
 *   dgamma = sum over rows of dy xh
 * dr is the gradient that h receives from the residual stream behind it
 * (NULL: none); dh is the gradient of res, dx that of x: equal for p = 0, and
 * either may be NULL. dgamma fp32 [D], overwritten (zeros for R = 0; NULL: not
 * wanted, and no workspace needed). dh and dx may each be dy, dr or h, but
 * not the same. p, seed and step as in the forward pass. */
size_t rn18op_rmsnorm_bwd_workspace(int prec, int64_t R, int D);
int rn18op_rmsnorm_bwd(int prec, const void* dy, const void* dr, const void* h, const float* gamma, const float* rstd,
                       void* dh, void* dx, float* dgamma, int64_t R, int D, int64_t lddy, int64_t lddr, int64_t ldh,
                       int64_t lddh, int64_t lddx, float p, uint64_t seed, uint64_t step, const uint64_t* step_add,
                       void* workspace, size_t workspace_bytes, void* hip_stream);

/* The K largest of the C logits of each row, 1 <= K <= min(C, 256):
 *   vals fp32 [R][K] in descending order, idx int32 [R][K] their classes
 * Equal values (the two zeros are equal) go in the order of their classes; a
 * NaN is larger than every number. What a teacher keeps of its logits. */
size_t rn18op_topk_logits_workspace(int prec, int64_t R, int C, int K);
int rn18op_topk_logits(int prec, const void* z, float* vals, int32_t* idx, int64_t R, int C, int64_t ldz, int K,
                       void* workspace, size_t workspace_bytes, void* hip_stream);

/* Distillation from a teacher's top logits, with the labels' cross-entropy,
 * and the gradient of the student's logits z [R][C]:
 *   P = softmax(z / T), p = softmax(z), q = softmax of t_vals / T over the
 *   row's valid entries (0 <= t_idx < C and t_vals not -inf)
 *   row_loss = w * (alpha T^2 sum_k q_k (log q_k - log P[t_idx_k])
 *                   + (1 - alpha) (-log p[label]))
 *   loss = scale * sum of row_loss
 *   dz_j = scale * w * (alpha T (P_j - sum of q_k with t_idx_k = j)
 *                       + (1 - alpha) (p_j - [j = label]))
 * t_vals fp32, t_idx int32 [R][K], 0 <= K <= 256 (K = 0: both may be NULL), in
 * any order; an entry that is not valid is left out (a short list is filled
 * with t_idx = -1), and entries of one class add up. Terms with q_k = 0 are 0.
 * alpha = 0 leaves out the soft term and alpha = 1 the hard one, whatever
 * their inputs hold; otherwise a valid entry of NaN or +inf makes its row's
 * loss and the gradient of the row's listed classes NaN (the other classes'
 * gradient needs the student's logits alone and stays a number). A listed
 * class that the student masks has an infinite loss, and a loss beyond fp32
 * is infinite. A row without a valid entry has no soft term; one whose label
 * is outside [0, C) (-1, say; labels NULL: every row) has no hard term; a row
 * whose logits are all -inf (every class masked) has neither. Masked classes
 * hold -inf and get a zero gradient. w: row_weight fp32 [R] (NULL: 1); a row of
 * weight 0 has loss 0 and gradient 0 whatever its logits hold.
 * row_loss fp32 [R]; loss 1 fp32 (may be NULL); dz as z (NULL: no gradient;
 * may be z itself). temperature positive and finite, from 4.24e-39 on (log2(e)
 * over it is finite), alpha in [0, 1], scale finite (1/R for the batch's mean,
 * times a loss scale in fp16). */
size_t rn18op_distill_loss_workspace(int prec, int64_t R, int C, int K);
int rn18op_distill_loss(int prec, const void* z, const float* t_vals, const int32_t* t_idx, const int32_t* labels,
                        const float* row_weight, void* dz, float* row_loss, float* loss, int64_t R, int C,
                        int64_t ldz, int64_t lddz, int K, float temperature, float alpha, float scale,
                        void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- Linear attention with a decay for each head ---------------------------
 * A causal mixer of the tokens of B sequences of up to T tokens, H query
 * heads over Hk key and value heads (H a multiple of Hk; query head h reads
 * key head h div (H / Hk)), a state S of Dk x Dv for each sequence and query
 * head:
 *   S_t = exp(g_h) S_(t-1) + k_t v_t^T,   o_t = scale S_t^T q_t
 * q [B T][H Dk], k [B T][Hk Dk], v [B T][Hk Dv], o [B T][H Dv]: token t of
 * sequence b is row b T + t, rows are ld elements apart (any ld from the
 * width on; elements need only their own alignment, so that all may be parts
 * of one buffer). log_decay fp32 [H]: g, a constant of the model that no
 * gradient is taken of; -infinity is a head without memory, and g above 0 a
 * growing one: up to 2.5 its results are right as long as they and the states
 * are in fp32's range, beyond, where the powers of 32 tokens leave it, some may
 * be infinite or NaN instead (a single token's: beyond 88). lengths int32 [B]
 * on the device (NULL: all T; values are taken into [0, T]): tokens from a
 * sequence's length on are neither read nor written. States are fp32 [B][H][Dk][Dv], dense: s0 before the first token
 * (NULL: zeros), sT after the last (NULL: not wanted; may be s0 itself). Dk
 * and Dv from 1 to 256, B T H up to 2^31 - 1, B H up to 2^20, T up to 2^26.
 * Sums and states are fp32; the products of 16-bit types keep the decayed and
 * summed operands in parts of 8 bits that add up to 16 bits or more, and o is
 * rounded once. A NaN or an infinity changes nothing before its token; from
 * there on it may make a sequence's head NaN, but one in v, or in the state, only
 * its column. Outputs overlap no input but for sT. Results do not depend on the
 * order in which blocks run. Workspaces are those of the row operators. */
size_t rn18op_linattn_fwd_workspace(int prec, int B, int T, int H, int Hk, int Dk, int Dv);
int rn18op_linattn_fwd(int prec, const void* q, const void* k, const void* v, const float* log_decay,
                       const int32_t* lengths, const float* s0, void* o, float* sT, int B, int T, int H, int Hk, int Dk,
                       int Dv, int64_t ldq, int64_t ldk, int64_t ldv, int64_t ldo, float scale, void* workspace,
                       size_t workspace_bytes, void* hip_stream);

/* Its backward pass, from the forward pass's inputs (dO is `dout`, dS_T the
 * gradient of sT, NULL: zeros):
 *   S_t as above,  dq_t = scale S_t dO_t,
 *   G_t = exp(g) G_(t+1) + scale q_t dO_t^T,  exp(g) G_(length) = dS_T
 *   dk_t = G_t v_t,  dv_t = G_t^T k_t,  ds0 = exp(g) G_0
 * dk and dv are added up over the query heads that share a key head (in 64 bits).
 * ds0 may be NULL, or dS_T itself. */
size_t rn18op_linattn_bwd_workspace(int prec, int B, int T, int H, int Hk, int Dk, int Dv);
int rn18op_linattn_bwd(int prec, const void* q, const void* k, const void* v, const void* dout,
                       const float* log_decay, const int32_t* lengths, const float* s0, const float* dsT, void* dq,
                       void* dk, void* dv, float* ds0, int B, int T, int H, int Hk, int Dk, int Dv, int64_t ldq,
                       int64_t ldk, int64_t ldv, int64_t lddout, int64_t lddq, int64_t lddk, int64_t lddv, float scale,
                       void* workspace, size_t workspace_bytes, void* hip_stream);

/* One token of each of B sequences, for serving: rows are the sequences.
 * state_out [B][H][Dk][Dv] may be state_in itself. */
int rn18op_linattn_step(int prec, const void* q, const void* k, const void* v, const float* log_decay,
                        const float* state_in, void* o, float* state_out, int B, int H, int Hk, int Dk, int Dv,
                        int64_t ldq, int64_t ldk, int64_t ldv, int64_t ldo, float scale, void* hip_stream);

/* Debugging aids (not part of the training path).
 * rn18_debug_set(ctx, RN18_DBG_STOP_BLOCKS, k): later train steps end their
 * backward pass after k residual blocks (no stem backward, no SGD update);
 * k = -1 restores full steps.
 * rn18_debug_copy: copy `bytes` of a workspace tensor of the (N,H,W) plan to
 * the device buffer dst, enqueued on the context's stream. `which` selects
 * the tensor (NHWC in the compute type, or fp32 for grad/mean/rstd),
 * `index` the conv layer (forward order) or the residual block. The
 * backward buffers hold what the last step left there: GA / GB the
 * gradients of block outputs (ping-pong), GZ the data gradient of a block's
 * second conv, GY the stem conv's dY, GYD a projection conv's dY. */
enum {
  RN18_DBG_STOP_BLOCKS = 0,
  /* process-wide: force gather-conv kernel configuration `value` (1..45,
   * see conv.hip) for every forward / data-gradient launch; 0 = automatic.
   * ctx may be NULL for this key. For tuning and for testing every
   * configuration. */
  RN18_DBG_GATHER_CONFIG = 1,
  /* process-wide: force weight-gradient kernel configuration `value`
   * (1..10, see conv.hip); 0 = automatic. Plans built afterwards size their
   * split-K scratch for it. ctx may be NULL. */
  RN18_DBG_WGRAD_CONFIG = 2,
  /* per context: launch each convolution of a training step or eval pass
   * over batch chunks of at most `value` images (0 = only where a tensor
   * would exceed the kernels' 32-bit byte offsets). Plans built before are
   * dropped. For testing the chunked path at small sizes. */
  RN18_DBG_CONV_CHUNK = 3,
  /* per context: value != 0 keeps every launch of a training step on the
   * caller's stream (the weight gradients otherwise run on a second stream
   * beside the data-gradient chain). For timing kernels one at a time. */
  RN18_DBG_SERIAL = 4,
  /* process-wide: split count of the K reduction of every forward and
   * stride-1 data-gradient gather launch of a training step or eval pass
   * (at most the launch's K stages, at most 64; 0 = automatic: only
   * launches with fewer output tiles than the chip has compute units
   * split; 1 = never). Plans built afterwards size their split-K scratch
   * for it. ctx may be NULL. For tuning and for testing the split path. */
  RN18_DBG_GATHER_SPLIT = 5
};
enum {
  RN18_DBG_Y = 0, RN18_DBG_Z1 = 1, RN18_DBG_OUT = 2, RN18_DBG_GA = 3, RN18_DBG_GB = 4, RN18_DBG_GZ = 5,
  RN18_DBG_GY = 6, RN18_DBG_GYD = 7, RN18_DBG_GRAD = 8, RN18_DBG_WF = 9, RN18_DBG_WD = 10,
  RN18_DBG_MEAN = 11, RN18_DBG_RSTD = 12, RN18_DBG_ZSTEM = 13, RN18_DBG_PARG = 14
};
/* rn18_debug_capture(ctx, kind, index, dst, bytes): during later train
 * steps, copy a backward-pass tensor to dst as soon as it is produced:
 * RN18_CAP_DY (index = conv layer: the gradient entering its conv),
 * RN18_CAP_DZ1 (block: data gradient of its second conv), RN18_CAP_DX
 * (block: gradient wrt the block input; in a projection block the data
 * gradients of the first conv and of the projection are summed in one GEMM
 * and rounded once), RN18_CAP_DA_AVG (gradient entering
 * the last block from the average pool), RN18_CAP_DA_POOL (max-pool data
 * gradient). dst = NULL clears every capture. */
enum {
  RN18_CAP_DY = 0, RN18_CAP_DZ1 = 1, RN18_CAP_DX = 3, RN18_CAP_DA_AVG = 4, RN18_CAP_DA_POOL = 5
};
int rn18_debug_capture(struct rn18_ctx* ctx, int kind, int index, void* dst, size_t bytes);
int rn18_debug_set(struct rn18_ctx* ctx, int key, long value);
int rn18_debug_copy(struct rn18_ctx* ctx, int N, int H, int W, int which, int index, void* dst, size_t bytes);

#ifdef __cplusplus
}
#endif
#endif
