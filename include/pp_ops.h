/* pp_ops.h -- op-level entry points of the same library: the dense contractions of the local step and the losses of its output head, callable
 * on their own so that each kernel can be checked against a plain definition and timed against its roofline.
 * All pointers are device pointers owned by the caller; all calls only enqueue work on `hip_stream`.
 * dtype: PP_F32 or PP_BF16 storage (see pp.h).  Return PP_OK or a negative PP_E* code (pp_last_error()).
 */
#ifndef PP_OPS_H
#define PP_OPS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* C[M x N] = A[M x K] * B[N x K]^T (+ R[M x N] if R != NULL), row-major with leading dimensions lda, ldb, ldc
 * (R uses ldc).  Every matmul of the forward pass and of the partial backward (Appendix "Partial Backward":
 * dA = V_n^T G, dX = sum_n W_n^T dH_n, dW_n = dH_n X^T, dV_n = G A_n^T) is issued in this form.
 * out_f32 != 0: C is float (weight gradients); then R must be NULL.
 * splits > 1 (needs out_f32, scratch_dev of M*N*splits floats): K is cut into `splits` equal ranges whose
 * partial products are summed in fixed order into C.
 * path: 0 = automatic (bf16 MFMA kernels when dtype is bf16 and K % 64 == 0, lda % 8 == 0, ldb % 8 == 0, otherwise the fp32-multiply
 * MFMA kernel, which returns the plain kernel's bits), 1 = plain (vector FMA) kernel. */
int pp_op_gemm_nt(void* hip_stream, int dtype, const void* A_dev, int lda, const void* B_dev, int ldb, void* C_dev, int ldc,
                  int M, int N, int K, const void* R_dev, int out_f32, int splits, float* scratch_dev, int path);

/* The weight-gradient contraction in the layout the step has it in (Appendix "Partial Backward": dW_n = dH_n X^T,
 * dV_n = G A_n^T, with tokens as the contraction index): C[M x N] (float, ldc) = A^T B, A: [K x .] and B: [K x N] row-major
 * bf16 with leading dimensions lda, ldb -- both token-major, no transposed copies.  Column m of the product is column
 * (m / m_blk) * a_blk_stride + m % m_blk of A (m_blk = M, a_blk_stride = 0 for one contiguous column range).
 * splits > 1 (scratch_dev of M*N*splits floats): K is cut into at most `splits` equal ranges (fewer when those fill the GPU)
 * whose partial products are summed in fixed order.  MFMA kernel only (bf16): needs M, N, lda, ldb, m_blk, a_blk_stride multiples of 8, K a multiple of
 * 64*splits, and m_blk a multiple of 128 when M > m_blk; other shapes return PP_EINVAL (pp_local_step itself runs the kernel for any token
 * count and column blocks of any multiple of 8, in ranges of its own, and goes through transposed copies for the rest). */
int pp_op_gemm_tn(void* hip_stream, const void* A_dev, int lda, int m_blk, int64_t a_blk_stride, const void* B_dev, int ldb, float* C_dev,
                  int ldc, int M, int N, int K, int splits, float* scratch_dev);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc): the split-K form of pp_op_gemm_nt with fp32 output, C[M x N] (ldc) = A[M x K] * B[N x K]^T, whose
 * partial products [splits][M][N] live in a 16 MiB device array built into the library instead of a caller's scratch
 * buffer.  Same kernels, same summation order and therefore the same bits as pp_op_gemm_nt(..., out_f32 = 1, splits,
 * scratch, path).  Requirements: splits >= 2, K % splits == 0, M*N*splits <= PP_STATIC_SCRATCH_FLOATS, else PP_EINVAL
 * with a message that names the limit.  Calls no hipMalloc / hipFree and nothing that allocates; only enqueues on
 * hip_stream.  The first call on a GPU also looks up that GPU's address of the array (the HIP runtime materialises a
 * module's device variables at that moment: make one call per GPU before entering a region that must not allocate).
 * Every call on one GPU uses that GPU's one array (it keeps the previous call's partials; each call overwrites all it
 * reads): calls that overlap on one GPU -- different streams or threads -- race; calls on one stream are ordered and
 * safe.  Each GPU the library runs on holds its own 16 MiB until process exit. */
#define PP_STATIC_SCRATCH_FLOATS (4u << 20)
int pp_op_gemm_nt_splitk_static(void* hip_stream, int dtype, const void* A_dev, int lda, const void* B_dev, int ldb, float* C_dev,
                                int ldc, int M, int N, int K, int splits, int path);

/* Causal softmax attention (Appendix "MHA with frozen heads", forward of every head; mask from the autoregressive
 * factorisation of Section 2.1).  qkv_dev: [B*S x 3*h*dh], columns q | k | v, head j at columns j*dh of each part
 * (q and k already rotated).  o_dev: [B*S x h*dh].  lse_dev: float [B*h*S], log-sum-exp of the scaled scores.
 * scratch_dev: not used (the matrix-core kernels read q, k, v as stored); kept in the signature, may be NULL.
 * path: 0 = automatic (bf16 MFMA kernels for bf16 with dh 64 or 128; otherwise, where there are rows enough for them, the fp32-multiply
 * MFMA kernels for dh 16, 32, 64, 128 -- forward up to 1184 positions --, which return the plain kernels' bits), 1 = plain kernels. */
int pp_op_attention_fwd(void* hip_stream, int dtype, const void* qkv_dev, void* o_dev, float* lse_dev, void* scratch_dev,
                        int B, int S, int h, int dh, int path);

/* Backward of the above for all heads: dqkv_dev [B*S x 3*h*dh] receives dq | dk | dv (in the rotated frame);
 * D_dev: float [B*h*S], receives the row sums of dO * O.  scratch_dev: not used, may be NULL. */
int pp_op_attention_bwd(void* hip_stream, int dtype, const void* qkv_dev, const void* o_dev, const float* lse_dev, const void* dO_dev,
                        void* dqkv_dev, float* D_dev, void* scratch_dev, int B, int S, int h, int dh, int path);

/* ---- Losses of the output head over a large vocabulary, without the logits being kept.
 *
 * z = X W^T for hidden states X [n x d] and head weights W [vocab x d] (row-major, ldx and ldw elements apart); z exists a piece of rows
 * at a time, in the workspace, and never as a whole.  One call forms the losses and, where asked for, the gradients
 *   dX = dz W [n x d]   and   dW = dz^T X for the rows [dw_lo, dw_hi) of W
 * of   loss = sum_t w_t l_t,   w_t = row_weight[t], or 1 / (number of rows that are not left out) where row_weight is NULL (the mean, as in pp_local_step).
 *   pp_op_head_ce       l_t = lse(z_t) - z_t[target]; a row whose target is outside [0, vocab) is left out.
 *   pp_op_head_distill  l_t = (1 - share) CE_t + share temperature^2 D_t with CE_t as above and, over the entries (id_j, logit_j) of the `top` that the teacher lists for the row,
 *                         D_t = sum_j q_j (log q_j - log p[id_j]),   q = softmax(logits / temperature) over the entries,   p = softmax(z_t / temperature) over the vocabulary:
 *                       KL(q || p) of a list of different ids.  An id that is listed more than once stands for the sum of its entries in the gradients, which are those of that divergence; in
 *                       D_t each entry keeps its own logarithm, so that D_t is lower than the divergence by sum_j q_j log(Q_j / q_j), Q_j the sum of the entries with id_j (it does not depend on
 *                       z, and D_t may be negative: merge the entries first where the value has to be a divergence).
 *                       An id outside [0, vocab) or a logit of -inf is no entry, whatever its other half holds.  A row without entries has no D_t, a row without target no CE term, a row
 *                       without either (terms with a share of 0 do not count) is left out.
 * A row of weight 0 is left out too.  Rows that are left out have row_loss = row_lse = 0 and a dX row of zeros, and neither their values nor infinities or NaN among them reach
 * anything else.  n == 0 gives loss 0 and dW = 0.
 * Sums, exponentials and losses are fp32.  With bf16 storage and more than 16 rows, a row of dz enters the gradients' products as a multiple of a row that is rounded to
 * bf16 (at most 2^-8 relative), its multiple moved by at most 2^-8 so that the largest element is not rounded; the rows of X are scaled by the multiple and rounded to bf16 for dW.  Where both
 * softmaxes count at a temperature other than 1 they are formed from the sharper one's exponent y (of two, against a reference no larger than the row's maximum), rounded to steps of 2^-8 down to
 * y = -64 and of 2^-4 below, and taken as nothing below -2096: another 2^-9 ln 2, below -64 2^-5 ln 2, of the sharper part of an element and that over the ratio of the temperatures of the softer
 * part.  Weights below 2^-100 in size may lose bits there.  dX and dW are rounded once from fp32 sums.  Results do not depend on the run. */
#define PP_HEAD_TOP_MAX 128
typedef struct {
  const void *x, *w;               /* storage type dtype */
  const float* row_weight;         /* [n] or NULL */
  float* loss;                     /* [1] or NULL */
  float *row_loss, *row_lse;       /* [n] or NULL: l_t; log-sum-exp of z_t / temperature (pp_op_head_ce and share 0: of z_t).  None of the three may overlap an input. */
  void *dx, *dw;                   /* dx [n x d], storage type, or NULL; dw [(dw_hi - dw_lo) x d], or NULL if dw_lo == dw_hi.  Neither may
                                      overlap another operand (column ranges of one buffer do not). */
  int32_t ldx, ldw, lddx, lddw;    /* elements from row to row, >= d (lddx, lddw: where dx, dw are given) */
  int32_t dtype, n, vocab, d;      /* PP_F32 or PP_BF16; n <= 2^24, vocab <= 2^20, d <= 2^14 */
  int32_t dw_lo, dw_hi;            /* 0 <= dw_lo <= dw_hi <= vocab; row 0 of dw is row dw_lo of W */
  int32_t dw_f32;                  /* 0: dw in storage type; 1: dw float; 2: dw float, and the gradient is added to what it holds */
  int32_t piece;                   /* rows of a piece, rounded up to a multiple of 64 and at most as many as keep a piece's buffer within 2 GiB (256 rows in any case);
                                      0: as many as keep it within 512 MiB, or within the size of dW's float sums, up to 1 GiB, where that is larger */
} pp_head;
/* Workspace of a call with these sizes, options and operand alignment (top: entries per row, 0 for pp_op_head_ce); 0 and an error text on invalid arguments. */
size_t pp_op_head_bytes(const pp_head* head, int32_t top);
/* targets_dev: int32 [n].  ws_dev: 256-byte aligned, ws_bytes >= pp_op_head_bytes; it may overlap no operand; the content does not matter and is not kept.
 * Calls that overlap in time need a workspace each. */
int pp_op_head_ce(void* hip_stream, const pp_head* head, const int32_t* targets_dev, void* ws_dev, size_t ws_bytes);
/* ids_dev: int32 [n x top], logits_dev: float [n x top], 1 <= top <= PP_HEAD_TOP_MAX; temperature in [2^-6, 2^6]; share in [0, 1]; targets_dev may be NULL if share == 1. */
int pp_op_head_distill(void* hip_stream, const pp_head* head, const int32_t* ids_dev, const float* logits_dev, int32_t top, float temperature, float share,
                       const int32_t* targets_dev, void* ws_dev, size_t ws_bytes);

#ifdef __cplusplus
}
#endif
#endif /* PP_OPS_H */
