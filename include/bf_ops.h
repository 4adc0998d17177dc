/*
 * libbf — the single kernels of the transformer layer (App. A.1 of arXiv 2211.05953:
 * self-attention with N_heads heads of size S_head followed by a two-layer MLP), exported
 * one by one so that each can be checked against the CPU oracle and timed on its own.
 * bf_run_step (bf.h) chains exactly these.
 *
 * All tensor pointers are device pointers; row-major; `dtype` is a bf_dtype and names the
 * storage type of activations and weights (bf16 or fp32; accumulation is always fp32).
 * bias / LayerNorm parameters / statistics / lse / main-grads are fp32.
 * `kernels` is a bf_kernels value.  `stream` is a hipStream_t (NULL = default stream);
 * every call is asynchronous on it.  Nothing is allocated; the caller owns every buffer.
 * Errors: BF_EINVAL for bad sizes / null pointers / unknown enums, BF_EDEVICE if the
 * launch fails; bf_last_error() has the text.
 */
#ifndef BF_OPS_H
#define BF_OPS_H

#include "bf.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Operand layouts of the three linear-layer products (8 flop per parameter and token in
 * total, App. A.1):
 *   BF_NN  forward  C[M,N] = A[M,K] B[K,N]
 *   BF_NT  dgrad    C[M,N] = A[M,K] Bt[N,K]^T          (B passed as [N,K])
 *   BF_TN  wgrad    C[M,N] = At[K,M]^T B[K,N]          (A passed as [K,M]; C is fp32) */
typedef enum { BF_NN = 0, BF_NT = 1, BF_TN = 2 } bf_layout;

/* What happens to the fp32 accumulator acc[m,n] before it is stored:
 *   BF_EPI_NONE       C = acc
 *   BF_EPI_BIAS       C = acc + bias[n]
 *   BF_EPI_BIAS_RES   C = acc + bias[n] + R[m,n]
 *   BF_EPI_BIAS_GELU  C = acc + bias[n] (rounded to dtype), C2 = gelu_tanh(C)
 *   BF_EPI_GELU_BWD   C = acc * gelu_tanh'(R[m,n])
 *   BF_EPI_ACCUM      fp32 C = (accumulate ? C : 0) + acc        (main-grad accumulation) */
typedef enum { BF_EPI_NONE = 0, BF_EPI_BIAS = 1, BF_EPI_BIAS_RES = 2, BF_EPI_BIAS_GELU = 3,
               BF_EPI_GELU_BWD = 4, BF_EPI_ACCUM = 5 } bf_epilogue;

bf_status bf_op_gemm(int dtype, int kernels, int layout, int epilogue, int M, int N, int K,
                     const void* A, const void* B, void* C, const float* bias, const void* R, void* C2,
                     int accumulate, void* stream);
/* The dgrad product in front of a GeLU with the bias gradient of the linear layer below it (App. A.1: the first
 * linear layer of the MLP) taken on the way:
 *   C[M,N] = (A[M,K] Bt[N,K]^T) * gelu_tanh'(R[M,N])            (BF_NT with BF_EPI_GELU_BWD)
 *   db[N]  = (accumulate ? db : 0) + sum_m C[m,:]                of the stored (rounded) C
 * part: device fp32 scratch of ceil(M / 128) * N elements, owned by the caller: with it the MFMA kernel takes the
 * sums in its epilogue (one row of partial sums per row of tiles, added up in a fixed order by a small kernel);
 * NULL, a product of few tiles (see bf_op_gemm_tile) or one that goes to another kernel: a second pass over C takes
 * them and the scratch is left alone.  db: device fp32 [N]. */
bf_status bf_op_gemm_gelu_bwd_colsum(int dtype, int kernels, int M, int N, int K, const void* A, const void* Bt, void* C,
                                     const void* R, float* db, float* part, int accumulate, void* stream);
/* bf_op_gemm for the forward / dgrad layouts (BF_NN, BF_NT; epilogues none, bias, bias + residual) with scratch for a
 * split contraction: a bf16 product on the matrix cores whose tiles would fill at most half of the chip in its only
 * round, with K >= 2048, runs K in bf_op_gemm_splitk_slices(...) slices on that many times the workgroups; each slice
 * leaves an fp32 plane in `planes` (device, slices * M * N floats, owned by the caller) and a second kernel adds the
 * planes in ascending order and applies the epilogue, so the result does not depend on the order the slices finish
 * in.  Any other shape, dtype or kernel choice, planes == NULL or planes_elems too small: exactly bf_op_gemm. */
bf_status bf_op_gemm_splitk(int dtype, int kernels, int layout, int epilogue, int M, int N, int K, const void* A,
                            const void* B, void* C, const float* bias, const void* R, float* planes,
                            size_t planes_elems, void* stream);
/* Slices that call uses for this shape, given the scratch for them (1: the contraction is not split). */
int bf_op_gemm_splitk_slices(int layout, int epilogue, int M, int N, int K);
/* 1 if the problem is whole tiles of the bf16 MFMA kernel (M and N multiples of 128, K of 64), 0 if not: not whether
 * matrix cores serve it.  Other bf16 problems run on the same kernel with partly empty tiles where their rows are whole
 * 16-byte chunks (N % 8 == 0, and K % 8 == 0 or, weight gradient, M % 8 == 0), and where they are not on the fp32
 * matrix instructions or, a short contraction into a large output, on the plain kernel, whichever is faster. */
int bf_op_gemm_uses_mfma(int layout, int epilogue, int M, int N, int K);
/* The tile of C (rows x columns per workgroup) that the MFMA kernel runs an unsplit product of this shape on by itself:
 * 256 x 256, 256 x 128, 128 x 128, or 256 x 192 (forward and dgrad layouts with the epilogues none, bias, bias + residual
 * and N a multiple of 192, where that fills the rounds of the grid better: 2048 x 6144 outputs are 256 such tiles).  A
 * step that runs two chains of micro-batches does not take the last shape.  Not what every call runs on: products of few
 * tiles (at most 512 of 64 x 64, weight gradients 256) run on 64 x 64 ones instead, and weight gradients with an odd
 * multiple of 128 on partly empty 256 x 256 ones where that is faster; the shape given is the whole tile they would
 * otherwise take.  Host arithmetic only.  Returns 1 and the tile in tile_m / tile_n (host ints), or 0 (and 0 x 0) where
 * bf_op_gemm_uses_mfma is 0. */
int bf_op_gemm_tile(int layout, int epilogue, int M, int N, int K, int* tile_m, int* tile_n);

/* Weight and bias gradient of one linear layer over all the micro-batches of a stage in one
 * product (breadth-first order: every micro-batch of the stage has been through its backward
 * before the gradient is needed, Sec. 4.2; fp32 main-grads, App. D):
 *   G[M,N]  = (accumulate ? G  : 0) + sum_{i < n_seg} X_i[K,M]^T dY_i[K,N]
 *   db[N]   = (accumulate ? db : 0) + sum_{i < n_seg} sum_k dY_i[k,:]          (db may be NULL)
 * X_i = X + i * stride_x and dY_i = dY + i * stride_dy (strides in elements; the bf16 MFMA kernel takes
 * segments that are 16-byte aligned, others run on the fp32 matrix instructions), both in the activation dtype, device
 * memory; G and db fp32, device memory, owned by the caller.  BF_EINVAL for bad sizes, null X / dY / G or n_seg < 1. */
bf_status bf_op_wgrad(int dtype, int kernels, int M, int N, int K, int n_seg, const void* X, size_t stride_x,
                      const void* dY, size_t stride_dy, float* G, float* db, int accumulate, void* stream);

/* y = (x - mean) * rstd * g + b per row of x[T,h]; stats[T][2] = (mean, rstd), rstd = 1/sqrt(var + eps). */
bf_status bf_op_layernorm_fwd(int dtype, int T, int h, const void* x, const float* g, const float* b, float eps,
                              void* y, float* stats, void* stream);
/* dx[T,h] = LN'(dy) (+ dres if non-null); dg[h], db[h] (fp32) = or += the column sums. */
bf_status bf_op_layernorm_bwd(int dtype, int T, int h, const void* dy, const void* x, const float* g,
                              const float* stats, const void* dres, void* dx, float* dg, float* db,
                              int accumulate, void* stream);
/* The same with everything a LayerNorm needs in the backward pass taken in one pass over dy and x:
 * dx as above; dg, db as above; dcs[h] (fp32, may be NULL) = or += the column sums of the stored dx, which are the bias
 * gradient of the linear layer that produced x (x = residual + linear output).
 * part: device fp32 scratch of bf_op_layernorm_bwd_part_elems(T, h) elements, owned by the caller: with it (and h a
 * multiple of the vector width, at most 4 x 256 vectors per row) a workgroup walks a run of rows with its column sums in
 * registers and a second small kernel adds the workgroups' partial sums in a fixed order; NULL: separate passes. */
bf_status bf_op_layernorm_bwd_fused(int dtype, int T, int h, const void* dy, const void* x, const float* g,
                                    const float* stats, const void* dres, void* dx, float* dg, float* db, float* dcs,
                                    float* part, int accumulate, void* stream);
size_t bf_op_layernorm_bwd_part_elems(int T, int h);
/* out[N] (fp32) = or += sum over rows of dY[T,N]: the bias gradient. */
bf_status bf_op_colsum(int dtype, int T, int N, const void* dY, float* out, int accumulate, void* stream);

/* Multi-head attention.  qkv [S_mb, S_seq, 3 S_hidden] packed [Q | K | V] with head a at
 * columns a*S_head.. of each third; ctx [S_mb, S_seq, S_hidden]; lse [S_mb, N_heads, S_seq] =
 * log-sum-exp of a row's scaled (1/sqrt(S_head)) and masked scores.  causal = 1 masks j > i. */
bf_status bf_op_attention_fwd(int dtype, int kernels, int S_mb, int S_seq, int N_heads, int S_head, int causal,
                              const void* qkv, void* ctx, float* lse, void* stream);
/* dqkv from dctx; delta is fp32 scratch of S_mb * N_heads * S_seq elements. */
bf_status bf_op_attention_bwd(int dtype, int kernels, int S_mb, int S_seq, int N_heads, int S_head, int causal,
                              const void* qkv, const void* ctx, const float* lse, const void* dctx,
                              void* dqkv, float* delta, void* stream);
/* The same with the bias gradient of the QKV projection (App. A.1: qkv = a W_qkv + b_qkv, so the gradient of b_qkv
 * is the column sum of dqkv over the S_mb * S_seq rows): db_qkv[3 S_hidden] (device fp32) = (accumulate ? db_qkv : 0)
 * + those sums.  part: device fp32 scratch of bf_op_attention_bwd_part_elems(...) elements owned by the caller (0
 * elements: not whole blocks of 128 rows of heads of 64 or 128); with it the two backward kernels leave per query / key
 * block partial sums of what they store (before rounding to bf16) and one small kernel adds them in a fixed order;
 * NULL, fp32, or another shape: dqkv is read a second time (bf_op_colsum). */
bf_status bf_op_attention_bwd_bias(int dtype, int kernels, int S_mb, int S_seq, int N_heads, int S_head, int causal,
                                   const void* qkv, const void* ctx, const float* lse, const void* dctx,
                                   void* dqkv, float* delta, float* db_qkv, float* part, int accumulate, void* stream);
size_t bf_op_attention_bwd_part_elems(int S_mb, int S_seq, int N_heads, int S_head);
/* bf_op_attention_bwd for callers that cannot allocate device memory and have no buffer to lend (code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation): the same kernels, with `delta` in an
 * array built into the library (BF_ATTENTION_BWD_STATIC_MAX floats = 4 MiB, which every GPU the library runs on
 * holds until the process ends).  Allocates nothing and calls no allocating routine.  BF_EINVAL if
 * S_mb * N_heads * S_seq exceeds the array.  All calls on one GPU share the array: calls that overlap on one GPU
 * (different streams or threads) race; calls on one stream do not.  Nothing in the array has to be cleared
 * between calls (each call writes every element it reads). */
#define BF_ATTENTION_BWD_STATIC_MAX ((size_t)1 << 20)
bf_status bf_op_attention_bwd_static(int dtype, int kernels, int S_mb, int S_seq, int N_heads, int S_head, int causal,
                                     const void* qkv, const void* ctx, const float* lse, const void* dctx,
                                     void* dqkv, void* stream);
int bf_op_attention_uses_mfma(int S_seq, int S_head);

/* Masked attention here, and below the loss without logits and the clipping of gradients, are for training loops that call single kernels: the
 * stack's own steps (bf.h) take no masks, keep their logits and clip nothing.  No output of these three overlaps an input or another output
 * but where it says so.
 *
 * Attention under masks, with capped scores, a distance bias and shared key / value heads (for sequences that hold several
 * documents).  A row's keys are one interval, its span:
 *   _spans  from doc (device int32 [S_mb, S_seq], or NULL: a sequence is one document): a document is a run of equal ids; its
 *           tokens see that document and nothing else.  A token of a negative id is padding: it sees nothing and no token
 *           sees it.  causal = 1: keys j <= i only, or j < prefix[b] (device int32 [S_mb], or NULL) where that is more; the
 *           first prefix[b] tokens of a sequence are then seen from in front of them too, inside their documents.
 *           spans: device int32, 16-byte aligned, bf_op_attention_spans_elems(S_mb, S_seq) elements (0 for bad sizes): made once, used by
 *           every layer's forward and backward.  S_seq is at most 2^24.
 *   _fwd    ctx = softmax(b) V over each row's span with b_ij = c_ij - slopes[head] |i - j| (slopes: device fp32 [N_heads], or
 *           NULL), c_ij = cap tanh(scale q_i.k_j / cap), or scale q_i.k_j where cap is 0 (any finite cap; bf16 caps past 1024
 *           take a longer tanh).  lse [S_mb, N_heads, S_seq] (device fp32, may
 *           be NULL) = log-sum-exp of a row's b.  A row without keys: ctx 0, lse -infinity.
 *   _bwd    dq, dk, dv from dctx, with the ctx and lse of the forward pass; dk and dv are the sums over the N_heads / N_kv_heads
 *           query heads of a key / value head, head a reading key / value head a / (N_heads / N_kv_heads).  A row
 *           without keys has dq 0 and no part in dk and dv, whatever its q and dctx hold; a row of one key has no part in
 *           dq and dk.  Slopes have no gradient.  work: device scratch, 256-byte aligned, of _bwd_work_bytes(cfg)
 *           bytes (0 for a bad cfg), owned by the caller; calls that overlap need their own.
 * Token t of sequence b starts (b S_seq + t) ld elements into its tensor, head a another a S_head elements on; ld_q, ld_k, ld_v (for
 * q and dq, k and dk, v and dv) and ld_ctx (ctx, dctx) of 0 mean rows without gaps, so that a packed [Q | K | V] is three pointers
 * into it and its row length.  Tensors are aligned to their elements.  Nothing between the rows is written.  What a mask hides never reaches a result, infinities and NaN
 * included.  Sums have a fixed order: no atomics on memory.
 * S_head 1 to 1024, S_mb * N_heads up to 65535, and on the matrix cores times S_seq / 128 under 2^24 (backward 2^23).  S_head up to 128 on the matrix cores (bf16: probabilities and their gradients in bf16 as they enter the products;
 * fp32: fp32 throughout), fastest where rows are whole 16-byte chunks; above, for up to 4 tokens, and with BF_KERNELS_PLAIN, on plain kernels. */
typedef struct {
  int32_t dtype, kernels;                            /* bf_dtype of all tensors but lse and slopes; bf_kernels */
  int32_t S_mb, S_seq, N_heads, N_kv_heads, S_head;  /* N_kv_heads divides N_heads */
  float scale;                                       /* up to 2^126; 0: 1/sqrt(S_head) */
  float cap;                                         /* 0: none */
  int64_t ld_q, ld_k, ld_v, ld_ctx;
} bf_attn_config;
size_t bf_op_attention_spans_elems(int S_mb, int S_seq);
bf_status bf_op_attention_spans(int S_mb, int S_seq, int causal, const int32_t* doc, const int32_t* prefix, int32_t* spans,
                                void* stream);
bf_status bf_op_attention_masked_fwd(const bf_attn_config* cfg, const void* q, const void* k, const void* v,
                                     const int32_t* spans, const float* slopes, void* ctx, float* lse, void* stream);
size_t bf_op_attention_masked_bwd_work_bytes(const bf_attn_config* cfg);
bf_status bf_op_attention_masked_bwd(const bf_attn_config* cfg, const void* q, const void* k, const void* v,
                                     const int32_t* spans, const float* slopes, const void* ctx, const float* lse,
                                     const void* dctx, void* dq, void* dk, void* dv, void* work, size_t work_bytes,
                                     void* stream);

/* Input layer (App. A.1): x[t, :] = e_tok[tokens[t], :] + e_pos[t mod S_seq, :] for n_rows = S_mb * S_seq rows.
 * tokens: device int32 [n_rows]; e_tok [S_voc, S_hidden], e_pos [S_seq, S_hidden] device fp32; x in `dtype`.
 * An id outside 0..S_voc-1 contributes no token row. */
bf_status bf_op_embedding_fwd(int dtype, int n_rows, int S_seq, int S_voc, int S_hidden, const int32_t* tokens,
                              const float* e_tok, const float* e_pos, void* x, void* stream);
/* Its gradient for one micro-batch d [S_mb, S_seq, S_hidden]: g_tok[tokens[t], :] += d[t, :] (always added,
 * ascending t, no atomics); g_pos[i, :] = (accumulate_pos ? g_pos[i, :] : 0) + sum over samples of d[b, i, :]. */
bf_status bf_op_embedding_bwd(int dtype, int S_mb, int S_seq, int S_voc, int S_hidden, const int32_t* tokens,
                              const void* d, float* g_tok, float* g_pos, int accumulate_pos, void* stream);
/* Softmax cross-entropy over rows of logits z [n_rows, S_voc] (`dtype`), in place: z becomes
 * (softmax(z) - onehot(label)) * scale; row_loss[t] = (logsumexp(z[t]) - z[t, label]) * scale (device fp32
 * [n_rows]); loss_out[0] = sum of row_loss in a fixed order.  A label outside 0..S_voc-1 zeroes its row. */
bf_status bf_op_ce_loss(int dtype, int n_rows, int S_voc, void* z, const int32_t* labels, float scale, float* row_loss,
                        float* loss_out, void* stream);
/* The output projection and its softmax cross-entropy in one, in pieces of the vocabulary: the logits z = y w_out^T of
 * n_rows rows (w_out [S_voc, S_hidden], y [n_rows, S_hidden], both `dtype`) are never kept.
 *   _fwd  lse[t] = logsumexp(z[t]);  row_loss[t] = (lse[t] - z[t, label]) * scale;  loss_out[0] = sum of row_loss, added in
 *         a fixed order (in fp64).  All device fp32.
 *   _bwd  from that lse: with dz = (softmax(z) - onehot(label)) * scale,
 *         dy[n_rows, S_hidden] (`dtype`) = dz w_out;  dw[S_voc, S_hidden] (fp32) = (accumulate ? dw : 0) + dz^T y
 * labels: device int32 [n_rows].  A row whose label is outside 0..S_voc-1 has row_loss 0, dy 0 and no part in dw, whatever
 * its y holds.  Sums have a fixed order: no atomics.  bf16 tensors run on the
 * bf16 matrix cores with logits and statistics in fp32 (rows that are not 16-byte aligned, S_hidden % 8 or
 * tensors that start elsewhere, through copies in the scratch); fp32 tensors as fp32 products.  dz enters the bf16 gradient products in bf16
 * parts: dw's in three, from S_hidden 8192 and 257 rows on in two (dw 1e-6 and 1.7e-6 off), dy's in one, up to 256 rows in two (dy 1.9e-3 off, or its
 * storage's rounding of 1.7e-3 alone).
 * S_piece: columns of a piece, in bf16 rounded up to whole chunks of 8 (0: the library's choice, 256 MiB of dz, and a bf16 forward, which
 * keeps nothing of a piece, in one; given, the scratch does not grow with the vocabulary); work: device scratch, 256-byte aligned, of
 * bf_op_vocab_loss_work_bytes(..., backward = 0 or 1) bytes (0 for bad sizes), owned by the caller; calls that overlap need
 * their own.  Sizes are 1 to 2^21; tensors are aligned to their elements. */
size_t bf_op_vocab_loss_work_bytes(int dtype, int n_rows, int S_hidden, int S_voc, int S_piece, int backward);
bf_status bf_op_vocab_loss_fwd(int dtype, int n_rows, int S_hidden, int S_voc, int S_piece, const void* y, const void* w_out,
                               const int32_t* labels, float scale, float* lse, float* row_loss, float* loss_out, void* work,
                               size_t work_bytes, void* stream);
bf_status bf_op_vocab_loss_bwd(int dtype, int n_rows, int S_hidden, int S_voc, int S_piece, const void* y, const void* w_out,
                               const int32_t* labels, const float* lse, float scale, void* dy, float* dw, int accumulate,
                               void* work, size_t work_bytes, void* stream);

/* Fused Adam over n contiguous fp32 parameters (bias-corrected, decoupled weight decay), step t >= 1;
 * w_lp: bf16 copy of w to refresh, or NULL. */
bf_status bf_op_adam(size_t n, float* w, float* m, float* v, const float* g, void* w_lp, int t,
                     float lr, float beta1, float beta2, float adam_eps, float weight_decay, void* stream);

/* Gradient norm and clipping, global over a list of tensors of one type (`dtype`: fp32 main-grads or bf16 gradients).  The list is
 * what this process holds: where ranks hold parts of a model, the squares of their out[0] add up to the whole norm's, and the
 * coefficient from that sum is the caller's to make (_scale and _adam_clipped take any).  The lists (g, dst, n, tensors) are host arrays, read during the call; the tensors they name are device memory, aligned to their
 * elements and no more.  A tensor of no elements is skipped, its pointers may be NULL.
 *
 *   out[0] = norm = sqrt(sum over all tensors and elements of g^2), squares and sums in fp64 and in a fixed order
 *   out[1] = coefficient = norm > max_norm ? max_norm / norm : 1;  NaN where a gradient is infinite or NaN
 *
 * out: device fp32 [2].  max_norm > 0 (infinity: the norm alone).  work: device scratch of bf_op_grad_norm_work_bytes(...)
 * bytes, 8-byte aligned, owned by the caller; calls that overlap need their own.  Nothing waits on the host. */
size_t bf_op_grad_norm_work_bytes(int n_tensors, const size_t* n);
bf_status bf_op_grad_norm(int dtype, int n_tensors, const void* const* g, const size_t* n, float max_norm, float* out,
                          void* work, size_t work_bytes, void* stream);
/* dst_i = g_i * coef[0], rounded once; dst_i may be g_i, but no tensor may overlap another.  coef: device fp32. */
bf_status bf_op_grad_scale(int dtype, int n_tensors, const void* const* g, void* const* dst, const size_t* n,
                           const float* coef, void* stream);
/* bf_op_adam on g_i * coef[0] for a list of tensors in one go (the gradients themselves stay as they are).  A coefficient
 * that is not finite leaves the step out: w, m, v and w_lp stay as they were.  No two tensors may overlap. */
typedef struct {
  float *w, *m, *v;
  const float* g;
  void* w_lp; /* bf16 copy of w to refresh, or NULL */
  size_t n;
} bf_adam_tensor;
bf_status bf_op_adam_clipped(int n_tensors, const bf_adam_tensor* tensors, const float* coef, int t, float lr, float beta1,
                             float beta2, float adam_eps, float weight_decay, void* stream);

/* Training in 8 bits: operands of products as 8-bit floating-point codes with a scale for each block of 128, and Adam's moments in 8 bits.
 * These are for training loops that call single kernels, beside bf_op_gemm and bf_op_adam_clipped; the stack's own steps do not use them.
 *
 * The 8-bit form of a matrix of `rows` rows of n elements, blocks along its rows:
 *   codes   [rows][bf_op_fp8_row_bytes(n)] bytes (n rounded up to 128; zeros behind element n): BF_E4M3 (largest value 448) or
 *           BF_E5M2 (57344; its infinities are not used)
 *   scales  [ceil(n / 128)][rows rounded up to 16] bytes, bf_op_fp8_scale_elems(rows, n) in all: byte b, 254 at most, stands for 2^(b - 127); element k of row r
 *           is code[r][k] * 2^(scale[k / 128][r] - 127).  Bytes behind the last row are 127.
 * Both 16-byte aligned.  A linear layer y = x W (x [T, h_in], W [h_in, h_out]) takes, as A and B of bf_op_fp8_gemm:
 *   forward          y  [T, h_out]      x along its rows      W down its columns
 *   input gradient   dx [T, h_in]       dy along its rows     W along its rows
 *   weight gradient  dW [h_in, h_out]   x down its columns    dy down its columns
 *
 * _quantize  the forms of x [rows, cols] (`dtype`, rows ld_x elements apart, 0: cols) along its rows (q, scale) and down its columns (qt, scale_t: the
 *            form of the transpose), either pair or both in one pass over x; NULL: not that one.  The scale is the smallest power of two, 2^-127 or
 *            more, that brings the block's largest finite value into the format's range (of a block of zeros 2^0), codes are rounded once, to nearest
 *            even; infinities and NaN become NaN codes and leave the others as they are.  rows, cols up to 2^21.
 * _gemm      C[M,N] = A B^T + bias + R from the forms A [M, K] and B [N, K], dense C and R [M, N] in `dtype`, bias fp32 [N]; bias, R may be NULL,
 *            R may be C.  accumulate = 1 (fp32 only): C += that.  A bf16 C comes from the 8-bit matrix instructions, whose sums inside a block keep about 16
 *            bits (1.5e-5 of the result in 2-norm for normal operands, 8e-5 with large outliers in every block: under bf16's rounding of 1.7e-3; an element is off by less than 2^-12 of
 *            its products' magnitudes, which is more than its own rounding where they cancel, and such elements land on another bf16 number than an fp32 sum: 1 to 4 % of them); an fp32 C
 *            from operands widened to bf16, with fp32 sums: exactly, but for bits under 2^-133 (of e4m3 under scales of 2^-124, of e5m2 of 2^-117) and codes that
 *            stand for 2^128 or more, which become infinite.  Sums have a fixed order: no atomics.  work: device scratch, 256-byte aligned, of
 *            _work_bytes(...) bytes (0: none needed, or bad sizes), owned by the caller; calls that overlap need their own.  Sizes are 1 to 2^21.
 * _gemm_tile what a product of this shape runs on: tiles of edge x edge (256, 128, 64), `waves` to a workgroup, the contraction in `slices` (1: not cut).  Host arithmetic only.
 *            Returns 1, or 0 (and zeros) for sizes or a type that _gemm refuses. */
typedef enum { BF_E4M3 = 0, BF_E5M2 = 1 } bf_fp8_format;
size_t bf_op_fp8_row_bytes(int n);
size_t bf_op_fp8_scale_elems(int rows, int n);
bf_status bf_op_fp8_quantize(int dtype, int format, int rows, int cols, const void* x, size_t ld_x, void* q, void* scale, void* qt, void* scale_t,
                             void* stream);
size_t bf_op_fp8_gemm_work_bytes(int dtype, int M, int N, int K);
int bf_op_fp8_gemm_tile(int dtype, int M, int N, int K, int* edge, int* waves, int* slices);
bf_status bf_op_fp8_gemm(int format_a, int format_b, int dtype, int M, int N, int K, const void* A, const void* scale_a, const void* B,
                         const void* scale_b, void* C, const float* bias, const void* R, int accumulate, void* work, size_t work_bytes, void* stream);

/* bf_op_adam_clipped with both moments of a tensor in 8 bits (2 1/64 bytes per parameter instead of 8):
 *   state   device, 16-byte aligned, bf_op_adam8_state_bytes(n) bytes: for each 128 elements 128 codes of m (BF_E4M3) and 128 of v, and
 *           behind all blocks two scale bytes for each (m's and v's; 2^(b - 127) as above).  v's codes have no sign: 4 bits of exponent, 4 of mantissa,
 *           code c below 16 is c / 16, above (1 + c % 16 / 16) 2^(c / 16 - 1).  All zero bytes: moments of zero.
 *   g       fp32 or bf16 (`dtype`), used times coef[0]
 * The new moments are beta1 m + (1 - beta1) g and beta2 v + (1 - beta2) g g in fp32, each operation rounded by itself (so that their codes are the same bits wherever that is done),
 * and the step is taken from them before they are rounded, with a root and a quotient to an ulp each and a root of 2^-63 at least: where sqrt(v / (1 - beta2^t)) is less than that,
 * gradients under 1e-19, and adam_eps does not cover it, the step is smaller than the formula's.  The moments are then rounded at random, up with the chance of their distance from the code below
 * (in 65536ths): a mean that moves by less than half a code each step still moves.  The random numbers are a hash of (seed, t, the tensor's place
 * in the list, element): the same call gives the same bits.  (A tensor takes a stretch of one sequence of 2^32 numbers, from a place that seed, t and its place in the list give.  Stretches may
 * overlap, among 24 tensors of 4 to 16 Mi elements about one pair a step, and those elements are rounded by the same numbers; a tensor past 2^32 elements meets its own again.)  A v above zero is kept at the smallest code or more, 2^-18.95 of the block's
 * largest, so that no step is divided by a v that was rounded away.  Values that are not finite stay with their element, out of its block's scales: a m that is infinite or NaN
 * becomes NaN; a v that overflows to infinity beside a finite m is kept as that, by the code 0xff of m, which stands for m = 0 and v = infinity: but for the weight decay its
 * weight rests from then on, as in bf_op_adam_clipped.  t and seed are values of the call: a captured graph repeats them.
 * The rates are double, as 1 - beta2 of an fp32 0.999 is 5e-5 off.  A coefficient that is not finite leaves the step out.  No two tensors may overlap. */
typedef struct {
  float* w;
  void* state;
  const void* g;
  void* w_lp; /* bf16 copy of w to refresh, or NULL */
  size_t n;
} bf_adam8_tensor;
size_t bf_op_adam8_state_bytes(size_t n);
bf_status bf_op_adam8(int dtype, int n_tensors, const bf_adam8_tensor* tensors, const float* coef, uint64_t seed, int t, double lr, double beta1, double beta2,
                      double adam_eps, double weight_decay, void* stream);
/* What states stand for: m and v of n elements each in `dtype` (bf16 holds every code times its scale exactly, but under 2^-126), either may be NULL. */
typedef struct {
  const void* state;
  void *m, *v;
  size_t n;
} bf_adam8_moments_tensor;
bf_status bf_op_adam8_moments(int dtype, int n_tensors, const bf_adam8_moments_tensor* tensors, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* BF_OPS_H */
