/*
 * atom_kernels.h - kernel-level entry points of libatom.
 *
 * The swapped step (atom.h) composes these kernels; they are exported on
 * their own so each can be checked against a reference in isolation.  All
 * pointers are device pointers except where noted; `stream` is a hipStream_t
 * (NULL = the default stream).  Every call only enqueues work and returns
 * ATOM_OK, ATOM_EINVAL (shape, alignment or dtype not supported) or ATOM_EHIP
 * (launch failed).  dtype is ATOM_F32 or ATOM_BF16 (bf16 tensors are raw
 * 16-bit patterns); accumulation is fp32 in every kernel.
 *
 * A call repeats its results bit for bit.  The order of its sums, and so their
 * last bits, follows from all of its sizes: tiles, splits and work per thread
 * are chosen by them (a product by M, N, K, epilogue and workspace; a head's
 * attention beyond 256 rows by the number of heads in the call; a row's
 * LayerNorm gradient at 2048 < d <= 4096 by the number of rows; column sums by
 * the number of rows).  Rows of different calls are equal to rounding only.
 */
#ifndef ATOM_KERNELS_H
#define ATOM_KERNELS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Epilogues of atom_k_gemm. */
enum {
  ATOM_EPI_STORE = 0,       /* C = acc                        (dtype)  */
  ATOM_EPI_STORE_F32 = 1,   /* C = acc                        (fp32)   */
  ATOM_EPI_ACC_F32 = 2,     /* C += acc                       (fp32)   */
  ATOM_EPI_BIAS = 3,        /* C = acc + bias[n]              (dtype)  */
  ATOM_EPI_BIAS_GELU = 4,   /* aux = acc + bias[n]; C = GELU(aux)     */
  ATOM_EPI_BIAS_RESID = 5,  /* C = resid + acc + bias[n]      (fp32)   */
  ATOM_EPI_GELU_BWD = 6     /* C = acc * GELU'(aux)           (dtype)  */
};

/* Matrix product of a linear layer y = x W^T + b and its two gradients
 * (the decoder-block GEMMs of the GPT-3 model, Section III-B).
 *   C[m][n] = sum_k A(m,k) B(k,n), with
 *   A(m,k) = a_kcontig ? A[m*lda + k] : A[k*lda + m],
 *   B(k,n) = b_kcontig ? B[n*ldb + k] : B[k*ldb + n].
 * C, resid, aux are row-major with leading dimensions ldc (resid shares ldc)
 * and ldaux.  Requirements: K % 8 == 0 (bf16) or K % 4 == 0 (fp32); the
 * leading dimension of a k-contiguous operand a multiple of 8 (bf16) or 4
 * (fp32); for bf16 an operand that is not k-contiguous needs an even row
 * count and an even leading dimension; A, B, C 16-byte aligned.
 * ws (fp32, ws_bytes, 16-byte aligned, may be NULL) lets a problem with few
 * output tiles and a long k split k over workgroups for the store epilogues
 * (STORE, STORE_F32, ACC_F32); the partials are summed in a fixed order.  The
 * other epilogues neither read nor write it. */
int atom_k_gemm(int dtype, int a_kcontig, int b_kcontig, int epi, int M, int N, int K, const void* A, int64_t lda,
                const void* B, int64_t ldb, void* C, int64_t ldc, const void* bias, const float* resid, void* aux,
                int64_t ldaux, float* ws, uint64_t ws_bytes, void* stream);

/* LayerNorm forward over rows of d (d % 64 == 0, d <= 8192), eps 1e-5,
 * biased variance: y = (x - mean) * rstd * gamma + beta.  x fp32 [rows][d];
 * y dtype; mean, rstd fp32 [rows]. */
int atom_k_layernorm_fwd(int dtype, const float* x, const void* gamma, const void* beta, void* y, float* mean,
                         float* rstd, int64_t rows, int d, void* stream);

/* Scratch floats atom_k_layernorm_bwd needs in `part`. */
int64_t atom_k_layernorm_bwd_part_floats(int64_t rows, int d);

/* LayerNorm backward: dx = rstd * (g' - mean(g') - xhat * mean(g' xhat)),
 * g' = dy * gamma; dres (fp32) = dx or dres + dx (accumulate); dres_lp
 * (dtype, may be NULL) receives the updated dres rounded; dgamma, dbeta
 * (fp32 [d]) = column sums of dy * xhat and dy (fixed order). */
int atom_k_layernorm_bwd(int dtype, const void* dy, const float* x, const float* mean, const float* rstd,
                         const void* gamma, float* dres, void* dres_lp, int accumulate, float* dgamma, float* dbeta,
                         float* part, int64_t rows, int d, void* stream);

/* Causal self-attention on qkv [B*T][3*d] (q, k, v at column offsets 0, d,
 * 2d; head h at h*dh), dh in {64, 128}, scale 1/sqrt(dh): o [B*T][d] and
 * lse [B][H][T] (natural-log row log-sum-exp of the scaled scores). */
int atom_k_attn_fwd(int dtype, const void* qkv, void* o, float* lse, int B, int T, int H, int dh, void* stream);

/* Its backward: dqkv [B*T][3*d] from dout [B*T][d]; delta is fp32 scratch
 * of [B][H][T]. */
int atom_k_attn_bwd(int dtype, const void* qkv, const void* o, const void* dout, const float* lse, float* delta,
                    void* dqkv, int B, int T, int H, int dh, void* stream);

/* atom_k_attn_bwd for callers that cannot allocate (code under HIP graph
 * capture, serving loops, harnesses that forbid hipMalloc): the same kernels,
 * with the D scratch in a library-owned device array of
 * ATOM_ATTN_NOALLOC_MAX_ROWS floats (4 MiB per GPU, held until the process
 * ends) instead of a `delta` argument.  Allocates nothing.  B * H * T above
 * the limit: ATOM_EINVAL.  Every call on one GPU uses the same array, so
 * calls that overlap on one GPU (different streams, or threads) race; calls
 * in order on one stream do not.  Nothing in the array must start at zero. */
#define ATOM_ATTN_NOALLOC_MAX_ROWS (1 << 20)
int atom_k_attn_bwd_noalloc(int dtype, const void* qkv, const void* o, const void* dout, const float* lse,
                            void* dqkv, int B, int T, int H, int dh, void* stream);

/* Scratch floats atom_k_colsum needs in `part`. */
int64_t atom_k_colsum_part_floats(int64_t rows, int cols);

/* out[j] = sum over rows of x[r][j] (x dtype [rows][cols], out fp32),
 * fixed order. */
int atom_k_colsum(int dtype, const void* x, int64_t rows, int cols, float* out, float* part, void* stream);

/* Softmax cross-entropy rows: logits fp32 [rows][ldz] with V valid columns,
 * target ids tgt[rows]; dz = (softmax - onehot) * scale (dtype, row pitch
 * lddz, columns V..lddz-1 zeroed); loss_rows = logsumexp - z[y] (NaN for a
 * target outside [0, V), which is never read). */
int atom_k_xent(int dtype, const float* logits, int64_t ldz, const int32_t* tgt, void* dz, int64_t lddz,
                float* loss_rows, int64_t rows, int V, float scale, void* stream);

/* Cross-entropy of a linear head over a vocabulary, with no logits in memory
 * (the "Logits" layer, Section III-B; atom_k_gemm and atom_k_xent do it with
 * the logits of a range of tokens):
 *   z[n][v] = sum_c x[n][c] w[v][c],  lse[n] = log sum_v exp z[n][v],
 *   loss_rows[n] = lse[n] - z[n][tgt[n]].
 * x [rows][ldx] and w [V][ldw] in dtype, d columns of each; tgt, lse and
 * loss_rows [rows].  A token whose target is negative (ATOM_XENT_IGNORE) takes
 * no part: lse and loss 0, whatever its row holds.  A target of V or more:
 * loss NaN (it is never read).  Logits of a whole row at -infinity, or one at
 * +infinity or NaN: loss NaN (fp32 of 768 rows and 2^32 products or more,
 * which runs on three bf16 planes: infinite inputs too).
 * Requirements: d a positive multiple of 8 (bf16) or 4 (fp32), ldx and ldw
 * multiples of the same, at least d; x, w and ws 16-byte aligned; rows up to
 * 2^28 (0: nothing is done, and no pointer looked at), V from 1 to 2^28, d up to
 * 2^24, with less than 2^30 tiles of 32 x 32 between any two of them, and for
 * the forward call less than 2^24 tiles of logits where it takes tiles of less
 * than 256 rows (fp32 of less than 768 rows: 64 x 64).  ws: device scratch of at
 * least the bytes that the query returns (0 for sizes it refuses); calls that
 * may overlap need scratch of their own. */
#define ATOM_XENT_IGNORE (-1)
uint64_t atom_k_linear_xent_fwd_ws_bytes(int dtype, int64_t rows, int V, int d);
int atom_k_linear_xent_fwd(int dtype, const void* x, int64_t ldx, const void* w, int64_t ldw, const int32_t* tgt,
                           float* lse, float* loss_rows, int64_t rows, int V, int d, void* ws, uint64_t ws_bytes,
                           void* stream);

/* Its gradients, in pieces of the vocabulary:
 *   dz[n][v] = (exp(z[n][v] - lse[n]) - [v = tgt[n]]) * drow[n]
 *   dx[n][c] = scale * sum_v dz[n][v] w[v][c]   (dtype, [rows][lddx])
 *   dw[v][c] = scale * sum_n dz[n][v] x[n][c]   ([V][lddw])
 * z is computed again, `piece` columns at a time (rounded up to a multiple of
 * 8, at most V; 0: the library's choice, dz of up to 512 MB and 2048 columns at
 * least), and dz of a piece, drow in it, goes through the workspace in dtype
 * (fewer columns take less of it and more time).  lse comes from the forward
 * call; drow (NULL: 1) weighs a token (a factor of all tokens is more accurate as
 * scale, which no bf16 dz rounds).  A token with a negative target or with drow 0
 * adds nothing, whatever its row of x holds, and its row of dx is zero (of a
 * finite w); one with a target of V or more makes both gradients NaN.  dx or dw
 * may be NULL (not wanted).
 * dw_epi: ATOM_EPI_STORE (dw in dtype), ATOM_EPI_STORE_F32 or ATOM_EPI_ACC_F32
 * (dw fp32, += the gradient).  rows 0: dw is zeroed, or kept by
 * ATOM_EPI_ACC_F32, and no other pointer looked at.  dx and dw must not overlap
 * the inputs.  Requirements as above, for dx and lddx, dw and lddw as well. */
uint64_t atom_k_linear_xent_bwd_ws_bytes(int dtype, int64_t rows, int V, int d, int piece);
int atom_k_linear_xent_bwd(int dtype, const void* x, int64_t ldx, const void* w, int64_t ldw, const int32_t* tgt,
                           const float* lse, const float* drow, float scale, void* dx, int64_t lddx, void* dw,
                           int64_t lddw, int dw_epi, int64_t rows, int V, int d, int piece, void* ws,
                           uint64_t ws_bytes, void* stream);

/* Token and position embedding (node 0 of the layer chain):
 * x[n][c] = wte[tok[n]][c] + wpe[n % T][c]; x fp32 [n_tok][d].  A token id
 * outside [0, V) yields a NaN row (no out-of-range read). */
int atom_k_embed_fwd(int dtype, const int32_t* tok, const void* wte, const void* wpe, float* x, int64_t n_tok,
                     int T, int V, int d, void* stream);

/* Orthogonalised update of a weight matrix by Newton-Schulz products (the
 * Muon optimiser's step for the linear layers' weights), for `batch` matrices
 * g [rows][ldg] in dtype, stride_g elements apart:
 *   X = g / (|g|_F + 1e-7); for each step k, with A = X X^T,
 *   X <- a_k X + (b_k A + c_k A A) X;  then, with O = scale * X,
 *   out = O (ATOM_EPI_STORE: dtype; ATOM_EPI_STORE_F32: fp32), or
 *   out = keep * out + O (ATOM_EPI_ACC_F32: fp32, the weights themselves with
 *   scale = -lr * ... and keep = 1 - lr * decay).  `keep` is read by the last
 *   form only.
 * coef: HOST array [steps][3] of a, b, c, read before the call returns; NULL:
 * the quintic (3.4445, -4.7750, 2.0315) in every step.  The products run on
 * the shorter side: A = X^T X and X (...) where rows > cols.  A matrix of
 * zeros gives zeros; one with an infinity or a NaN gives NaN throughout.  Where
 * |g|_F is far below 1e-7 X is small, and as accurate as any other: it is held
 * relative to a bound of its singular values (22 bits, down to 2^-35 of the bound).
 * The result's type sets the precision: in bf16, products in fp16 with fp32 sums
 * (X itself in 22 bits), off by about the result's own rounding; in fp32 (of bf16
 * gradients too, ATOM_EPI_STORE_F32 and ATOM_EPI_ACC_F32), every factor in 22
 * bits, in 2.1 to 2.9 times the time.
 * Any rows, cols >= 1 (with less than 2^30 tiles of 64 x 64, and 2^24 of the
 * products' tiles of 64 to 256, in a batch), leading
 * dimensions >= cols, 0 <= batch <= 65535 (0: nothing is done), 0 <= steps <=
 * 64; stride_g >= 0; the outputs of a batch must not overlap: stride_o >=
 * (rows - 1) * ldo + cols, or matrices side by side, cols <= stride_o with
 * batch * stride_o <= ldo; any stride for one matrix.  g and out are aligned to
 * their elements, ws to 16 bytes; out may be g itself (same type, ld and
 * stride), else they must not overlap.  Steps whose polynomial takes singular
 * values of [0, 1] beyond 4, or b t + c t^2 beyond 32 on the way, do not fit
 * fp16: ATOM_EINVAL.  ws: as for atom_k_linear_xent_fwd. */
#define ATOM_NS_MAX_STEPS 64
uint64_t atom_k_orthogonalize_ws_bytes(int dtype, int batch, int rows, int cols);
int atom_k_orthogonalize(int dtype, const void* g, int64_t ldg, int64_t stride_g, void* out, int64_t ldo,
                         int64_t stride_o, int out_epi, float keep, float scale, int batch, int rows, int cols,
                         const float* coef, int steps, void* ws, uint64_t ws_bytes, void* stream);

/* Plain device copy of `bytes` (a multiple of 16; both pointers 16-byte
 * aligned, not overlapping): reads and writes each byte once.  Measurement
 * only: its known traffic calibrates the HBM byte counters. */
int atom_k_copy(const void* src, void* dst, int64_t bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ATOM_KERNELS_H */
