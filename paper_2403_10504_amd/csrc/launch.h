// Internal launchers of the libatom kernels (host side).  Every launcher only
// enqueues work on the given stream and returns the launch status.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace atom {

enum { DT_F32 = 0, DT_BF16 = 1 };

enum Epilogue {
  EPI_STORE = 0,       // C = acc                          (element type)
  EPI_STORE_F32 = 1,   // C = acc                          (fp32)
  EPI_ACC_F32 = 2,     // C += acc                         (fp32)
  EPI_BIAS = 3,        // C = acc + bias[n]                (element type)
  EPI_BIAS_GELU = 4,   // aux = acc + bias[n]; C = GELU(aux)
  EPI_BIAS_RESID = 5,  // C = resid + (acc + bias[n])      (fp32)
  EPI_GELU_BWD = 6,    // C = acc * GELU'(aux)             (element type)
  // the linear head's loss (loss.hip); not reachable through atom_k_gemm
  EPI_LSE = 7,         // per row and half tile: max and sum of exponentials of acc
  EPI_DZ = 8,          // C = (exp(acc - lse[m]) - [target]) * rowscale[m]  (element type)
  EPI_SCALE = 9,       // C = alpha * acc                  (element type)
  EPI_SCALE_F32 = 10,  // C = alpha * acc                  (fp32)
  EPI_SCALE_ACC = 11,  // C += alpha * acc                 (fp32)
  EPI_SUM_SCALE = 12,  // C = alpha * (resid + acc)        (element type; resid fp32)
  // the Newton-Schulz products (orthogonalize.hip); see NsArgs
  EPI_NS_GRAM = 13,    // C = alpha * acc, symmetric
  EPI_NS_POLY = 14,    // C = alpha * acc + beta * aux, symmetric
  EPI_NS_STEP = 15,    // C = alpha * acc + beta * aux, or the result from it
  EPI_NS_PART = 16,    // a range of k of EPI_NS_GRAM: raw fp32 tiles to C
};

// A dispatch counts its threads along a dimension in 32 bits: workgroups of 256.
constexpr int64_t MAX_WORKGROUPS = 1 << 24;

// The epilogues of the Newton-Schulz products.  Matrices are fp16 in one or two
// planes (value = hi + lo); every length is a multiple of 32.  A symmetric
// product computes the tiles on and below the diagonal and stores each on both
// sides of it.
constexpr int NS_EXPS = 64;  // most steps
struct NsArgs {
  int64_t sa, sb, sc;        // elements from one matrix of the batch to the next: A, B; C and aux
  int64_t pa, pb;            // elements from the hi to the lo plane of A and B
  int kp;                    // k tiles of 32 of one pass over k (two planes: three passes, three: six)
  int ranges, range;         // EPI_NS_PART: ranges of k, k tiles of each (the last may be shorter)
  const void *aux, *aux_lo;  // as C
  void* C_lo;
  float beta;
  // X of a step is held times 2^e, e per matrix and step (orthogonalize.hip):
  // this step's of matrix 0, the next step's behind it, matrices NS_EXPS apart
  const int* exps;
  // the last step: out = scale * (...), of orows x ocols, instead of C
  void* out;
  int64_t ldo, so;
  int out_mode;              // 0 bf16, 1 fp32, 2 fp32 out = keep * out + ..., 3 none (C)
  int orows, ocols;
  bool vec;                  // out's rows hold whole aligned 4-vectors
  float scale, keep;
};

// A product of fp32 operands held as three bf16 planes each (x = h + m + l,
// loss.hip): pa, pb and kp above, the k of one pass, and the planes of EPI_DZ's
// result.
struct PlaneArgs {
  int64_t pa, pb, pc;
  int kp, k;  // kp 0: not such a product
};

struct GemmArgs {
  const void* A;
  const void* B;
  void* C;
  const void* bias;
  const float* resid;
  void* aux;
  int64_t lda, ldb, ldc, ldaux;
  int M, N, K;
  float* ws;          // optional fp32 workspace for a split over k (may be null)
  uint64_t ws_bytes;  // its size; a split needs splits * M * N * 4 bytes
  int splits, kquads; // set by the launcher: k ranges and the groups of 128 k of each
  bool stream;        // set by the launcher: fp32 results are stored past the caches
  // the loss epilogues
  float alpha;            // EPI_SCALE*, EPI_SUM_SCALE
  const int32_t* tgt;     // EPI_LSE, EPI_DZ: target column of each row, negative: none
  const float* lse;       // EPI_DZ: natural log-sum-exp of each row
  const float* rowscale;  // EPI_DZ: factor of each row, null: 1
  float* ztgt;            // EPI_LSE: receives acc at each row's target
  int v0, V;              // EPI_DZ: column 0 is column v0 of the V of the vocabulary
  NsArgs ns;
  PlaneArgs pl;
};

// The layout and epilogue combinations of the training step: forward, data
// gradient and weight gradient of a linear layer.
constexpr bool gemm_main_combo(bool akc, bool bkc, int epi) {
  if (akc && bkc) return epi != EPI_ACC_F32 && epi != EPI_GELU_BWD;
  if (akc) return epi == EPI_STORE || epi == EPI_STORE_F32 || epi == EPI_GELU_BWD;
  return !bkc && (epi == EPI_STORE || epi == EPI_STORE_F32 || epi == EPI_ACC_F32);
}

// Those of the linear head's loss: logits, then both gradients.
constexpr bool gemm_loss_combo(bool akc, bool bkc, int epi) {
  if (epi == EPI_LSE || epi == EPI_DZ) return akc && bkc;
  if (epi == EPI_SCALE || epi == EPI_SCALE_ACC) return !bkc;
  if (epi == EPI_SCALE_F32) return !akc && !bkc;
  return epi == EPI_SUM_SCALE && akc && !bkc;
}

// The same of fp32 operands in three bf16 planes: every result is fp32.
constexpr bool gemm_planes_combo(bool akc, bool bkc, int epi) {
  if (epi == EPI_LSE || epi == EPI_DZ) return akc && bkc;
  return !bkc && (epi == EPI_SCALE_F32 || epi == EPI_SCALE_ACC);
}

// Tile configurations of the direct-load kernel (gemm_dl.h); 256x192 and
// 256x128 exist for gemm_main_combo only.
hipError_t gemm_dl_256(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_dl_192(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_dl_256x128(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_dl_128(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_dl_64(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_dl_f32_64(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_dl_f32_32(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);

// The same tiles with the loss epilogues (gemm_loss_combo).
hipError_t gemm_loss_256(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_loss_192(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_loss_256x128(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_loss_128(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_loss_64(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_planes_256(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);  // three planes
hipError_t gemm_planes_192(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_planes_256x128(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_planes_128(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_planes_64(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_loss_f32_64(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);
hipError_t gemm_loss_f32_32(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s);

// Newton-Schulz products on square tiles of bs (64, 128, 192 or 256; EPI_NS_PART:
// 64 alone); planes 1 or 2, `batch` matrices.
hipError_t gemm_ns(const GemmArgs& g, int bs, int planes, int batch, bool akc, bool bkc, int epi, hipStream_t s);

hipError_t gemm_check(const GemmArgs& g, int dtype, bool a_kcontig, bool b_kcontig);
hipError_t gemm(const GemmArgs& g, int dtype, bool a_kcontig, bool b_kcontig, int epi, hipStream_t s);
// The products of the linear head's loss: the epilogues of gemm_loss_combo, and
// EPI_STORE_F32 with A k-contiguous and B not.  Unlike gemm(),
// M and K may be any length where the memory of A holds whole chunks: rows of a
// not k-contiguous A up to the next chunk may be read (they reach no output),
// and a k-contiguous A holds zeros from K to the next chunk.  With g.pl.kp, A
// and B are three bf16 planes, N and K any multiples of 4 (operands hold zeros
// up to whole chunks), and the results fp32: EPI_LSE, EPI_DZ (three planes),
// EPI_SCALE_F32 and EPI_SCALE_ACC.
hipError_t gemm_loss(const GemmArgs& g, int dtype, bool a_kcontig, bool b_kcontig, int epi, hipStream_t s);
// Parts of a row (a maximum and a sum each) that EPI_LSE writes, [part][M].
int gemm_lse_parts(int dtype, int M, int N, int K);  // (three planes: bf16, six times the k)
// Whether its launches have less than MAX_WORKGROUPS.
bool gemm_lse_fits(int dtype, int M, int N, int K);

// LayerNorm over rows of length d (d % 64 == 0, d <= 8192).
//   y = (x - mean) * rstd * gamma + beta, x fp32, y element type.
hipError_t layernorm_fwd(int dtype, const float* x, const void* gamma, const void* beta, void* y, float* mean,
                         float* rstd, int64_t rows, int d, hipStream_t s);
// dres (+)= LN backward of dy; also writes dres_lp (element-type copy of the
// updated dres, may be null) and per-block partial column sums of dy*xhat and
// dy into part[nblk][2][d] (nblk from layernorm_bwd_blocks).
int64_t layernorm_bwd_blocks(int64_t rows, int d);
hipError_t layernorm_bwd(int dtype, const void* dy, const float* x, const float* mean, const float* rstd,
                         const void* gamma, float* dres, void* dres_lp, bool accumulate, float* part, int64_t rows,
                         int d, hipStream_t s);

// Deterministic column sums of a [rows][cols] matrix, out[j] (op)= sum of
// column j (out types and accumulate as for sum_parts): one launch for few
// rows, else partials of 16 rows into part (colsum_blocks(rows) * cols floats)
// and their sum.
int64_t colsum_blocks(int64_t rows);
hipError_t colsum(int in_dtype, const void* x, int64_t rows, int cols, int64_t ld, float* part, int out_dtype,
                  void* out, bool accumulate, hipStream_t s);
// out[j] (op)= sum over nparts of part[p][j] (+ stride between slabs); out
// type: DT_F32 with accumulate flag, or the element type (overwrite).
hipError_t sum_parts(const float* part, int64_t nparts, int cols, int64_t part_stride, int out_dtype, void* out,
                     bool accumulate, hipStream_t s);
// The same with two targets of one dtype and mode in one launch: columns
// c < split go to out[c], the rest to out2[c - split].
hipError_t sum_parts2(const float* part, int64_t nparts, int cols, int64_t part_stride, int out_dtype, void* out,
                      void* out2, int split, bool accumulate, hipStream_t s);

// Embedding: x[n] = wte[tok[n]] + wpe[n % T] (x fp32); ids outside [0, V)
// give NaN rows.
hipError_t embed_fwd(int dtype, const int32_t* tok, const void* wte, const void* wpe, float* x, int64_t n_tok,
                     int T, int V, int d, hipStream_t s);
// dwte rows of the listed unique tokens = sum of dx rows in `perm` order;
// all other rows zero (unless accumulate); dwpe[t] (op)= sum_b dx[b*T + t].
hipError_t embed_bwd(int out_dtype, const float* dx, const int32_t* perm, const int32_t* seg,
                     const int32_t* uniq, int n_uniq, void* dwte, void* dwpe, int V, int T, int B, int d,
                     bool accumulate, hipStream_t s);

// Cross-entropy rows: logits fp32 [rows][ldz] (V valid columns); writes
// dz = (softmax - onehot) * scale in the element type ([rows][lddz], padding
// columns up to lddz zeroed) and loss_rows[r] = logsumexp - z[y].
hipError_t xent_fwd_bwd(int dtype, const float* logits, int64_t ldz, const int32_t* tgt, void* dz, int64_t lddz,
                        float* loss_rows, int64_t rows, int V, float scale, hipStream_t s);

// Sum of n fp32 values in a fixed order, result in out[0] (fp32).
hipError_t sum_fixed(const float* x, int64_t n, float* out, hipStream_t s);

// fp32 -> element type conversion (n elements).
hipError_t convert_f32(int dtype, const float* x, void* y, int64_t n, hipStream_t s);
hipError_t fill_zero(void* p, int64_t bytes, hipStream_t s);
// Working-memory probe: fill `bytes` (a multiple of 16, 16-byte aligned) with
// a 32-bit word; high_water raises *out (a device counter) to 1 + the index of
// the last 16-byte unit that no longer holds it.
hipError_t fill_word(void* p, int64_t bytes, uint32_t word, hipStream_t s);
hipError_t high_water(const void* p, int64_t bytes, uint32_t word, unsigned long long* out, hipStream_t s);
// Streaming device copy of `bytes` (multiple of 16, 16-byte aligned).
hipError_t copy_bytes(const void* src, void* dst, int64_t bytes, hipStream_t s);
// Copy n 32-bit words on stream s by a kernel; src may be mapped pinned host
// memory (small uploads that must not occupy a DMA engine).
hipError_t copy_words(const uint32_t* src, uint32_t* dst, int64_t n, hipStream_t s);
// Makes device memory written by a DMA engine (after the host saw the copy
// complete) visible to the kernels enqueued after it on stream s.
hipError_t dma_acquire(hipStream_t s);

// Loss of a linear head and its gradients (atom_k_linear_xent_*); false where
// the sizes are refused.
bool linear_xent_ok(int dtype, int64_t rows, int V, int d);
bool linear_xent_fwd_ok(int dtype, int64_t rows, int V, int d);
uint64_t linear_xent_fwd_ws(int dtype, int64_t rows, int V, int d);
hipError_t linear_xent_fwd(int dtype, const void* x, int64_t ldx, const void* w, int64_t ldw, const int32_t* tgt,
                           float* lse, float* loss_rows, int64_t rows, int V, int d, void* ws, hipStream_t s);
uint64_t linear_xent_bwd_ws(int dtype, int64_t rows, int V, int d, int piece);
hipError_t linear_xent_bwd(int dtype, const void* x, int64_t ldx, const void* w, int64_t ldw, const int32_t* tgt,
                           const float* lse, const float* drow, float scale, void* dx, int64_t lddx, void* dw,
                           int64_t lddw, int dw_epi, int64_t rows, int V, int d, int piece, void* ws, hipStream_t s);

// Newton-Schulz orthogonalisation (atom_k_orthogonalize).  out_epi: EPI_STORE,
// EPI_STORE_F32 or EPI_ACC_F32; coef: host [steps][3].
bool orthogonalize_ok(int batch, int rows, int cols);
bool orthogonalize_coef_ok(const float* coef, int steps);
uint64_t orthogonalize_ws(int batch, int rows, int cols);
hipError_t orthogonalize(int dtype, const void* g, int64_t ldg, int64_t stride_g, void* out, int64_t ldo,
                         int64_t stride_o, int out_epi, float keep, float scale, int batch, int rows, int cols,
                         const float* coef, int steps, void* ws, hipStream_t s);

// Causal attention on a fused qkv [B*T][3*d] (element type), heads of dh in
// {64, 128}.  o [B*T][d], lse [B][H][T] fp32 (natural log).
hipError_t attn_fwd(int dtype, const void* qkv, void* o, float* lse, int B, int T, int H, int dh,
                    hipStream_t s);
// Backward: delta [B][H][T] fp32 scratch; dqkv [B*T][3*d].
hipError_t attn_bwd(int dtype, const void* qkv, const void* o, const void* dout, const float* lse, float* delta,
                    void* dqkv, int B, int T, int H, int dh, hipStream_t s);

// Cross attention (atom_k_cross_attn_*).  The launchers fill the fields from n_x on.
struct CrossArgs {
  const void *q, *k, *v, *dout;
  void *o, *dq, *dk, *dv;
  float *lse, *delta;  // [row][Hq]; [B * Hk][Tq G] of the workspace
  int64_t ldq, ldk, ldv, ldo, lddo, lddq, lddk, lddv;
  int64_t q_rows, k_rows;
  const int32_t *q_start, *q_len, *k_start, *k_len;
  int B, Tq, Tk, Hq, Hk, G;
  uint32_t gmul;  // ceil(2^32 / G): p / G is the high word of p gmul
  float scale;
  int n_x, splits;    // blocks of queries of a sequence and head group, ranges of its keys
  int k_x, k_splits;  // backward: blocks of keys, ranges of queries
  float *part, *part_k, *part_v;  // the ranges' sums of O or dQ, of dK and dV: [splits][B * Hk][rows][dh]
  float* ml;                      // forward: the ranges' maxima and sums, [splits][B * Hk][Tq G][2]
};

// Whether the sizes are taken, by the forward and the backward alike.
bool cross_attn_ok(int B, int Tq, int Tk, int Hq, int Hk, int dh);
uint64_t cross_attn_fwd_ws(int dtype, int B, int Tq, int Tk, int Hq, int Hk, int dh);
hipError_t cross_attn_fwd(int dtype, CrossArgs& a, int dh, void* ws, hipStream_t s);
uint64_t cross_attn_bwd_ws(int dtype, int B, int Tq, int Tk, int Hq, int Hk, int dh);
hipError_t cross_attn_bwd(int dtype, CrossArgs& a, int dh, void* ws, hipStream_t s);

// Rotary positions and the norms of queries and keys (atom_k_rope,
// atom_k_qknorm_rope_*).  back: the transposed turn.
hipError_t rope(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, const int32_t* pos, const double* freq,
                float mscale, int layout, bool back, int64_t rows, int T, int heads, int dh, int rot, hipStream_t s);
hipError_t qknorm_rope_fwd(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, const void* gq, const void* gk,
                           float eps, const int32_t* pos, const double* freq, float mscale, int layout, int64_t rows,
                           int T, int Hq, int Hk, int Hv, int dh, int rot, hipStream_t s);
uint64_t qknorm_rope_bwd_ws(int dh);
hipError_t qknorm_rope_bwd(int dtype, const void* dy, int64_t lddy, const void* x, int64_t ldx, void* dx, int64_t lddx,
                           const void* gq, const void* gk, float* dgq, float* dgk, float eps, const int32_t* pos,
                           const double* freq, float mscale, int layout, int64_t rows, int T, int Hq, int Hk, int Hv,
                           int dh, int rot, float* ws, hipStream_t s);

}  // namespace atom
