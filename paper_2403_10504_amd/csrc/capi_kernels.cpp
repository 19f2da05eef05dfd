// extern "C" wrappers of the kernel launchers (include/atom_kernels.h).
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/atom.h"
#include "../../include/atom_kernels.h"
#include "launch.h"

using namespace atom;

namespace {
inline int st(hipError_t e) {
  if (e == hipSuccess) return ATOM_OK;
  if (e == hipErrorInvalidValue) return ATOM_EINVAL;
  return ATOM_EHIP;
}
inline hipStream_t S(void* s) { return static_cast<hipStream_t>(s); }
inline bool dt_ok(int dt) { return dt == ATOM_F32 || dt == ATOM_BF16; }
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
// rows of d elements, ld apart, in whole 16-byte chunks
inline bool rows_ok(int dt, const void* p, int64_t ld, int d) {
  return p && !misaligned(p) && ld >= d && ld % (dt == ATOM_BF16 ? 8 : 4) == 0;
}
inline bool aligned_to(int dt, const void* p) { return reinterpret_cast<uintptr_t>(p) % (dt == ATOM_BF16 ? 2 : 4) == 0; }
// rows, heads and turns of atom_k_rope and atom_k_qknorm_rope_*
inline bool turn_ok(int dt, int layout, int64_t rows, int64_t heads, int dh, int rot, float mscale) {
  return dt_ok(dt) && (layout == ATOM_ROPE_HALF || layout == ATOM_ROPE_PAIRS) && rows >= 0 && rows <= INT32_MAX &&
         heads >= 0 && heads <= 1 << 16 && dh >= 2 && dh <= 256 && dh % 2 == 0 && rot >= 0 && rot <= dh && rot % 2 == 0 &&
         isfinite(mscale);
}
inline bool heads_ok(int dt, const void* p, int64_t ld, int64_t heads, int dh) {
  return p && aligned_to(dt, p) && ld >= heads * dh && ld <= INT64_MAX / 8 / INT32_MAX;
}
inline bool positions_ok(const int32_t* pos, const double* freq, int T, int rot) {
  return rot == 0 || (freq && reinterpret_cast<uintptr_t>(freq) % 8 == 0 && reinterpret_cast<uintptr_t>(pos) % 4 == 0 &&
                      (pos || T >= 1));
}
inline bool cross_ok(int dt, const atom_cross_shape* s) {
  return dt_ok(dt) && s && cross_attn_ok(s->B, s->Tq, s->Tk, s->Hq, s->Hk, s->dh);
}
// starts come with lengths; without them the rows hold the padded batch
inline bool side_ok(const int32_t* start, const int32_t* len, int64_t rows, int64_t B, int64_t T) {
  if (reinterpret_cast<uintptr_t>(start) % 4 || reinterpret_cast<uintptr_t>(len) % 4 || rows < 0) return false;
  return start ? len != nullptr && rows <= INT32_MAX : rows >= B * T;
}
inline bool cross_rows_ok(int dt, const void* p, int64_t ld, int64_t heads, int dh) {
  return p && !misaligned(p) && ld >= heads * dh && ld % (dt == ATOM_BF16 ? 8 : 4) == 0 && ld < 1 << 24;
}
inline CrossArgs cross_args(const atom_cross_shape* s, const void* q, int64_t ldq, const void* k, int64_t ldk,
                            const void* v, int64_t ldv, float scale) {
  CrossArgs a{};
  a.q = q, a.k = k, a.v = v, a.ldq = ldq, a.ldk = ldk, a.ldv = ldv, a.scale = scale;
  a.B = s->B, a.Tq = s->Tq, a.Tk = s->Tk, a.Hq = s->Hq, a.Hk = s->Hk, a.G = s->Hq / s->Hk;
  a.gmul = static_cast<uint32_t>(((1ull << 32) + a.G - 1) / a.G);
  a.q_rows = s->q_rows, a.k_rows = s->k_rows;
  a.q_start = s->q_start, a.q_len = s->q_len, a.k_start = s->k_start, a.k_len = s->k_len;
  return a;
}
}  // namespace

extern "C" {

int atom_k_gemm(int dtype, int a_kcontig, int b_kcontig, int epi, int M, int N, int K, const void* A, int64_t lda,
                const void* B, int64_t ldb, void* C, int64_t ldc, const void* bias, const float* resid, void* aux,
                int64_t ldaux, float* ws, uint64_t ws_bytes, void* stream) {
  if (!dt_ok(dtype) || !A || !B || !C || epi < ATOM_EPI_STORE || epi > ATOM_EPI_GELU_BWD) return ATOM_EINVAL;
  if ((epi == ATOM_EPI_BIAS || epi == ATOM_EPI_BIAS_GELU || epi == ATOM_EPI_BIAS_RESID) && !bias) return ATOM_EINVAL;
  if ((epi == ATOM_EPI_BIAS_GELU || epi == ATOM_EPI_GELU_BWD) && (!aux || ldaux < N)) return ATOM_EINVAL;
  if (epi == ATOM_EPI_BIAS_RESID && !resid) return ATOM_EINVAL;
  GemmArgs g{};
  g.A = A;
  g.B = B;
  g.C = C;
  g.bias = bias;
  g.resid = resid;
  g.aux = aux;
  g.lda = lda;
  g.ldb = ldb;
  g.ldc = ldc;
  g.ldaux = ldaux;
  g.M = M;
  g.N = N;
  g.K = K;
  // The workspace serves the store epilogues only: a caller may hand the same
  // one to products with other epilogues on other streams.  (The step's own
  // workspace, used on one stream, splits k before every epilogue.)
  const bool store = epi == ATOM_EPI_STORE || epi == ATOM_EPI_STORE_F32 || epi == ATOM_EPI_ACC_F32;
  g.ws = store ? ws : nullptr;
  g.ws_bytes = g.ws ? ws_bytes : 0;
  return st(gemm(g, dtype, a_kcontig != 0, b_kcontig != 0, epi, S(stream)));
}

int atom_k_layernorm_fwd(int dtype, const float* x, const void* gamma, const void* beta, void* y, float* mean,
                         float* rstd, int64_t rows, int d, void* stream) {
  if (!dt_ok(dtype) || !x || !gamma || !beta || !y || !mean || !rstd) return ATOM_EINVAL;
  return st(layernorm_fwd(dtype, x, gamma, beta, y, mean, rstd, rows, d, S(stream)));
}

int64_t atom_k_layernorm_bwd_part_floats(int64_t rows, int d) { return layernorm_bwd_blocks(rows, d) * 2 * d; }

int atom_k_layernorm_bwd(int dtype, const void* dy, const float* x, const float* mean, const float* rstd,
                         const void* gamma, float* dres, void* dres_lp, int accumulate, float* dgamma, float* dbeta,
                         float* part, int64_t rows, int d, void* stream) {
  if (!dt_ok(dtype) || !dy || !x || !mean || !rstd || !gamma || !dres || !dgamma || !dbeta || !part) return ATOM_EINVAL;
  int s = st(layernorm_bwd(dtype, dy, x, mean, rstd, gamma, dres, dres_lp, accumulate != 0, part, rows, d, S(stream)));
  if (s != ATOM_OK) return s;
  const int64_t np = layernorm_bwd_blocks(rows, d);
  return st(sum_parts2(part, np, 2 * d, 2 * static_cast<int64_t>(d), DT_F32, dgamma, dbeta, d, false, S(stream)));
}

int atom_k_attn_fwd(int dtype, const void* qkv, void* o, float* lse, int B, int T, int H, int dh, void* stream) {
  if (!dt_ok(dtype) || !qkv || !o || !lse) return ATOM_EINVAL;
  return st(attn_fwd(dtype, qkv, o, lse, B, T, H, dh, S(stream)));
}

int atom_k_attn_bwd(int dtype, const void* qkv, const void* o, const void* dout, const float* lse, float* delta,
                    void* dqkv, int B, int T, int H, int dh, void* stream) {
  if (!dt_ok(dtype) || !qkv || !o || !dout || !lse || !delta || !dqkv) return ATOM_EINVAL;
  return st(attn_bwd(dtype, qkv, o, dout, lse, delta, dqkv, B, T, H, dh, S(stream)));
}

int atom_rope_freqs(int rot, double base, int scaling, double factor, double trained, double slow, double fast,
                    double* freq) {
  if (!freq || rot < 2 || rot > 256 || rot % 2 || !(base > 0) || !isfinite(base)) return ATOM_EINVAL;
  if (scaling < ATOM_ROPE_PLAIN || scaling > ATOM_ROPE_PARTS) return ATOM_EINVAL;
  if (scaling != ATOM_ROPE_PLAIN && (!(factor > 0) || !isfinite(factor))) return ATOM_EINVAL;
  if (scaling == ATOM_ROPE_PARTS && !(slow >= 0 && slow < fast && isfinite(fast) && trained >= 1 && isfinite(trained)))
    return ATOM_EINVAL;
  double out[128];
  for (int i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2.0 * i / rot);
    if (scaling == ATOM_ROPE_LINEAR) f /= factor;
    // (the other base's power apart: that base itself may be beyond the numbers)
    if (scaling == ATOM_ROPE_BASE && i > 0) f *= pow(factor, -2.0 * i / (rot - 2));
    if (scaling == ATOM_ROPE_PARTS) {
      const double keep = fmin(1.0, fmax(0.0, (trained * f / (2.0 * M_PI) - slow) / (fast - slow)));
      f *= keep + (1.0 - keep) / factor;
    }
    if (!isfinite(f)) return ATOM_EINVAL;
    out[i] = f;
  }
  for (int i = 0; i < rot / 2; ++i) freq[i] = out[i];
  return ATOM_OK;
}

int atom_k_rope(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, const int32_t* pos, const double* freq,
                float mscale, int layout, int transposed, int64_t rows, int T, int heads, int dh, int rot, void* stream) {
  if (!turn_ok(dtype, layout, rows, heads, dh, rot, mscale)) return ATOM_EINVAL;
  if (rows == 0 || heads == 0) return ATOM_OK;
  if (!heads_ok(dtype, x, ldx, heads, dh) || !heads_ok(dtype, y, ldy, heads, dh) || !positions_ok(pos, freq, T, rot))
    return ATOM_EINVAL;
  if (x == y && ldx != ldy) return ATOM_EINVAL;
  return st(rope(dtype, x, ldx, y, ldy, pos, freq, mscale, layout, transposed != 0, rows, T, heads, dh, rot, S(stream)));
}

int atom_k_qknorm_rope_fwd(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, const void* gq, const void* gk,
                           float eps, const int32_t* pos, const double* freq, float mscale, int layout, int64_t rows,
                           int T, int Hq, int Hk, int Hv, int dh, int rot, void* stream) {
  if (Hq < 0 || Hk < 0 || Hv < 0 || !(eps >= FLT_MIN) || !isfinite(eps)) return ATOM_EINVAL;
  const int64_t heads = static_cast<int64_t>(Hq) + Hk + Hv;
  if (!turn_ok(dtype, layout, rows, heads, dh, rot, mscale)) return ATOM_EINVAL;
  if (rows == 0 || heads == 0) return ATOM_OK;
  if (!heads_ok(dtype, x, ldx, heads, dh) || !heads_ok(dtype, y, ldy, heads, dh) || !positions_ok(pos, freq, T, rot))
    return ATOM_EINVAL;
  if (!aligned_to(dtype, gq) || !aligned_to(dtype, gk) || (x == y && ldx != ldy)) return ATOM_EINVAL;
  return st(qknorm_rope_fwd(dtype, x, ldx, y, ldy, gq, gk, eps, pos, freq, mscale, layout, rows, T, Hq, Hk, Hv, dh, rot,
                            S(stream)));
}

uint64_t atom_k_qknorm_rope_bwd_ws_bytes(int64_t rows, int Hq, int Hk, int dh) {
  return Hq >= 0 && Hk >= 0 && turn_ok(ATOM_BF16, ATOM_ROPE_HALF, rows, static_cast<int64_t>(Hq) + Hk, dh, 0, 1.f)
             ? qknorm_rope_bwd_ws(dh)
             : 0;
}

int atom_k_qknorm_rope_bwd(int dtype, const void* dy, int64_t lddy, const void* x, int64_t ldx, void* dx, int64_t lddx,
                           const void* gq, const void* gk, float* dgq, float* dgk, float eps, const int32_t* pos,
                           const double* freq, float mscale, int layout, int64_t rows, int T, int Hq, int Hk, int Hv,
                           int dh, int rot, void* ws, uint64_t ws_bytes, void* stream) {
  if (Hq < 0 || Hk < 0 || Hv < 0 || !(eps >= FLT_MIN) || !isfinite(eps)) return ATOM_EINVAL;
  const int64_t heads = static_cast<int64_t>(Hq) + Hk + Hv;
  if (!turn_ok(dtype, layout, rows, heads, dh, rot, mscale)) return ATOM_EINVAL;
  if (!aligned_to(ATOM_F32, dgq) || !aligned_to(ATOM_F32, dgk)) return ATOM_EINVAL;
  if (rows > 0 && heads > 0) {
    if (!heads_ok(dtype, x, ldx, heads, dh) || !heads_ok(dtype, dy, lddy, heads, dh) ||
        !heads_ok(dtype, dx, lddx, heads, dh) || !positions_ok(pos, freq, T, rot))
      return ATOM_EINVAL;
    if (!aligned_to(dtype, gq) || !aligned_to(dtype, gk) || dx == x || (dx == dy && lddx != lddy)) return ATOM_EINVAL;
    if ((dgq || dgk) && (!ws || misaligned(ws) || ws_bytes < qknorm_rope_bwd_ws(dh))) return ATOM_EINVAL;
  }
  return st(qknorm_rope_bwd(dtype, dy, lddy, x, ldx, dx, lddx, gq, gk, dgq, dgk, eps, pos, freq, mscale, layout, rows, T,
                            Hq, Hk, Hv, dh, rot, static_cast<float*>(ws), S(stream)));
}

uint64_t atom_k_cross_attn_fwd_ws_bytes(int dtype, const atom_cross_shape* shape) {
  return cross_ok(dtype, shape) ? cross_attn_fwd_ws(dtype, shape->B, shape->Tq, shape->Tk, shape->Hq, shape->Hk, shape->dh)
                                : 0;
}

int atom_k_cross_attn_fwd(int dtype, const atom_cross_shape* shape, const void* q, int64_t ldq, const void* k,
                          int64_t ldk, const void* v, int64_t ldv, float scale, void* o, int64_t ldo, float* lse,
                          void* ws, uint64_t ws_bytes, void* stream) {
  if (!cross_ok(dtype, shape) || !(scale > 0) || !isfinite(scale)) return ATOM_EINVAL;
  const atom_cross_shape& c = *shape;
  if (!side_ok(c.q_start, c.q_len, c.q_rows, c.B, c.Tq) || !side_ok(c.k_start, c.k_len, c.k_rows, c.B, c.Tk))
    return ATOM_EINVAL;
  if (c.B == 0 || c.Tq == 0) return ATOM_OK;
  if (!cross_rows_ok(dtype, q, ldq, c.Hq, c.dh) || !cross_rows_ok(dtype, o, ldo, c.Hq, c.dh)) return ATOM_EINVAL;
  if (c.Tk > 0 && (!cross_rows_ok(dtype, k, ldk, c.Hk, c.dh) || !cross_rows_ok(dtype, v, ldv, c.Hk, c.dh)))
    return ATOM_EINVAL;
  const uint64_t need = cross_attn_fwd_ws(dtype, c.B, c.Tq, c.Tk, c.Hq, c.Hk, c.dh);
  if (!aligned_to(ATOM_F32, lse) || (need && (!ws || misaligned(ws) || ws_bytes < need))) return ATOM_EINVAL;
  CrossArgs a = cross_args(shape, q, ldq, k, ldk, v, ldv, scale);
  a.o = o, a.ldo = ldo, a.lse = lse;
  return st(cross_attn_fwd(dtype, a, c.dh, ws, S(stream)));
}

uint64_t atom_k_cross_attn_bwd_ws_bytes(int dtype, const atom_cross_shape* shape) {
  return cross_ok(dtype, shape) ? cross_attn_bwd_ws(dtype, shape->B, shape->Tq, shape->Tk, shape->Hq, shape->Hk, shape->dh)
                                : 0;
}

int atom_k_cross_attn_bwd(int dtype, const atom_cross_shape* shape, const void* q, int64_t ldq, const void* k,
                          int64_t ldk, const void* v, int64_t ldv, float scale, const void* o, int64_t ldo,
                          const void* dout, int64_t lddo, const float* lse, void* dq, int64_t lddq, void* dk,
                          int64_t lddk, void* dv, int64_t lddv, void* ws, uint64_t ws_bytes, void* stream) {
  if (!cross_ok(dtype, shape) || !(scale > 0) || !isfinite(scale)) return ATOM_EINVAL;
  const atom_cross_shape& c = *shape;
  if (!side_ok(c.q_start, c.q_len, c.q_rows, c.B, c.Tq) || !side_ok(c.k_start, c.k_len, c.k_rows, c.B, c.Tk))
    return ATOM_EINVAL;
  if ((dk == nullptr) != (dv == nullptr)) return ATOM_EINVAL;
  if (c.B == 0 || (c.Tq == 0 && c.Tk == 0) || (!dq && !dk)) return ATOM_OK;
  if (c.Tq > 0) {
    if (!cross_rows_ok(dtype, q, ldq, c.Hq, c.dh) || !cross_rows_ok(dtype, o, ldo, c.Hq, c.dh) ||
        !cross_rows_ok(dtype, dout, lddo, c.Hq, c.dh) || !lse || !aligned_to(ATOM_F32, lse))
      return ATOM_EINVAL;
    if (dq && !cross_rows_ok(dtype, dq, lddq, c.Hq, c.dh)) return ATOM_EINVAL;
    const uint64_t need = cross_attn_bwd_ws(dtype, c.B, c.Tq, c.Tk, c.Hq, c.Hk, c.dh);
    if (need && (!ws || misaligned(ws) || ws_bytes < need)) return ATOM_EINVAL;
  }
  if (c.Tk > 0) {
    if (!cross_rows_ok(dtype, k, ldk, c.Hk, c.dh) || !cross_rows_ok(dtype, v, ldv, c.Hk, c.dh)) return ATOM_EINVAL;
    if (dk && (!cross_rows_ok(dtype, dk, lddk, c.Hk, c.dh) || !cross_rows_ok(dtype, dv, lddv, c.Hk, c.dh))) return ATOM_EINVAL;
  }
  CrossArgs a = cross_args(shape, q, ldq, k, ldk, v, ldv, scale);
  a.o = const_cast<void*>(o), a.ldo = ldo, a.dout = dout, a.lddo = lddo, a.lse = const_cast<float*>(lse);
  a.dq = dq, a.lddq = lddq, a.dk = dk, a.lddk = lddk, a.dv = dv, a.lddv = lddv;
  return st(cross_attn_bwd(dtype, a, c.dh, ws, S(stream)));
}

int64_t atom_k_colsum_part_floats(int64_t rows, int cols) { return colsum_blocks(rows) * cols; }

int atom_k_colsum(int dtype, const void* x, int64_t rows, int cols, float* out, float* part, void* stream) {
  if (!dt_ok(dtype) || !x || !out || !part) return ATOM_EINVAL;
  return st(colsum(dtype, x, rows, cols, cols, part, DT_F32, out, false, S(stream)));
}

int atom_k_xent(int dtype, const float* logits, int64_t ldz, const int32_t* tgt, void* dz, int64_t lddz,
                float* loss_rows, int64_t rows, int V, float scale, void* stream) {
  if (!dt_ok(dtype) || !logits || !tgt || !dz || !loss_rows) return ATOM_EINVAL;
  return st(xent_fwd_bwd(dtype, logits, ldz, tgt, dz, lddz, loss_rows, rows, V, scale, S(stream)));
}

uint64_t atom_k_linear_xent_fwd_ws_bytes(int dtype, int64_t rows, int V, int d) {
  return dt_ok(dtype) && linear_xent_fwd_ok(dtype, rows, V, d) ? linear_xent_fwd_ws(dtype, rows, V, d) : 0;
}

int atom_k_linear_xent_fwd(int dtype, const void* x, int64_t ldx, const void* w, int64_t ldw, const int32_t* tgt,
                           float* lse, float* loss_rows, int64_t rows, int V, int d, void* ws, uint64_t ws_bytes,
                           void* stream) {
  if (!dt_ok(dtype) || !linear_xent_fwd_ok(dtype, rows, V, d)) return ATOM_EINVAL;
  if (rows == 0) return ATOM_OK;
  if (!rows_ok(dtype, x, ldx, d) || !rows_ok(dtype, w, ldw, d)) return ATOM_EINVAL;
  if (!tgt || !lse || !loss_rows) return ATOM_EINVAL;
  if (!ws || misaligned(ws) || ws_bytes < linear_xent_fwd_ws(dtype, rows, V, d)) return ATOM_EINVAL;
  return st(linear_xent_fwd(dtype, x, ldx, w, ldw, tgt, lse, loss_rows, rows, V, d, ws, S(stream)));
}

uint64_t atom_k_linear_xent_bwd_ws_bytes(int dtype, int64_t rows, int V, int d, int piece) {
  return dt_ok(dtype) && piece >= 0 && linear_xent_ok(dtype, rows, V, d) ? linear_xent_bwd_ws(dtype, rows, V, d, piece) : 0;
}

int atom_k_linear_xent_bwd(int dtype, const void* x, int64_t ldx, const void* w, int64_t ldw, const int32_t* tgt,
                           const float* lse, const float* drow, float scale, void* dx, int64_t lddx, void* dw,
                           int64_t lddw, int dw_epi, int64_t rows, int V, int d, int piece, void* ws,
                           uint64_t ws_bytes, void* stream) {
  if (!dt_ok(dtype) || piece < 0 || !linear_xent_ok(dtype, rows, V, d)) return ATOM_EINVAL;
  if (rows > 0 && (!rows_ok(dtype, x, ldx, d) || !rows_ok(dtype, w, ldw, d) || !tgt || !lse)) return ATOM_EINVAL;
  if (rows > 0 && dx && !rows_ok(dtype, dx, lddx, d)) return ATOM_EINVAL;
  if (dw && !rows_ok(dtype, dw, lddw, d)) return ATOM_EINVAL;
  int epi;
  switch (dw_epi) {
    case ATOM_EPI_STORE: epi = EPI_SCALE; break;
    case ATOM_EPI_STORE_F32: epi = EPI_SCALE_F32; break;
    case ATOM_EPI_ACC_F32: epi = EPI_SCALE_ACC; break;
    default: return ATOM_EINVAL;
  }
  if (!dx && !dw) return ATOM_OK;
  if (rows > 0 && (!ws || misaligned(ws) || ws_bytes < linear_xent_bwd_ws(dtype, rows, V, d, piece))) return ATOM_EINVAL;
  return st(linear_xent_bwd(dtype, x, ldx, w, ldw, tgt, lse, drow, scale, dx, lddx, dw, lddw, epi, rows, V, d, piece,
                            ws, S(stream)));
}

int atom_k_embed_fwd(int dtype, const int32_t* tok, const void* wte, const void* wpe, float* x, int64_t n_tok, int T,
                     int V, int d, void* stream) {
  if (!dt_ok(dtype) || !tok || !wte || !wpe || !x || T <= 0 || V <= 0 || d <= 0) return ATOM_EINVAL;
  return st(embed_fwd(dtype, tok, wte, wpe, x, n_tok, T, V, d, S(stream)));
}

uint64_t atom_k_orthogonalize_ws_bytes(int dtype, int batch, int rows, int cols) {
  return dt_ok(dtype) && batch > 0 && orthogonalize_ok(batch, rows, cols) ? orthogonalize_ws(batch, rows, cols) : 0;
}

int atom_k_orthogonalize(int dtype, const void* g, int64_t ldg, int64_t stride_g, void* out, int64_t ldo,
                         int64_t stride_o, int out_epi, float keep, float scale, int batch, int rows, int cols,
                         const float* coef, int steps, void* ws, uint64_t ws_bytes, void* stream) {
  if (!dt_ok(dtype) || !orthogonalize_ok(batch, rows, cols)) return ATOM_EINVAL;
  if (ldg < cols || ldo < cols || stride_g < 0) return ATOM_EINVAL;
  if (out_epi != ATOM_EPI_STORE && out_epi != ATOM_EPI_STORE_F32 && out_epi != ATOM_EPI_ACC_F32) return ATOM_EINVAL;
  if (batch > 0 && (!g || !out)) return ATOM_EINVAL;
  const uintptr_t esz = dtype == ATOM_BF16 ? 2 : 4, osz = out_epi == ATOM_EPI_STORE ? esz : 4;
  if (reinterpret_cast<uintptr_t>(g) % esz || reinterpret_cast<uintptr_t>(out) % osz) return ATOM_EINVAL;
  if (batch > 1 && stride_o < (rows - 1) * ldo + cols && !(stride_o >= cols && stride_o <= ldo / batch)) return ATOM_EINVAL;
  if (steps < 0 || steps > ATOM_NS_MAX_STEPS) return ATOM_EINVAL;
  static_assert(ATOM_NS_MAX_STEPS == NS_EXPS, "steps");
  float own[3 * ATOM_NS_MAX_STEPS];
  if (!coef) {
    for (int k = 0; k < steps; ++k) own[3 * k] = 3.4445f, own[3 * k + 1] = -4.7750f, own[3 * k + 2] = 2.0315f;
    coef = own;
  }
  if (!orthogonalize_coef_ok(coef, steps)) return ATOM_EINVAL;
  if (batch == 0) return ATOM_OK;
  if (!ws || misaligned(ws) || ws_bytes < orthogonalize_ws(batch, rows, cols)) return ATOM_EINVAL;
  return st(orthogonalize(dtype, g, ldg, stride_g, out, ldo, stride_o, out_epi, keep, scale, batch, rows, cols, coef,
                          steps, ws, S(stream)));
}

int atom_k_copy(const void* src, void* dst, int64_t bytes, void* stream) {
  if (!src || !dst || bytes < 0 || bytes % 16) return ATOM_EINVAL;
  return st(copy_bytes(src, dst, bytes, S(stream)));
}

}  // extern "C"
